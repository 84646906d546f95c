"""The KV cache's calls where no GPU is needed: what the host refuses, sizes of
workspaces, and the addresses the kernels form (tests/c/kv_addresses.cpp)."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20  # an address that is never read


def _desc(**kw):
    from paper_2606_17059_amd import router as R
    base = dict(device=0, dtype=0, layers=2, kv_heads=2, head_dim=64, page_tokens=16, num_pages=100, num_slots=9,
                slot_pages=8, k_scale=1.0, v_scale=1.0, k=FAKE, v=FAKE, table=FAKE, lengths=FAKE, refs=FAKE,
                free_pages=FAKE, skipped=FAKE)
    base.update(kw)
    page = base["kv_heads"] * base["head_dim"] * base["page_tokens"]
    for x in ("k", "v"):
        base.setdefault(x + "_page", page)
        base.setdefault(x + "_layer", page * base["num_pages"])
    return R.KvDescription(**base)


def _calls(d, n=3, rows=5, work=FAKE, size=1 << 30):
    """Every call with arguments that pass, as (name, args)."""
    r = ctypes.byref(d) if d is not None else None
    out = ctypes.c_int64(0)
    return {
        "pr_kv_init": [r, None],
        "pr_kv_workspace": [r, 0, n, rows, ctypes.byref(out)],
        "pr_kv_extend": [r, FAKE, FAKE, n, rows, FAKE, work, size, None],
        "pr_kv_write": [r, 0, FAKE, FAKE, 128, FAKE, 128, rows, 0, None],
        "pr_kv_attend": [r, 0, FAKE, n, FAKE, 4 * 64, 4, 0, 0.125, 0, FAKE + 1536, None, work, size, None],
        "pr_kv_fork": [r, FAKE, FAKE, FAKE, n, work, size, None],
        "pr_kv_trim": [r, FAKE, FAKE, 1, n, work, size, None],
        "pr_kv_compact": [r, None, work, size, None],
        "pr_kv_check": [r, None],
    }


@pytest.mark.parametrize("what", [
    dict(dtype=3), dict(dtype=-1), dict(device=-1), dict(layers=0), dict(kv_heads=0), dict(head_dim=80),
    dict(head_dim=512), dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=512), dict(num_pages=0),
    dict(num_slots=0), dict(slot_pages=0), dict(num_pages=1 << 27), dict(slot_pages=(1 << 26) + 1), dict(k=None),
    dict(layers=1 << 30), dict(kv_heads=1 << 21), dict(v=FAKE + 8), dict(table=None), dict(lengths=None), dict(refs=None), dict(free_pages=None),
    dict(skipped=None), dict(k_page=2044), dict(k_page=2040), dict(v_layer=-8), dict(v_layer=2040),
    dict(k_scale=0.5), dict(v_scale=float("nan")), dict(dtype=2, k_scale=0.0), dict(dtype=2, v_scale=float("inf")),
    dict(dtype=2, k_page=2056), None])
def test_a_bad_description_is_refused_by_every_call(what):
    """Before any device work: there is no GPU here."""
    from paper_2606_17059_amd import router as R
    d = None if what is None else _desc(**what)
    for name, args in _calls(d).items():
        assert getattr(R.lib(), name)(*args) == R.PR_EINVAL, (name, what)
        assert R.pr_last_error()


def test_the_binding_lays_out_the_description_as_the_header():
    import re
    from paper_2606_17059_amd import router as R
    src = open(os.path.join(ROOT, "include", "prefix_router.h")).read()
    body = re.findall(r"typedef struct \{([^}]*)\} pr_kv;", src, flags=re.S)[0]
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    names = []
    for kind, rest in re.findall(r"(int32_t|int64_t|uint64_t|float|void)\s+([^;]+);", body):
        names += [(x.strip().lstrip("*"), x.strip().startswith("*"), kind) for x in rest.split(",")]
    kinds = {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float}
    assert [(n, ctypes.c_void_p if p else kinds[k]) for n, p, k in names] == list(R.KvDescription._fields_)


BAD = [  # call, index of an argument, a value it refuses
    ("pr_kv_workspace", 1, 4), ("pr_kv_workspace", 2, -1), ("pr_kv_workspace", 3, 1 << 31),
    ("pr_kv_workspace", 4, None),
    ("pr_kv_extend", 1, None), ("pr_kv_extend", 2, None), ("pr_kv_extend", 3, -1), ("pr_kv_extend", 4, -1),
    ("pr_kv_extend", 3, 1 << 31), ("pr_kv_extend", 4, 1 << 31), ("pr_kv_extend", 5, None), ("pr_kv_extend", 6, None),
    ("pr_kv_extend", 6, FAKE + 4), ("pr_kv_extend", 7, 8),
    ("pr_kv_write", 1, -1), ("pr_kv_write", 1, 2), ("pr_kv_write", 2, None), ("pr_kv_write", 3, None),
    ("pr_kv_write", 3, FAKE + 1), ("pr_kv_write", 4, 127), ("pr_kv_write", 5, None), ("pr_kv_write", 6, 0),
    ("pr_kv_write", 7, -1), ("pr_kv_write", 8, 1), ("pr_kv_write", 8, 2),
    ("pr_kv_attend", 1, 2), ("pr_kv_attend", 2, None), ("pr_kv_attend", 3, -1), ("pr_kv_attend", 3, 1 << 24),
    ("pr_kv_attend", 4, None), ("pr_kv_attend", 4, FAKE + 1), ("pr_kv_attend", 5, 255), ("pr_kv_attend", 6, 3),
    ("pr_kv_attend", 6, 0), ("pr_kv_attend", 7, 1), ("pr_kv_attend", 8, float("nan")),
    ("pr_kv_attend", 8, float("inf")), ("pr_kv_attend", 8, 3e38), ("pr_kv_attend", 9, -1), ("pr_kv_attend", 10, None),
    ("pr_kv_attend", 10, FAKE + 8), ("pr_kv_attend", 10, FAKE + 1024), ("pr_kv_attend", 10, FAKE - 1024),
    ("pr_kv_fork", 1, None), ("pr_kv_fork", 2, None), ("pr_kv_fork", 3, None), ("pr_kv_fork", 4, -1),
    ("pr_kv_fork", 4, 65537),
    ("pr_kv_trim", 1, None), ("pr_kv_trim", 3, -1), ("pr_kv_trim", 4, -1), ("pr_kv_trim", 4, 1 << 22),
    ("pr_kv_compact", 2, None), ("pr_kv_compact", 2, FAKE + 4), ("pr_kv_compact", 3, 16),
]


@pytest.mark.parametrize("name,index,value", BAD)
def test_a_bad_argument_is_refused(name, index, value):
    from paper_2606_17059_amd import router as R
    d = _desc()
    args = _calls(d)[name]
    args[index] = value
    assert getattr(R.lib(), name)(*args) == R.PR_EINVAL
    assert R.pr_last_error()


def test_a_score_scale_past_float_is_refused():
    from paper_2606_17059_amd import router as R
    d = _desc(dtype=2, k_scale=1e30)
    args = _calls(d)["pr_kv_attend"]
    args[8] = 1e10
    assert R.lib().pr_kv_attend(*args) == R.PR_EINVAL
    assert "scale times k_scale" in R.pr_last_error()


def test_an_attention_that_splits_wants_its_workspace():
    from paper_2606_17059_amd import router as R
    L, need = R.lib(), ctypes.c_int64(0)
    for slot_pages, splits in ((1, False), (16, False), (1 << 12, True)):  # short sequences are not split
        d = _desc(slot_pages=slot_pages)
        assert L.pr_kv_workspace(ctypes.byref(d), 1, 3, 4, ctypes.byref(need)) == R.PR_OK
        assert (need.value > 0) == splits
        if splits:
            for work, size in ((None, need.value), (FAKE, need.value - 1), (FAKE + 8, need.value)):
                assert L.pr_kv_attend(*_calls(d, work=work, size=size)["pr_kv_attend"]) == R.PR_EINVAL
    assert L.pr_kv_workspace(ctypes.byref(_desc()), 1, 3, 5, ctypes.byref(need)) == R.PR_EINVAL  # 5 heads over 2


def test_large_forks_and_trims_want_their_workspace():
    from paper_2606_17059_amd import router as R
    L, need, d = R.lib(), ctypes.c_int64(0), _desc(slot_pages=1 << 12, num_slots=100)
    for n, large in ((15, False), (31, False), (32, True)):
        assert L.pr_kv_workspace(ctypes.byref(d), 3, n, 0, ctypes.byref(need)) == R.PR_OK
        assert (need.value > 0) == large
    for work, size in ((None, need.value), (FAKE, need.value - 1), (FAKE + 8, need.value)):
        calls = _calls(d, n=32, work=work, size=size)
        for name in ("pr_kv_fork", "pr_kv_trim"):
            assert getattr(L, name)(*calls[name]) == R.PR_EINVAL
    assert L.pr_kv_workspace(ctypes.byref(d), 3, 1 << 22, 0, ctypes.byref(need)) == R.PR_EINVAL


def test_empty_batches_do_nothing():
    """Zero entries need no pointers and no GPU."""
    from paper_2606_17059_amd import router as R
    L, d = R.lib(), _desc()
    r = ctypes.byref(d)
    assert L.pr_kv_extend(r, None, None, 0, 0, None, None, 0, None) == R.PR_OK
    assert L.pr_kv_write(r, 0, None, None, 0, None, 0, 0, 0, None) == R.PR_OK
    assert L.pr_kv_attend(r, 0, None, 0, None, 0, 4, 0, 1.0, 0, None, None, None, 0, None) == R.PR_OK
    assert L.pr_kv_fork(r, None, None, None, 0, None, 0, None) == R.PR_OK
    assert L.pr_kv_trim(r, None, None, 0, 0, None, 0, None) == R.PR_OK


def test_the_binding_takes_device_tensors_only():
    import torch
    from paper_2606_17059_amd import KVCache
    k, v = torch.zeros(1, 2, 1, 8, 16, 8).bfloat16(), torch.zeros(1, 2, 1, 4, 64, 4).bfloat16()
    ints = [torch.zeros(s, dtype=t) for s, t in (((3, 2), torch.int32), ((3,), torch.int32), ((2,), torch.int32),
                                                 ((1,), torch.int64))]
    with pytest.raises(TypeError):
        KVCache(k, v, *ints)


def test_addresses_stay_inside_their_pages(tmp_path):
    exe = str(tmp_path / "kv_addresses")
    cmd = ["g++", "-std=c++17", "-O2", "-Wall", "-Wextra", "-Werror", "-I",
           os.path.join(ROOT, "paper_2606_17059_amd", "csrc"), os.path.join(ROOT, "tests", "c", "kv_addresses.cpp"),
           "-o", exe]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=120)
    assert r.returncode == 0 and "kv_addresses: ok" in r.stdout, r.stdout

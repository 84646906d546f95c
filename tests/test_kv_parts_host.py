"""Where an attention's parts are kept (tests/c/kv_kept.cpp), and how much workspace that takes.  No GPU."""
import ctypes
import os
import subprocess

from test_kv_host import _desc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_parts_are_kept_apart_and_found_again(tmp_path):
    exe = str(tmp_path / "kv_kept")
    cmd = ["g++", "-std=c++17", "-O2", "-Wall", "-Wextra", "-Werror", "-I",
           os.path.join(ROOT, "paper_2606_17059_amd", "csrc"), os.path.join(ROOT, "tests", "c", "kv_kept.cpp"), "-o", exe]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=120)
    assert r.returncode == 0 and "kv_kept: ok" in r.stdout, r.stdout


def test_an_attentions_workspace_does_not_grow_with_its_output():
    """What is joined are parts of as many shares as the GPU has room for, not a part of every sequence."""
    from paper_2606_17059_amd import router as R
    for n, heads, kv_heads, dim in ((4096, 64, 8, 128), (256, 768, 1, 256), (100000, 16, 4, 64)):
        d = _desc(num_slots=n, slot_pages=1 << 12, kv_heads=kv_heads, head_dim=dim)
        need = ctypes.c_int64(0)
        assert R.lib().pr_kv_workspace(ctypes.byref(d), 1, n, heads, ctypes.byref(need)) == R.PR_OK
        ints = 20 * n + 64  # first parts, their numbers and the plan
        # at most four parts a share, and as many shares of a head as 256 units hold of the smallest workgroups
        assert need.value - ints <= 4 * 256 * 5 * (heads // kv_heads) * 4 * (dim + 2) + 64, (n, need.value)

"""The KV cache on the GPU against its plain model (tests/kv_model.py): pages,
tables and counts exactly, rows bit for bit, attention within what float32 sums
and one rounding of the output allow."""
import math
import os

import numpy as np
import pytest

import kv_model
from gpu_util import announce, device

pytestmark = pytest.mark.gpu


def _t(x, dtype):
    import torch
    return torch.tensor(x, dtype=dtype, device=device())


def _ints(x):
    import torch
    return _t(list(x), torch.int32)


def _offsets(counts):
    import torch
    return _t([0] + np.cumsum(counts).tolist(), torch.int64)


def _types():
    import torch
    return {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}


def _cache(layers=1, heads=2, dim=64, page=16, pages=40, slots=6, slot_pages=12, kind="bf16", **kw):
    from paper_2606_17059_amd import KVCache
    return KVCache.create(layers, heads, dim, page, pages, slots, slot_pages, _types()[kind], device(), **kw)


def _poison(c):
    """NaN wherever nothing was written: no result may take a number from there."""
    import torch
    for t in (c.k, c.v):
        t.view(torch.uint8).fill_(0xff)  # a NaN in bfloat16, float16 and e4m3


def _rows_of(c, layer, slot):
    """(k, v) of a sequence as float64 [tokens, kv_heads, dim], read from the pages by the layout's definition."""
    n = int(c.lengths[slot])
    T, D, H = c.page_tokens, c.head_dim, c.kv_heads
    pages = c.table[slot, :-(-n // T)].long().tolist()
    k = np.zeros((n, H, D))
    v = np.zeros((n, H, D))
    for j, p in enumerate(pages):
        m = min(T, n - j * T)
        kp = c.k[layer, p].float().cpu().double().numpy()  # [H, D / 8, T, 8]
        vp = c.v[layer, p].float().cpu().double().numpy()  # [H, T / 4, D, 4]
        k[j * T:j * T + m] = kp.transpose(2, 0, 1, 3).reshape(T, H, D)[:m]
        v[j * T:j * T + m] = vp.transpose(1, 3, 0, 2).reshape(T, H, D)[:m]
    return k * c.k_scale, v * c.v_scale


def _fill(c, lengths, seed=0, io=None):
    """Sequences of random rows in slots 0.. (through extend and write); returns (k, v) per layer as written."""
    import torch
    total = sum(lengths)
    place = c.extend(_ints(range(len(lengths))), _offsets(lengths), total)
    g = torch.Generator(device=device()).manual_seed(seed)
    io = io or (c.dtype if c.dtype.itemsize == 2 else torch.bfloat16)
    for layer in range(c.layers):
        k, v = (torch.empty((total, c.kv_heads, c.head_dim), device=device()).normal_(generator=g).to(io) for _ in "kv")
        c.write(layer, place, k, v)
    return place


def _check_attend(c, layer, slots, q, scale, window, out, lse):
    """Compare with float64; q's dtype's half step is eps / 2 relative to the value."""
    import torch
    half = torch.finfo(out.dtype).eps / 2
    tiny = torch.finfo(out.dtype).tiny * half * 2  # half a step below the normal numbers, rounded up
    o = out.double().cpu().numpy()
    ls = lse.double().cpu().numpy() if lse is not None else None
    for i, s in enumerate(slots):
        k, v = _rows_of(c, layer, s) if 0 <= s < c.lengths.numel() else (np.zeros((0, c.kv_heads, c.head_dim)),) * 2
        if window:
            k, v = k[-window:], v[-window:]
        ro, rl, err, lerr = kv_model.attend(q[i].double().cpu().numpy(), k, v, scale)
        bound = err + half * (np.abs(ro) + err) + tiny
        assert (np.abs(o[i] - ro) <= bound).all(), (i, s, len(k), np.max(np.abs(o[i] - ro) / bound))
        if ls is not None:
            if len(k) == 0:
                assert (ls[i] == -math.inf).all()
            else:
                assert (np.abs(ls[i] - rl) <= lerr).all(), (i, s, np.max(np.abs(ls[i] - rl) / lerr))


def _attend_case(kind, dim, page, heads, group, lengths, window=0, io=None, scale=None, seed=3, slot_pages=None):
    import torch
    announce(f"attend {kind} dim {dim} page {page} heads {heads}x{group} lengths {lengths[:8]} window {window}")
    need = [-(-n // page) for n in lengths]
    c = _cache(1, heads, dim, page, sum(need) + 2, len(lengths) + 1, slot_pages or max(max(need), 1), kind,
               **(dict(k_scale=0.5, v_scale=0.125) if kind == "e4m3" else {}))
    _poison(c)
    _fill(c, lengths, seed, io)
    io = io or (c.dtype if kind != "e4m3" else torch.bfloat16)
    g = torch.Generator(device=device()).manual_seed(seed + 1)
    q = torch.empty((len(lengths), heads * group, dim), device=device()).normal_(0, 2.0, generator=g).to(io)
    lse = torch.empty((len(lengths), heads * group), dtype=torch.float32, device=device())
    scale = dim ** -0.5 if scale is None else scale
    out = c.attend(0, _ints(range(len(lengths))), q, scale, window=window, lse=lse)
    _check_attend(c, 0, list(range(len(lengths))), q, scale, window, out, lse)
    c.check()
    return c, q, out, lse


@pytest.mark.parametrize("kind", ["bf16", "fp16", "e4m3"])
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
def test_attend_types_and_dims(kind, dim):
    _attend_case(kind, dim, 16, 2, 3, [1, 15, 16, 17, 33, 0, 128, 200])


@pytest.mark.parametrize("dim", [64, 192, 256])
@pytest.mark.parametrize("group", [1, 15, 16, 17, 33, 70])
def test_attend_groups(dim, group):
    """Query heads of a key head across the rows of one workgroup and of several."""
    _attend_case("bf16", dim, 32, 1, group, [5, 300, 64])


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("window", [0, 1, 31, 33, 257])
def test_attend_pages_and_windows(page, window):
    _attend_case("fp16", 64, page, 3, 2, [0, 1, 31, 32, 33, 255, 256, 257, 511, 700], window=window)


@pytest.mark.parametrize("kind,io", [("e4m3", "fp16"), ("bf16", None), ("fp16", None)])
def test_attend_split_lengths(kind, io):
    """Sequences cut into several chunks, next to short and empty ones."""
    _attend_case(kind, 128, 64, 2, 4, [3000, 1, 0, 5000, 255, 256, 257, 512, 513, 1025], io=_types()[io] if io else None)


@pytest.mark.parametrize("kind", ["bf16", "fp16", "e4m3"])
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("group", [3, 20])
def test_attend_shares(kind, dim, group):
    """Tables with room for long sequences: shares that end inside sequences, go on to the next ones and meet empty
    ones, for one sixteen of query heads and for two."""
    _attend_case(kind, dim, 16, 2, group, [2000, 1, 0, 0, 700, 129, 128, 127, 0, 3000, 0], slot_pages=500)
    _attend_case(kind, dim, 32, 1, group, [1500, 0, 40], window=600, slot_pages=300)


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 128, 129, 256, 257, 600])
def test_attend_batch_sizes(n):
    """Batches around the sizes where a wave looks through another 64 lengths, and past which a launch of its own
    does; most sequences short, so that with 16 key heads shares keep to them."""
    lengths = [(37 * i) % 300 for i in range(n)]
    _attend_case("bf16", 64, 16, 1, 2, lengths, slot_pages=100)
    _attend_case("fp16", 64, 16, 16, 1, lengths[:-1] + [1300], slot_pages=100)


def test_attend_one_long_sequence_and_many_short_ones():
    _attend_case("bf16", 64, 16, 1, 8, [40000])
    _attend_case("bf16", 64, 16, 1, 2, [17] * 300 + [3000] + [0] * 20)  # more entries than a wave looks through


def test_attend_one_page_of_room_has_nothing_to_split():
    _attend_case("bf16", 128, 256, 2, 4, [256, 1, 0, 100], slot_pages=1)


@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
def test_attend_scales(scale):
    """Scores of hundreds, all equal, and reversed."""
    _attend_case("bf16", 64, 16, 2, 2, [100, 700], scale=scale)


def test_attend_padding_and_unknown_slots():
    import torch
    c, q, out, lse = _attend_case("bf16", 64, 16, 2, 2, [20, 600, 3])
    announce("attend with padded, repeated and unknown slots")
    slots = [1, -1, 1, 77, 0, -2]
    q2 = torch.cat([q, q])
    out = torch.full_like(q2, 9.0)
    lse = torch.full((6, 4), 9.0, device=device())
    c.attend(0, _ints(slots), q2, 0.125, out=out, lse=lse)
    _check_attend(c, 0, slots, q2, 0.125, 0, out, lse)
    for i in (1, 3, 5):
        assert (out[i] == 0).all() and (lse[i] == -math.inf).all()
    with pytest.raises(Exception, match="2 batch entries"):
        c.check()
    c.check()


def test_attend_bad_pages_are_left_out():
    """Table entries out of range (the caller's memory, so they can be anything): their tokens do not count."""
    import torch
    c, q, _, _ = _attend_case("bf16", 64, 16, 2, 2, [100, 600, 3])
    announce("attend with table entries out of range")
    full = [_rows_of(c, 0, s) for s in range(3)]
    c.table[0, 2] = c.pages
    c.table[1, 0] = -1
    c.table[1, 20] = 2 ** 31 - 1
    c.table[2, 0] = -2 ** 31
    out = c.attend(0, _ints([0, 1, 2]), q, 0.125)
    for i, gone in enumerate(([2], [0, 20], [0])):
        stay = [t for t in range(len(full[i][0])) if t // 16 not in gone]
        ro, _, err, _ = kv_model.attend(q[i].double().cpu().numpy(), full[i][0][stay], full[i][1][stay], 0.125)
        o = out[i].double().cpu().numpy()
        if stay:
            assert (np.abs(o - ro) <= err + 2.0 ** -8 * (np.abs(ro) + err)).all()
        else:
            assert (o == 0).all()  # as a sequence without tokens


def test_attend_infinite_and_nan_numbers():
    """Keys that are infinite give what the formula gives, a value that is not finite a dimension that is not; behind
    the end and before the window nothing of them is seen."""
    import torch
    c, q, out, lse = _attend_case("fp16", 64, 16, 1, 2, [40, 40, 40, 600])
    announce("attend with infinities")
    page = c.table[:, 0].tolist()
    kv = lambda s, t: (int(c.table[s, t // 16]), t % 16)  # noqa: E731
    q[:, :, 0] = 1.0
    before = c.attend(0, _ints(range(4)), q, 0.125).clone()
    p, t = kv(0, 7)
    c.k[0, p, 0, 0, t, 0] = -math.inf  # a score of -inf: weight 0
    p, t = kv(1, 39)
    c.k[0, p, 0, 0, t, 0] = math.inf  # a score of +inf: inf - inf
    p, t = kv(2, 3)
    c.v[0, p, 0, t // 4, 5, t % 4] = math.nan
    p, t = kv(3, 11)
    c.v[0, p, 0, t // 4, 9, t % 4] = math.inf
    out = c.attend(0, _ints(range(4)), q, 0.125)
    k, v = _rows_of(c, 0, 0)
    stay = [x for x in range(40) if x != 7]
    ro, _, err, _ = kv_model.attend(q[0].double().cpu().numpy(), k[stay], v[stay], 0.125)
    assert (np.abs(out[0].double().cpu().numpy() - ro) <= err + 2.0 ** -11 * (np.abs(ro) + err)).all()
    assert out[1].isnan().all()
    assert out[2, :, 5].isnan().all() and torch.equal(out[2, :, 6:], before[2, :, 6:])
    assert not out[3, :, 9].isfinite().any() and torch.equal(out[3, :, 10:], before[3, :, 10:])
    w = c.attend(0, _ints([2, 3]), q[2:], 0.125, window=20)
    assert w.isfinite().all()


def test_attend_a_window_past_every_length_is_none():
    import torch
    c, q, _, _ = _attend_case("bf16", 64, 16, 2, 2, [1, 40, 600])
    announce("attend with wide windows")
    want = c.attend(0, _ints(range(3)), q, 0.125)
    for window in (2 ** 31 - 1, 2 ** 31, 2 ** 32 + 1, 2 ** 40):
        assert torch.equal(c.attend(0, _ints(range(3)), q, 0.125, window=window), want)


def test_attend_all_scores_minus_infinity():
    import torch
    c, q, _, _ = _attend_case("bf16", 64, 16, 1, 2, [40, 600])
    announce("attend where every score is -inf")
    c.k.fill_(-math.inf)
    q.fill_(0.0)
    q[:, :, 3] = 1.0
    c.k[:, :, :, 1:] = 0
    c.k[:, :, :, 0, :, :3] = 0
    c.k[:, :, :, 0, :, 4:] = 0
    lse = torch.zeros((2, q.shape[1]), device=device())
    out = c.attend(0, _ints([0, 1]), q, 0.125, lse=lse)
    assert (out == 0).all() and (lse == -math.inf).all()  # as rows without tokens


def test_attend_strides_and_alignment():
    """Queries inside a fused projection's rows, at any 2-byte address."""
    import torch
    c, q, out, _ = _attend_case("bf16", 96, 16, 2, 3, [50, 700, 9])
    announce("attend on strided queries")
    for lead in (0, 1, 8, 13):
        wide = torch.full((3, lead + 6 * 96 + 57), 7.0, dtype=torch.bfloat16, device=device())
        view = wide[:, lead:lead + 576].unflatten(1, (6, 96))
        view.copy_(q)
        assert torch.equal(c.attend(0, _ints([0, 1, 2]), view, 96 ** -0.5), out)


def test_attend_nothing():
    import torch
    announce("an attention of no sequence")
    c = _cache()
    q = torch.zeros((0, 4, 64), dtype=torch.bfloat16, device=device())
    assert c.attend(0, _ints([]), q).shape == (0, 4, 64)
    place = c.extend(_ints([3]), _offsets([0]), 0)
    c.write(0, place, q[:, :2], q[:, :2])
    c.fork(_ints([]), _ints([]), _ints([]))
    c.trim(_ints([]))
    assert c.compact().tolist() == [0, 0]
    c.check()


def test_attend_is_the_same_every_time_and_whatever_else_is_in_the_batch():
    import torch
    c, q, out, lse = _attend_case("bf16", 128, 16, 2, 4, [5000, 70, 900])
    announce("attend again")
    for _ in range(3):
        assert torch.equal(c.attend(0, _ints([0, 1, 2]), q, 128 ** -0.5), out)


def test_attend_pages_past_32_bits():
    """Pages whose numbers lie beyond 2^32 elements."""
    import torch
    from paper_2606_17059_amd import KVCache
    announce("attend beyond 2^32 elements")
    H, D, T = 8, 128, 256
    P = 2 ** 32 // (H * D * T) + 40
    c = KVCache.create(1, H, D, T, P, 2, 4, torch.bfloat16, device())
    c.refs.fill_(1)  # nothing but the last pages is free
    c.refs[P - 8:] = 0
    words = np.zeros((P + 63) // 64, np.uint64)
    for p in range(P - 8, P):
        words[p // 64] |= np.uint64(1) << np.uint64(p % 64)
    c.free.copy_(torch.from_numpy(words.view(np.int64)))
    _fill(c, [700, 300])
    assert c.table[0, :3].tolist() == [P - 8, P - 7, P - 6] and c.table[1, 0].item() == P - 5
    q = torch.randn((2, 8, D), device=device()).bfloat16()
    out = c.attend(0, _ints([0, 1]), q, 0.1)
    _check_attend(c, 0, [0, 1], q, 0.1, 0, out, None)
    c.trim(_ints([1]))
    m = c.compact()
    assert m.tolist() == [0, P - 5]
    del c
    torch.cuda.empty_cache()


# ---- rows -----------------------------------------------------------------------
@pytest.mark.parametrize("kind,io", [("bf16", "bf16"), ("fp16", "fp16"), ("e4m3", "bf16"), ("e4m3", "fp16")])
@pytest.mark.parametrize("counts", [[1, 1, 1], [3, 1, 40], [0, 17, 64], [5, 0, 0]])
def test_write_rows(kind, io, counts):
    """Rows arrive where extend said, in every layer, bit for bit; e4m3 by the nearest value."""
    import torch
    announce(f"write {kind} from {io}, {counts}")
    c = _cache(2, 3, 96, 16, 30, 4, 8, kind, **(dict(k_scale=0.3, v_scale=2.0) if kind == "e4m3" else {}))
    _poison(c)
    _fill(c, [2, 7, 16], io=_types()[io])
    before = [[_rows_of(c, layer, s) for s in range(3)] for layer in range(2)]
    total = sum(counts)
    place = c.extend(_ints([0, 1, 2]), _offsets(counts), total)
    rows = torch.randn((2, total, 2, 3, 96), device=device()).to(_types()[io]) * 3
    if total:
        rows[0, 0, 0, 0, :5] = torch.tensor([0.0, 1e4, -1e4, 1e-4, -1e-3], device=device())
    for layer in range(2):
        c.write(layer, place, rows[layer, :, 0], rows[layer, :, 1])
    at = np.cumsum([0] + counts)
    for layer in range(2):
        want = rows[layer].float().cpu().double().numpy()
        if kind == "e4m3":  # the quotient is a float32 number
            unit = np.array([0.3, 2.0], np.float32)[:, None, None]
            want = kv_model.e4m3((want.astype(np.float32) / unit).astype(np.float64)) * unit.astype(np.float64)
        for s in range(3):
            k, v = _rows_of(c, layer, s)
            old = before[layer][s]
            got = want[at[s]:at[s + 1]]
            if kind == "e4m3":  # the scales of _rows_of are the float64 ones
                np.testing.assert_allclose(k, np.concatenate([old[0], got[:, 0]]), rtol=2.0 ** -20)
                np.testing.assert_allclose(v, np.concatenate([old[1], got[:, 1]]), rtol=2.0 ** -20)
            else:
                assert np.array_equal(k, np.concatenate([old[0], got[:, 0]]))
                assert np.array_equal(v, np.concatenate([old[1], got[:, 1]]))


def test_write_every_e4m3_border():
    """All 16-bit numbers against the definition: ties, subnormals, the range's end, infinities and NaN."""
    import torch
    for io in ("bf16", "fp16"):
        announce(f"every {io} number as e4m3")
        c = _cache(1, 4, 256, 256, 1, 1, 1, "e4m3")
        place = c.extend(_ints([0]), _offsets([64]), 64)
        bits = torch.arange(65536, device=device()).to(torch.int16).view(_types()[io]).view(64, 4, 256)
        c.write(0, place, bits, bits)
        x = bits.float().cpu().double().numpy()
        with np.errstate(invalid="ignore"):
            want = np.where(np.isnan(x), np.nan, kv_model.e4m3(np.nan_to_num(x, nan=0.0, posinf=1e9, neginf=-1e9)))
        for got in _rows_of(c, 0, 0):
            assert np.array_equal(got, want, equal_nan=True)


def test_write_strides_alignment_and_left_out_rows():
    import torch
    announce("write from strided rows, some of them nowhere")
    c = _cache(1, 2, 64, 16, 10, 2, 5)
    place = c.extend(_ints([0]), _offsets([37]), 37)
    rows = torch.randn((37, 2, 64), device=device()).bfloat16()
    for lead, tail in ((0, 0), (3, 10), (8, 8), (16, 7)):
        _poison(c)
        wide = torch.zeros((37, lead + 128 + tail), dtype=torch.bfloat16, device=device())
        view = wide[:, lead:lead + 128].unflatten(1, (2, 64))
        view.copy_(rows)
        c.write(0, place, view, rows)
        for got in _rows_of(c, 0, 0):
            assert np.array_equal(got, rows.double().cpu().numpy())
    k0, v0 = c.k.clone(), c.v.clone()
    bad = torch.tensor([-1, 10 * 16, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device=device())
    c.write(0, bad, rows[:4], rows[:4])
    assert torch.equal(c.k.view(torch.int16), k0.view(torch.int16))
    assert torch.equal(c.v.view(torch.int16), v0.view(torch.int16))
    c.write(0, place[:0], rows[:0], rows[:0])


def test_write_pages_with_their_layers_together():
    """k and v whose layers of a page lie together (strides of another order)."""
    import torch
    from paper_2606_17059_amd import KVCache
    announce("a cache of another order")
    L, P, H, D, T = 3, 20, 2, 64, 16
    k = torch.zeros((P, L, H, D // 8, T, 8), dtype=torch.bfloat16, device=device()).transpose(0, 1)
    v = torch.zeros((P, L, H, T // 4, D, 4), dtype=torch.bfloat16, device=device()).transpose(0, 1)
    a = _cache(L, H, D, T, P, 4, 6)
    ints = [torch.empty_like(t) for t in (a.table, a.lengths, a.refs, a.free)]
    b = KVCache(k, v, *ints)
    b.init()
    for c in (a, b):
        _fill(c, [50, 20, 5], seed=5)
        c.fork(_ints([0, 0]), _ints([3, 1]), _ints([37, 1]))  # slot 1 is taken: skipped
        c.trim(_ints([1]))
        c.extend(_ints([3]), _offsets([2]), 2)
        c.compact()
    for s in (0, 2):
        for layer in range(L):
            for x, y in zip(_rows_of(a, layer, s), _rows_of(b, layer, s)):
                assert np.array_equal(x, y)
    assert np.array_equal(_rows_of(b, 2, 3)[0][:37], _rows_of(b, 2, 0)[0][:37])
    q = torch.randn((3, 4, D), device=device()).bfloat16()
    for layer in range(L):
        out = b.attend(layer, _ints([0, 2, 2]), q, 0.1)
        assert torch.equal(out, a.attend(layer, _ints([0, 2, 2]), q, 0.1))


# ---- pages --------------------------------------------------------------------------
def _same(c, m, what):
    assert c.lengths.tolist() == m.length, what
    assert c.refs.tolist() == m.refs, what
    assert np.array_equal(c.table.cpu().numpy(), m.table_array()), what
    assert np.array_equal(c.free.cpu().numpy(), m.free_words()), what


def _row(ids, heads, dim, layer, base):
    """Rows that tell their id, layer and dimension (bfloat16 holds these numbers exactly)."""
    import torch
    x = torch.tensor(ids, dtype=torch.int64, device=device())
    d = torch.arange(heads * dim, device=device())
    n = (x[:, None] * 31 + d[None] * 7 + layer * 13 + base * 101) % 251
    return n.to(torch.bfloat16).view(len(ids), heads, dim)


def _content_same(c, m, slots, what):
    for s in slots:
        ids = m.rows(s)
        if not ids:
            continue
        for layer in range(c.layers):
            k, v = _rows_of(c, layer, s)
            assert np.array_equal(k, _row(ids, c.kv_heads, c.head_dim, layer, 0).double().cpu().numpy()), (what, s, layer)
            assert np.array_equal(v, _row(ids, c.kv_heads, c.head_dim, layer, 1).double().cpu().numpy()), (what, s, layer)


@pytest.mark.parametrize("seed,page,pages,slots,slot_pages,batch", [
    (0, 16, 40, 12, 9, 6), (1, 16, 200, 40, 12, 30), (2, 64, 30, 20, 4, 10), (3, 32, 1, 3, 1, 3), (4, 16, 129, 60, 30, 50)])
def test_random_calls_match_the_model(seed, page, pages, slots, slot_pages, batch):
    """Extends, writes, forks, trims and compactions in random order, valid and invalid entries mixed, pools that run
    dry: tables, counts, free bits, places and every sequence's rows after each call."""
    import torch
    rng = np.random.default_rng(seed)
    c = _cache(2, 2, 64, page, pages, slots, slot_pages)
    _poison(c)
    m = kv_model.Pages(page, pages, slots, slot_pages)
    fresh = 0
    for step in range(60):
        what = rng.choice(["extend"] * 4 + ["fork"] * 2 + ["trim"] * 2 + ["compact"])
        n = int(rng.integers(1, batch + 1))
        announce(f"step {step}: {what} {n}")
        if what == "extend":
            s = rng.integers(-2, slots + 1, n) if rng.random() < 0.3 else rng.permutation(slots)[:n]
            s = s.tolist()
            counts = rng.choice([0, 1, 1, 1, 2, 5, page, 2 * page + 3], len(s)).tolist()
            off = [0] + np.cumsum(counts).tolist()
            rows = off[-1] + int(rng.integers(0, 3))  # rows of no entry
            place = c.extend(_ints(s), _t(off, torch.int64), rows)
            want = m.extend(s, off, rows)
            assert place.tolist() == want, step
            ids = list(range(fresh, fresh + rows))
            fresh += rows
            for layer in range(2):
                if rows:
                    c.write(layer, place, _row(ids, 2, 64, layer, 0), _row(ids, 2, 64, layer, 1))
            m.write(want, ids)
        elif what == "fork":
            src, dst = rng.integers(0, slots, n).tolist(), rng.integers(-1, slots, n).tolist()
            tokens = [int(rng.integers(0, m.length[a] + 1)) if rng.random() < 0.9 else m.length[a] + 1 for a in src]
            if rng.random() < 0.2:
                src[0], dst[-1] = slots, -3
            c.fork(_ints(src), _ints(dst), _ints(tokens))
            m.fork(src, dst, tokens)
        elif what == "trim":
            s = rng.integers(-1, slots, n).tolist()
            if rng.random() < 0.5:
                keep = [int(rng.integers(-1 if rng.random() < 0.1 else 0, slot_pages * page)) for _ in s]
                wide = torch.tensor([[0, k, 0] for k in keep], dtype=torch.int32, device=device())
                c.trim(_ints(s), wide[:, 1])
            else:
                keep = [0] * len(s)
                c.trim(_ints(s))
            m.trim(s, keep)
        else:
            assert c.compact().tolist() == m.compact(), step
        _same(c, m, (step, what))
        assert int(c.skipped) == m.skipped, (step, what)
        if step % 7 == 0 or what == "compact":
            _content_same(c, m, range(slots), (step, what))
    _content_same(c, m, range(slots), "end")


@pytest.mark.parametrize("n,slot_pages,parents", [(40, 4000, 3), (600, 700, 5), (1100, 130, 40)])
def test_large_forks_and_trims(n, slot_pages, parents):
    """Batches whose tables have many pages: counts that forks of one sequence change together, more sequences than
    a column has places for, entries past a workgroup's, and entries that are skipped among them."""
    import torch
    announce(f"fork and trim {n} entries of {parents} sequences")
    rng = np.random.default_rng(n)
    T, slots = 16, parents + n + 3
    held = rng.integers(slot_pages * T // 2, slot_pages * T, parents).tolist()
    P = sum(-(-x // T) for x in held) + 2 * n
    c = _cache(1, 1, 64, T, P, slots, slot_pages)
    m = kv_model.Pages(T, P, slots, slot_pages)
    junk = rng.permutation(slots)[:parents].tolist()  # scattered pages: some are taken and given back first
    for k in range(2):
        off = [0] + np.cumsum(held).tolist()
        s = junk if k == 0 else list(range(parents))
        assert c.extend(_ints(s), _t(off, torch.int64), off[-1]).tolist() == m.extend(s, off, off[-1])
        if k == 0:
            c.trim(_ints(s))
            m.trim(s, [0] * parents)
    src = rng.integers(0, parents, n).tolist()
    dst = list(range(parents, parents + n))
    tokens = [int(rng.integers(0, held[a] + 1)) for a in src]
    tokens[3], dst[5], src[7], dst[9], dst[11] = held[src[3]] + 1, -1, slots, dst[8], src[11]
    c.fork(_ints(src), _ints(dst), _ints(tokens))
    m.fork(src, dst, tokens)
    _same(c, m, "fork")
    assert int(c.skipped) == m.skipped >= 4
    s = rng.integers(-1, slots + 1, n).tolist()
    keep = rng.integers(-1, slot_pages * T, n).tolist()
    c.trim(_ints(s), _ints(keep))
    m.trim(s, keep)
    _same(c, m, "trim")
    c.extend(_ints(dst[:5]), _offsets([1] * 5), 5)
    m.extend(dst[:5], list(range(6)), 5)
    _same(c, m, "extend")
    c.trim(_ints(list(range(slots))))
    m.trim(list(range(slots)), [0] * slots)
    _same(c, m, "all")
    assert not any(m.refs) and int(c.skipped) == m.skipped


@pytest.mark.parametrize("n", [1023, 1024, 1025, 2500])
def test_extend_batches_past_a_workgroup(n):
    """More entries than the planning workgroup has threads, more pages than it has words at a time."""
    import torch
    announce(f"extend {n} entries")
    c = _cache(1, 1, 64, 16, 70000, 3000, 40)
    m = kv_model.Pages(16, 70000, 3000, 40)
    rng = np.random.default_rng(n)
    for _ in range(2):
        s = rng.permutation(3000)[:n].tolist()
        counts = rng.integers(0, 300, n).tolist()
        off = [0] + np.cumsum(counts).tolist()
        assert c.extend(_ints(s), _t(off, torch.int64), off[-1]).tolist() == m.extend(s, off, off[-1])
        _same(c, m, n)
        drop = rng.permutation(3000)[:700].tolist()
        c.trim(_ints(drop))
        m.trim(drop, [0] * 700)
        _same(c, m, n)
    assert c.compact().tolist() == m.compact()
    _same(c, m, n)


def test_extend_that_finds_too_few_pages():
    """The first entry that finds too few pages left is refused with every later one that needs a page; entries
    within their last page go on."""
    announce("extend past the pool")
    c = _cache(1, 1, 64, 16, 6, 5, 8)
    m = kv_model.Pages(16, 6, 5, 8)
    for s, counts in (([0, 1], [20, 20]), ([0, 2, 1, 3], [2, 60, 2, 1]), ([3, 0], [32, 1]), ([4], [1])):
        off = [0] + np.cumsum(counts).tolist()
        import torch
        assert c.extend(_ints(s), _t(off, torch.int64), off[-1]).tolist() == m.extend(s, off, off[-1])
        _same(c, m, (s, counts))
    assert int(c.skipped) == m.skipped > 0


def test_extend_refuses_offsets_out_of_order():
    """Offsets that decrease, overlap or leave the rows: those entries are skipped, memory stays whole."""
    import torch
    announce("extend with bad offsets")
    for off in ([0, 5, 3, 6], [-1, 2, 4, 6], [0, 2, 9, 6], [0, 2 ** 40, 4, 6], [4, 4, 4, 4]):
        c = _cache(1, 1, 64, 16, 12, 4, 8)
        place = c.extend(_ints([0, 1, 2]), _t(off, torch.int64), 6).tolist()
        ok = [0 <= off[i] <= off[i + 1] <= 6 for i in range(3)]
        assert c.lengths.tolist()[:3] == [off[i + 1] - off[i] if ok[i] else 0 for i in range(3)], off
        assert int(c.skipped) == 3 - sum(ok)
        held = c.table[c.table >= 0].tolist()
        assert sorted(held) == [p for p in range(12) if int(c.refs[p]) == 1] and len(set(held)) == len(held)
        assert all(-1 <= p < 12 * 16 for p in place)


def test_extend_nothing():
    import torch
    announce("extend without entries, rows or tokens")
    c = _cache()
    assert c.extend(_ints([]), _t([0], torch.int64), 3).tolist() == [-1, -1, -1]
    assert c.extend(_ints([1, 1, -1]), _t([0, 0, 0, 0], torch.int64), 0).numel() == 0
    c.check()
    assert c.lengths.tolist() == [0] * 6


def test_a_description_of_the_held_pages_after_compaction():
    """The pages past the held ones are the caller's: a smaller cache over the same memory goes on."""
    import torch
    from paper_2606_17059_amd import KVCache
    announce("a smaller cache after a compaction")
    c = _cache(2, 2, 64, 16, 100, 6, 12)
    _fill(c, [100, 60, 30, 90])
    c.trim(_ints([0, 2]))
    held = int(c.compact()[1])
    assert held == 4 + 6
    rows = [_rows_of(c, 1, s) for s in (1, 3)]
    small = KVCache(c.k[:, :held], c.v[:, :held], c.table, c.lengths, c.refs[:held].clone(),
                    c.free[:(held + 63) // 64].clone() & ((1 << held) - 1))
    c.k[:, held:] = math.nan
    small.extend(_ints([0, 1]), _offsets([1, 1]), 2)  # slot 0 needs a page: none; slot 1 has room in its last
    assert small.lengths.tolist() == [0, 61, 0, 90, 0, 0] and int(small.skipped) == 1
    for s, old in zip((1, 3), rows):
        assert np.array_equal(_rows_of(small, 1, s)[0][:60], old[0][:60])
    assert small.attend(1, _ints([3]), torch.randn((1, 2, 64), device=device()).bfloat16()).isfinite().all()


# ---- together ------------------------------------------------------------------------
def test_decode_steps_in_a_graph():
    """A decode step (room, rows, attention on both layers, a trim) captured once and replayed on other batches,
    with eager work between, against an eager twin."""
    import torch
    announce("decode steps captured and replayed")
    n, H, D, L = 7, 2, 64, 2
    a, b = (_cache(L, H, D, 16, 300, 12, 40) for _ in range(2))
    for c in (a, b):
        _fill(c, [3, 16, 500, 31, 0, 47, 200, 1], seed=9)
    slots, off = _ints([0, 1, 2, 3, 4, 5, -1]), _offsets([1] * 6 + [0])
    kv, q = (torch.zeros(s, dtype=torch.bfloat16, device=device()) for s in ((L, 6, 2, H, D), (L, n, 6, D)))
    keep = _ints([1 << 20] * n)
    lse = torch.zeros((n, 6), device=device())

    def step(c):
        c.trim(slots, keep)
        place = c.extend(slots, off, 6)
        outs = []
        for layer in range(L):
            c.write(layer, place, kv[layer, :, 0], kv[layer, :, 1])
            outs.append(c.attend(layer, slots, q[layer], 0.2, lse=lse))
        return place, outs

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(b)
    torch.cuda.current_stream().wait_stream(side)
    b.trim(slots, _ints([3, 16, 500, 31, 0, 47, 0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        place, outs = step(b)
    b.check()
    gen = torch.Generator(device=device()).manual_seed(1)
    for k in range(6):
        kv.normal_(generator=gen)
        q.normal_(generator=gen)
        if k == 3:
            slots.copy_(_ints([7, 6, -1, 2, 0, 5, -1]))
            keep.copy_(_ints([0, 199, 0, 450, 1 << 20, 3, 0]))
        pe, oe = step(a)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(pe, place), k
        for x, y in zip(oe, outs):
            assert torch.equal(x, y), k
        for x, y in ((a.table, b.table), (a.lengths, b.lengths), (a.refs, b.refs), (a.free, b.free)):
            assert torch.equal(x, y), k
        torch.empty(1 << 20, device=device()).normal_()
    live = [s for s in range(8) if int(b.lengths[s])]
    for s in live:
        for x, y in zip(_rows_of(a, 1, s), _rows_of(b, 1, s)):
            assert np.array_equal(x, y)


def test_two_graphs_of_one_cache_on_two_streams():
    """Attentions may overlap: each captured call has scratch of its own."""
    import torch
    announce("two captured attentions replayed side by side")
    c = _cache(1, 2, 128, 16, 700, 4, 300)
    _fill(c, [4000, 3000, 2500])
    qs = [torch.randn((3, 8, 128), device=device()).bfloat16() for _ in range(2)]
    slots = [_ints([0, 1, 2]), _ints([2, 2, 0])]
    want = [c.attend(0, s, q, 0.1).clone() for s, q in zip(slots, qs)]
    graphs, outs = [], []
    for s, q in zip(slots, qs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(c.attend(0, s, q, 0.1))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for st, g in zip(streams, graphs):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o, w)


def test_calls_on_another_stream():
    import torch
    announce("calls on a stream that is not current")
    a, b = _cache(), _cache()
    st = torch.cuda.Stream()
    _fill(a, [20, 40])
    _fill(b, [20, 40])
    rows = torch.randn((3, 2, 64), device=device()).bfloat16()
    q = torch.randn((2, 4, 64), device=device()).bfloat16()
    slots, off, keep = _ints([0, 1]), _offsets([2, 1]), _ints([19, 33])
    src, dst, tok = _ints([1]), _ints([2]), _ints([18])
    torch.cuda.synchronize()
    outs = []
    for c, s in ((a, None), (b, st)):
        c.trim(slots, keep, stream=s)
        c.fork(src, dst, tok, stream=s)
        place = c.extend(slots, off, 3, stream=s)
        c.write(0, place, rows, rows, stream=s)
        outs.append(c.attend(0, slots, q, stream=s))
        c.compact(stream=s)
        c.check(stream=s)
    torch.cuda.synchronize()
    assert torch.equal(*outs) and torch.equal(a.table, b.table) and torch.equal(a.refs, b.refs)
    c.init(stream=st)
    torch.cuda.synchronize()
    assert c.lengths.tolist() == [0] * 6 and c.refs.sum() == 0 and (c.table == -1).all()


def test_the_binding_refuses_what_does_not_fit():
    import torch
    from paper_2606_17059_amd import KVCache
    announce("binding refusals")
    c = _cache()
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device=device())
    two = _ints([0, 1])
    place = _ints([0, 1])
    rows = q[:, :2].contiguous()
    for f, kind in (
            (lambda: c.attend(0, two.long(), q), TypeError), (lambda: c.attend(0, _ints([0]), q), ValueError),
            (lambda: c.attend(0, two, q.half()), TypeError), (lambda: c.attend(0, two, q[:, :, :32]), ValueError),
            (lambda: c.attend(0, two, q.transpose(1, 2).contiguous().transpose(1, 2)), ValueError),
            (lambda: c.attend(0, two, q[:, :3].contiguous()), RuntimeError), (lambda: c.attend(1, two, q), RuntimeError),
            (lambda: c.attend(0, two, q, window=-1), RuntimeError), (lambda: c.attend(0, two, q, math.nan), RuntimeError),
            (lambda: c.attend(0, two, q, out=torch.zeros_like(q).float()), ValueError),
            (lambda: c.attend(0, two, q, out=q), RuntimeError),
            (lambda: c.attend(0, two, q, lse=torch.zeros(2, 3, device=device())), ValueError),
            (lambda: c.attend(0, two, q.cpu()), TypeError), (lambda: c.attend(0, two, q[:1].expand(2, 4, 64)), RuntimeError),
            (lambda: c.write(0, place, rows, rows[:1]), ValueError), (lambda: c.write(0, place, q, q), ValueError),
            (lambda: c.write(0, place, rows.half(), rows.half()), TypeError),
            (lambda: c.write(2, place, rows, rows), RuntimeError),
            (lambda: c.extend(two, two, 2), TypeError), (lambda: c.extend(two, _offsets([1]), 1), ValueError),
            (lambda: c.extend(two, _offsets([1, 1]), -1), ValueError),
            (lambda: c.extend(two, _offsets([1, 1]), 2, place=_ints([0])), ValueError),
            (lambda: c.fork(two, two, _ints([1])), ValueError), (lambda: c.trim(two, _ints([1])), ValueError),
            (lambda: c.trim(two, torch.zeros(2, device=device())), TypeError),
            (lambda: KVCache(c.k, c.v.half(), c.table, c.lengths, c.refs, c.free), TypeError),
            (lambda: KVCache(c.v, c.k, c.table, c.lengths, c.refs, c.free), ValueError),
            (lambda: KVCache(c.k, c.v, c.table, c.lengths[:3], c.refs, c.free), ValueError),
            (lambda: KVCache(c.k, c.v, c.table, c.lengths, c.refs[:3], c.free), ValueError),
            (lambda: KVCache(c.k, c.v, c.table, c.lengths, c.refs, c.free, k_scale=2.0), RuntimeError),
            (lambda: KVCache(c.k[:1].expand(2, *c.k.shape[1:]), c.v[:1].expand(2, *c.v.shape[1:]), c.table, c.lengths,
                             c.refs, c.free), RuntimeError),
            (lambda: _cache(dim=80), RuntimeError), (lambda: _cache(page=8), RuntimeError),
            (lambda: _cache(slots=0), ValueError)):
        with pytest.raises(kind):
            f()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.trim(two)
        with pytest.raises(RuntimeError, match="capture"):
            c.check()


def test_the_calls_from_c(tmp_path):
    """tests/c/kv_check.c, plain C11 against the header and the built library."""
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    pkg, rocm = os.path.join(root, "paper_2606_17059_amd"), os.environ.get("ROCM_PATH", "/opt/rocm")
    exe = str(tmp_path / "kv_check")
    r = subprocess.run(["gcc", "-std=c11", "-Wall", "-Wextra", "-pedantic", "-Werror", "-D__HIP_PLATFORM_AMD__",
                        "-isystem", os.path.join(rocm, "include"), "-I", os.path.join(root, "include"),
                        os.path.join(root, "tests", "c", "kv_check.c"), "-o", exe, "-L", pkg, "-lprefix_router",
                        "-Wl,-rpath," + pkg, "-L", os.path.join(rocm, "lib"), "-lamdhip64",
                        "-Wl,-rpath," + os.path.join(rocm, "lib"), "-lm"],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    announce("KV cache from C")
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=60)
    assert r.returncode == 0 and "kv_check: ok" in r.stdout, r.stdout

"""What an 8-bit KV cache holds: the nearest e4m3 value of number / scale, for scales that are no powers of two; and what
forks, copied pages and compactions leave of it, next to the 16-bit types."""
import numpy as np
import pytest

import kv_model
from gpu_util import announce, device
from test_kv_gpu import _cache, _ints, _offsets, _rows_of, _types

pytestmark = pytest.mark.gpu


def _scales():
    """Scales that put a number beside a tie by their own rounding (x / middle), those of a largest number at 448, and
    the ends of the range."""
    ties = [np.float32(x / mid) for x in (1.0, 1.25, 1.40625) for mid in (17, 19, 21, 23, 25, 27, 29, 31)]
    tops = [np.float32((1 + m / 128) / 448) for m in range(0, 128, 9)]
    return [float(np.float32(s)) for s in ties + tops + [1e-40, 1e-30, 0.3, 3e20, 3e38]]  # as the library has them


@pytest.mark.parametrize("io", ["bf16", "fp16"])
def test_write_the_nearest_e4m3_of_an_inexact_quotient(io):
    """Every 16-bit number by every scale against the quotient in 64 bits (which lies on the exact one's side of each
    middle: these are at least 2^-25 of the quotient apart, or equal)."""
    import torch
    bits = torch.arange(65536, device=device()).to(torch.int16).view(_types()[io]).view(64, 4, 256)
    x = bits.float().cpu().double().numpy()
    tiny = np.abs(x) < 2.0 ** -100  # what the quotient's rounding left may be no float32 number there
    near = 0
    for scale in _scales():
        announce(f"every {io} number by {scale}")
        c = _cache(1, 4, 256, 256, 1, 1, 1, "e4m3", k_scale=scale, v_scale=scale)
        place = c.extend(_ints([0]), _offsets([64]), 64)
        c.write(0, place, bits, bits)
        with np.errstate(invalid="ignore", over="ignore"):
            y = x / scale
            clean = np.nan_to_num(y, nan=0.0, posinf=1e9, neginf=-1e9)
            want = np.where(np.isnan(x), np.nan, kv_model.e4m3(clean))
            near += int((kv_model.e4m3(clean.astype(np.float32).astype(np.float64)) != kv_model.e4m3(clean)).sum())
        for pool, at in ((c.k, (0, 0, slice(None), slice(None), slice(0, 64))), (c.v, (0, 0, slice(None), slice(0, 16)))):
            got = pool[at].float().cpu().double().numpy()
            if pool is c.k:  # [4, 32, 64, 8]
                got = got.transpose(2, 0, 1, 3).reshape(64, 4, 256)
            else:            # [4, 16, 256, 4]
                got = got.transpose(1, 3, 0, 2).reshape(64, 4, 256)
            assert np.array_equal(got[~tiny], want[~tiny], equal_nan=True), scale
    assert near > 100  # numbers that a rounded quotient would have put on the other side


@pytest.mark.parametrize("kind,dim,heads,page,layers", [
    ("e4m3", 64, 2, 16, 2), ("e4m3", 96, 3, 32, 1), ("e4m3", 128, 1, 16, 3), ("e4m3", 192, 1, 64, 2),
    ("e4m3", 256, 2, 128, 1), ("e4m3", 64, 1, 256, 2), ("fp16", 96, 1, 16, 2), ("bf16", 256, 1, 32, 1)])
def test_copies_and_moves_of_every_width(kind, dim, heads, page, layers):
    """Forks that end inside a page and are appended to, at every number of tokens to copy in a 4-token block, and a
    compaction: every sequence's numbers stay as they were, on every layer, byte for byte."""
    import torch
    announce(f"copies and moves, {kind} {dim} {heads} {page}")
    n = 8
    c = _cache(layers, heads, dim, page, 5 * n + 3, 2 * n + 1, 3, kind)
    for t in (c.k, c.v):
        t.view(torch.uint8).fill_(0xff)
    held = [page + 1 + (5 * i) % (page - 1) for i in range(n)]
    total = sum(held)
    g = torch.Generator(device=device()).manual_seed(dim)
    io = torch.bfloat16 if kind == "e4m3" else c.dtype
    rows = torch.empty((layers, 2, total + n, heads, dim), device=device()).normal_(generator=g).to(io)
    place = c.extend(_ints(range(n)), _offsets(held), total)
    for layer in range(layers):
        c.write(layer, place, rows[layer, 0, :total], rows[layer, 1, :total])
    start = [min(held[i], page + 1 + i) for i in range(n)]  # 1 to 8 tokens of the last page
    c.fork(_ints(range(n)), _ints(range(n, 2 * n)), _ints(start))
    place = c.extend(_ints(range(n, 2 * n)), _offsets([1] * n), n)
    for layer in range(layers):
        c.write(layer, place, rows[layer, 0, total:], rows[layer, 1, total:])
    c.check()
    want = rows.float().to(c.dtype).double().cpu().numpy() if kind == "e4m3" else rows.double().cpu().numpy()
    at = np.cumsum([0] + held)

    def same(slots):
        for layer in range(layers):
            for s in slots:
                got = _rows_of(c, layer, s)
                for x in (0, 1):
                    w = want[layer, x, at[s % n]:at[s % n + 1]]
                    if s >= n:
                        w = np.concatenate([w[:start[s - n]], want[layer, x, total + s - n][None]])
                    assert np.array_equal(got[x], w), (layer, s, x)

    same(range(2 * n))
    c.trim(_ints([0, 2, 3, 9, 12]))
    moved, kept = c.compact().tolist()
    assert moved > 0 and kept == int((c.refs > 0).sum()) and not int((c.refs[kept:] > 0).sum())
    same([s for s in range(2 * n) if s not in (0, 2, 3, 9, 12)])
    q = torch.randn((2 * n, heads, dim), device=device()).to(io)
    assert c.attend(layers - 1, _ints(range(2 * n)), q).isfinite().all()
    c.check()

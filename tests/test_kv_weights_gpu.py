"""Attention where one token's weight is far above the others' and its value is 0, as with an attention sink: the
output is the sum of many small weights, each of which has to be good by itself."""
import math

import pytest

from gpu_util import announce, device
from test_kv_gpu import _cache, _check_attend, _ints, _offsets, _types

pytestmark = pytest.mark.gpu


def _sink_case(kind, io, dim, lengths, gap, at, slot_pages=None, size=1.0):
    """Sequences of equal scores but one, 2^gap times as heavy, at token `at` of each.  Scores are products of powers
    of two by the scale, so that they are exact; values of the others lie in [size / 2, 3 size / 2]."""
    import torch
    announce(f"attend {kind} {io} dim {dim} lengths {lengths} gap {gap} at {at}")
    heads, total = 2, sum(lengths)
    c = _cache(1, heads, dim, 16, sum(-(-n // 16) for n in lengths) + 1, len(lengths),
               slot_pages or max(-(-n // 16) for n in lengths), kind,
               **(dict(k_scale=0.5, v_scale=max(1.0, size / 256)) if kind == "e4m3" else {}))
    place = c.extend(_ints(range(len(lengths))), _offsets(lengths), total)
    g = torch.Generator(device=device()).manual_seed(dim)
    k = torch.zeros((total, heads, dim), device=device())
    v = torch.empty((total, heads, dim), device=device()).uniform_(0.5 * size, 1.5 * size, generator=g)
    for i, n in enumerate(lengths):
        row = sum(lengths[:i]) + at % n
        k[row, :, dim - 1] = 16.0
        v[row] = 0.0
    c.write(0, place, k.to(_types()[io]), v.to(_types()[io]))
    q = torch.zeros((len(lengths), 2 * heads, dim), dtype=_types()[io], device=device())
    q[:, :, dim - 1] = 1.0
    scale = gap * math.log(2.0) / 16.0
    lse = torch.empty((len(lengths), 2 * heads), device=device())
    out = c.attend(0, _ints(range(len(lengths))), q, scale, lse=lse)
    # the library's scale is a float32 number
    _check_attend(c, 0, list(range(len(lengths))), q, scale, 0, out, lse)
    c.check()
    return out


@pytest.mark.parametrize("kind,io", [("fp16", "fp16"), ("e4m3", "fp16"), ("e4m3", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("gap", [6.0, 18.5, 20.4, 23.5, 25.2])
def test_attend_one_heavy_token_without_value(kind, io, dim, gap):
    """A workgroup a sequence, and shares with their joins; the heavy token first and last."""
    for at in (0, -1):
        _sink_case(kind, io, dim, [32, 611, 5], gap, at)
        _sink_case(kind, io, dim, [2816, 40], gap, at, slot_pages=400)


@pytest.mark.parametrize("kind,io", [("fp16", "fp16"), ("e4m3", "fp16")])
@pytest.mark.parametrize("gap", [32.0, 38.0])
def test_attend_small_weights_of_large_values(kind, io, gap):
    """Weights far below the smallest half number whose products with the values are not."""
    out = _sink_case(kind, io, 64, [611], gap, 0, size=24576.0)
    assert (out > 0).all()
    _sink_case(kind, io, 128, [2816], gap, 0, slot_pages=400, size=24576.0)


def test_attend_half_values_in_full():
    """Every finite half value, one a sequence of equal tokens: the output is the value, bit for bit.  (Weights are 1:
    the value's two parts and the division by their number are exact.)"""
    import torch
    announce("attend to every half value")
    dim, heads, n = 64, 8, 128
    c = _cache(1, heads, dim, 16, n, n, 1, "fp16")
    bits = torch.arange(65536, device=device()).to(torch.int16).view(torch.float16).view(n, heads, dim)
    x = torch.where(bits.isfinite(), bits, torch.zeros_like(bits))
    place = c.extend(_ints(range(n)), _offsets([2] * n), 2 * n)
    rows = x.repeat_interleave(2, 0)
    c.write(0, place, torch.zeros_like(rows), rows)
    out = c.attend(0, _ints(range(n)), torch.ones((n, heads, dim), dtype=torch.float16, device=device()), 1.0)
    assert torch.equal(out + 0.0, x + 0.0)  # -0 is 0
    c.check()


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_attend_no_weight_beside_values_that_are_not_finite(kind):
    """Scores that are all -infinity are a row without tokens, whatever the values hold."""
    import torch
    announce(f"attend without weights, {kind}, values not finite")
    for lengths, slot_pages in (([40, 3], 3), ([3000, 5], 400)):  # a workgroup a sequence; shares and their join
        c = _cache(1, 1, 64, 16, sum(-(-n // 16) for n in lengths), 2, slot_pages, kind)
        place = c.extend(_ints([0, 1]), _offsets(lengths), sum(lengths))
        k = torch.zeros((sum(lengths), 1, 64), dtype=_types()[kind], device=device())
        v = torch.ones_like(k)
        k[:, :, 3] = -math.inf
        v[1::3, :, 5], v[::7, :, 9], v[2::5, :, 60] = math.inf, math.nan, -math.inf
        c.write(0, place, k, v)
        q = torch.zeros((2, 2, 64), dtype=k.dtype, device=device())
        q[:, :, 3] = 1.0
        lse = torch.zeros((2, 2), device=device())
        out = c.attend(0, _ints([0, 1]), q, 1.0, lse=lse)
        assert (out == 0).all() and (lse == -math.inf).all(), lengths
        c.k[:, :, :, 0, :, 3] = 0  # all weights the same: each dimension is what its values make it
        out = c.attend(0, _ints([0, 1]), q, 1.0, lse=lse)
        assert not out[0, :, [5, 9, 60]].isfinite().any() and (out[:, :, [0, 4, 6, 63]] == 1).all()


@pytest.mark.parametrize("kind,io", [("fp16", "fp16"), ("e4m3", "fp16")])
def test_attend_numbers_below_the_normal_ones(kind, io):
    """Subnormal half keys with large queries, and subnormal queries with large keys, make scores like any others."""
    import torch
    announce(f"attend with subnormal numbers, {kind}")
    lengths, dim = [300, 20], 64
    for small_keys in (True, False):
        if small_keys and kind == "e4m3":
            continue  # its smallest number is a normal half number
        c = _cache(1, 2, dim, 16, 25, 2, 20, kind)
        place = c.extend(_ints([0, 1]), _offsets(lengths), sum(lengths))
        g = torch.Generator(device=device()).manual_seed(1)
        k, v = (torch.empty((sum(lengths), 2, dim), device=device()).normal_(generator=g) for _ in "kv")
        q = torch.empty((2, 4, dim), device=device()).normal_(generator=g)
        k, q = (k * 2.0 ** -17, q * 2.0 ** 12) if small_keys else (k * 2.0 ** 6, q * 2.0 ** -17)
        q = q.to(_types()[io])
        c.write(0, place, k.to(_types()[io]), v.to(_types()[io]))
        scale = 2.0 ** 4 if small_keys else 2.0 ** 10
        lse = torch.empty((2, 4), device=device())
        out = c.attend(0, _ints([0, 1]), q, scale, lse=lse)
        _check_attend(c, 0, [0, 1], q, scale, 0, out, lse)

"""A sequence's attention in different batches: alone, beside others that move the borders of the shares, and several
times in one batch.  The order of its sums differs, so the results are compared with 64 bits, not with each other."""
import pytest

from gpu_util import announce, device
from test_kv_gpu import _cache, _check_attend, _fill, _ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "fp16", "e4m3"])
@pytest.mark.parametrize("slot_pages", [60, 500])
def test_attend_in_any_batch(kind, slot_pages):
    import torch
    lengths = [900, 1, 33, 0, 257, 640, 31, 512]
    c = _cache(1, 2, 64, 16, sum(-(-n // 16) for n in lengths), len(lengths), slot_pages, kind)
    _fill(c, lengths, seed=4)
    io = torch.bfloat16 if kind == "e4m3" else c.dtype
    g = torch.Generator(device=device()).manual_seed(8)
    q = torch.empty((len(lengths), 6, 64), device=device()).normal_(0, 2.0, generator=g).to(io)
    batches = [[i] for i in range(8)] + [[0, 7], [7, 0], [3, 0, 3], [0, 0, 0, 0], list(range(8)), list(range(7, -1, -1)),
                                         [5] * 40 + [0], [0] + [1] * 200, list(range(8)) * 40]
    for slots in batches:
        announce(f"attend {kind}, {len(slots)} of {slots[:8]}, room for {slot_pages} pages")
        lse = torch.empty((len(slots), 6), device=device())
        out = c.attend(0, _ints(slots), q[slots], 0.125, lse=lse)
        first = {s: slots.index(s) for s in slots}
        some = list(first.values()) + ([len(slots) - 1] if len(slots) > 1 else [])
        _check_attend(c, 0, [slots[i] for i in some], q[slots][some], 0.125, 0, out[some], lse[some])
        again = torch.empty_like(lse)
        assert torch.equal(c.attend(0, _ints(slots), q[slots], 0.125, lse=again), out) and torch.equal(again, lse)
    c.check()


@pytest.mark.parametrize("n", [100, 200, 300, 700])
@pytest.mark.parametrize("kind,heads", [("fp16", 16), ("e4m3", 8), ("bf16", 1)])
def test_attend_short_sequences_with_several_long_ones(n, kind, heads):
    """Shares that keep to sequences (many heads) and that do not, with parts of several sequences kept at once; batches
    that waves look through and that a launch of its own does."""
    import torch
    lengths = [(37 * i) % 200 for i in range(n)]
    for k in range(0, n, 23):
        lengths[k] = 900 + 70 * (k % 19)
    announce(f"attend {n} sequences, {kind}, {heads} heads")
    c = _cache(1, heads, 64, 16, sum(-(-x // 16) for x in lengths), n, 140, kind)
    _fill(c, lengths, seed=6)
    io = torch.bfloat16 if kind == "e4m3" else c.dtype
    g = torch.Generator(device=device()).manual_seed(3)
    q = torch.empty((n, 2 * heads, 64), device=device()).normal_(0, 2.0, generator=g).to(io)
    lse = torch.empty((n, 2 * heads), device=device())
    for window in (0, 500):
        out = c.attend(0, _ints(range(n)), q, 0.125, window=window, lse=lse)
        some = sorted(set(range(0, n, 23)) | {1, 2, n - 1} | set(range(0, n, 31)))
        _check_attend(c, 0, some, q[some], 0.125, window, out[some], lse[some])
    c.check()

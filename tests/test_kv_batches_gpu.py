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

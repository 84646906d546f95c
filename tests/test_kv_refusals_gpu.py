"""What the KV cache's binding refuses, and what it must go on taking."""
import pytest

from gpu_util import announce, device
from test_kv_gpu import _cache, _fill, _ints, _offsets

pytestmark = pytest.mark.gpu


def _ready():
    import torch
    c = _cache(2)
    _fill(c, [5, 20])
    q = torch.randn((2, 4, 64), device=device()).bfloat16()
    return c, _ints([0, 1]), q


def test_gradients_are_refused_not_dropped():
    import torch
    import torch.autograd.forward_ad as forward_ad
    from paper_2606_17059_amd import KVCache
    announce("tensors that require gradients")
    c, slots, q = _ready()
    want = c.attend(0, slots, q)
    place = c.extend(slots, _offsets([1, 1]), 2)
    rows = q[:, :2].contiguous()
    leaf, lse = q.clone().requires_grad_(), torch.zeros((2, 4), device=device())
    for f in (lambda: c.attend(0, slots, leaf), lambda: c.attend(0, slots, leaf * 2),
              lambda: c.attend(0, slots, q, out=torch.zeros_like(q).requires_grad_()),
              lambda: c.attend(0, slots, q, lse=lse.clone().requires_grad_()),
              lambda: c.write(0, place, rows.clone().requires_grad_(), rows),
              lambda: c.write(0, place, rows, rows.clone().requires_grad_()),
              lambda: KVCache(c.k.clone().requires_grad_(), c.v, c.table, c.lengths, c.refs, c.free),
              lambda: KVCache(c.k, c.v.clone().requires_grad_(), c.table, c.lengths, c.refs, c.free)):
        with pytest.raises(ValueError, match="gradients"):
            f()
    with torch.no_grad(), forward_ad.dual_level():
        dual = forward_ad.make_dual(rows, rows)
        for f in (lambda: c.attend(0, slots, forward_ad.make_dual(q, q)), lambda: c.write(0, place, dual, rows),
                  lambda: c.write(0, place, rows, dual)):
            with pytest.raises(ValueError, match="tangent"):
                f()
        c.write(0, place, rows, rows)  # others go on
    c.trim(slots, _ints([5, 20]))
    for ask in (torch.no_grad, torch.inference_mode):
        with ask():
            got = c.attend(0, slots, leaf)
            assert torch.equal(got, want) and not got.requires_grad
    assert torch.equal(c.attend(0, slots, leaf.detach()), want)
    c.check()


@pytest.mark.parametrize("layer", [-1, 2, 2 ** 31, -2 ** 31, 2 ** 32, 2 ** 32 + 1, -2 ** 32, 2 ** 64, -2 ** 64])
def test_layers_past_32_bits_are_no_layers(layer):
    """A layer's number is 32 bits wide in the C call: what does not fit must not become another layer."""
    announce(f"layer {layer}")
    c, slots, q = _ready()
    place = c.extend(slots, _offsets([1, 1]), 2)
    rows = q[:, :2].contiguous()
    k, v = c.k.clone(), c.v.clone()
    with pytest.raises(RuntimeError, match="layer"):
        c.attend(layer, slots, q)
    with pytest.raises(RuntimeError, match="layer"):
        c.write(layer, place, rows, rows)
    import torch
    assert torch.equal(c.k.view(torch.int16), k.view(torch.int16)) and torch.equal(c.v.view(torch.int16), v.view(torch.int16))


@pytest.mark.parametrize("window", [-1, -2 ** 31, -2 ** 31 - 1, -2 ** 32, -2 ** 32 + 7, -2 ** 64])
def test_negative_windows_past_32_bits_are_negative(window):
    announce(f"window {window}")
    c, slots, q = _ready()
    with pytest.raises(RuntimeError, match="window"):
        c.attend(0, slots, q, window=window)


def test_checks_lose_no_entries_that_other_streams_count():
    """Attentions of unknown slots go on while another stream's checks report and reset the count: all are reported."""
    import re
    import torch
    from paper_2606_17059_amd import RouterError
    announce("checks beside attentions on another stream")
    c, _, q = _ready()
    bad = _ints([99, -7])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    total = 0

    def check():
        try:
            c.check()
        except RouterError as e:
            return int(re.search(r"(\d+) batch entries", str(e))[1])
        return 0

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(100):
            c.attend(0, bad, q)
    for _ in range(10):
        with torch.cuda.stream(side):
            for _ in range(5):
                graph.replay()
            done = torch.cuda.Event()
            done.record()
        while not done.query():
            total += check()
    torch.cuda.synchronize()
    total += check()
    assert total == 10 * 5 * 100 * 2 and int(c.skipped) == 0

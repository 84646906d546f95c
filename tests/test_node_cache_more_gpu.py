"""NodeCache over many admissions and with callers that reuse their buffers."""
import numpy as np
import pytest

from gpu_util import announce, device

pytestmark = pytest.mark.gpu


def _node(slots=6, pages=60, slot_pages=8):
    import torch
    from paper_2606_17059_amd import Forest, KVCache, NodeCache
    f = Forest(2)
    return f, NodeCache(f, 0, KVCache.create(1, 1, 64, 16, pages, slots, slot_pages, torch.bfloat16, device()))


def _insert(f, seqs):
    import torch
    t = torch.from_numpy(np.concatenate(seqs)).to(device())
    o = torch.tensor([0] + np.cumsum([len(s) for s in seqs]).tolist(), device=device())
    f.merge(torch.zeros(len(seqs), dtype=torch.int32, device=device()), t, o)


def test_a_callers_array_is_not_kept():
    """A prompt buffer that the caller fills anew does not change what is cached."""
    announce("admissions from one buffer")
    f, node = _node()
    rng = np.random.default_rng(1)
    prompts = [rng.integers(0, 1000, 40).astype(np.int32) for _ in range(3)]
    _insert(f, prompts)
    buf = np.zeros(40, np.int32)
    for p in prompts:
        buf[:] = p
        node.admit(buf)
    buf[:] = 7
    assert node.follow() == 0  # the tree holds all three
    for i, p in enumerate(prompts):
        assert node.lookup(p) == (i, 40) and np.array_equal(node.tokens[i], p)
    assert node.lookup(buf) == (-1, 0)
    node.close()
    f.close()


def test_the_index_stays_as_small_as_what_is_cached():
    """Thousands of sequences through a few slots: the index holds the last ones, not all there were, and finds them."""
    announce("1,500 admissions to six slots")
    f, node = _node()
    rng = np.random.default_rng(2)
    head = rng.integers(0, 1000, 40).astype(np.int32)
    most = 0
    for i in range(1500):
        t = np.concatenate([head, rng.integers(0, 1000, 60).astype(np.int32)])
        a = node.admit(t)
        assert a.cached >= 40 * (i > 0)
        info = node.index.info()
        most = max(most, info["num_nodes"] + info["pool_tokens"])
        if i % 100 == 0:
            for s, x in node.tokens.items():
                assert node.lookup(x)[1] == len(x)
    # twice what six sequences of 100 tokens need, the spare room, and what one admission adds
    assert most < 2 * 6 * 200 + node.SPARE + 4096
    node.cache.check()
    node.close()
    f.close()

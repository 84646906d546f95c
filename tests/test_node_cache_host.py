"""NodeCache's index belongs to the cache's device, also where another one is current.  No GPU: the forest and the
device guard are stand-ins that write down what was current when the forest was first used."""
from types import SimpleNamespace

import numpy as np


def test_the_index_is_made_on_the_caches_device(monkeypatch):
    import torch
    from paper_2606_17059_amd import node_cache
    current, seen = [0], []

    class Guard:
        def __init__(self, device):
            self.index = torch.device(device).index

        def __enter__(self):
            self.before, current[0] = current[0], self.index

        def __exit__(self, *exc):
            current[0] = self.before

    class Index:
        def __init__(self, slots):
            pass

        def load_snapshot_device(self, slot, tokens, offsets):
            seen.append(current[0])

        def info(self):
            return {"num_nodes": 1 << 20 if len(seen) == 2 else 0, "pool_tokens": 0}

        def compact(self):
            seen.append(current[0])

    monkeypatch.setattr(torch.cuda, "device", Guard)
    monkeypatch.setattr(node_cache, "Forest", Index)
    monkeypatch.setattr(node_cache.NodeCache, "_csr", lambda self, seqs: (None, None))
    cache = SimpleNamespace(device=torch.device("cuda", 3), lengths=np.zeros(4))
    node = node_cache.NodeCache(None, 0, cache)
    node._set(1, np.arange(5, dtype=np.int32))
    node._set(1, np.zeros(0, np.int32))
    assert seen == [3, 3, 3] and current == [0]

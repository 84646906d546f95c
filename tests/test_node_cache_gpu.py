"""A node's KV cache in step with its tree: the closed loop with caches gives the
same trace as without, reuses exactly the tokens the tree matches, and answers
every request as the whole prompt would, through forks, copies of shared pages,
evictions and compactions."""
import numpy as np
import pytest

import kv_model
from gpu_util import announce, device

pytestmark = pytest.mark.gpu


def _held_consistently(cache):
    """Tables, counts, lengths and free bits tell the same."""
    import torch
    t, T = cache.table, cache.page_tokens
    used = torch.bincount(t[t >= 0].long(), minlength=cache.pages)
    assert torch.equal(used.int(), cache.refs)
    assert torch.equal((t >= 0).sum(1), (cache.lengths.long() + T - 1) // T)
    bits = (cache.free[:, None] >> torch.arange(64, device=cache.device)) & 1
    assert torch.equal(bits.flatten()[:cache.pages] == 0, cache.refs > 0)


@pytest.mark.parametrize("variant", ["routed", "alone", "few_slots"])
def test_served_answers(variant):
    from paper_2606_17059_amd.sim import CacheConfig, RouterBackend, SimConfig, simulate
    cfg = SimConfig(nodes=3, requests=120, topics=7, prefix_len=(30, 60), question_len=(1, 20), vocab=50,
                    comm_ms=2.0, poll_ms=150.0, kv_tokens=500, base_ms=5.0, prefill_ms_per_token=0.5,
                    route=variant != "alone")
    cc = CacheConfig(layers=2, slots=6 if variant == "few_slots" else 64, max_tokens=80)
    checked = []

    class Checked(RouterBackend):
        def insert(self, peer, q):
            super().insert(peer, q)
            if peer != self.local:
                return
            s, ids = self.cache, self.cache.row_ids(q)
            before = getattr(self, "seen", 0)
            self.seen = s.cached
            checked.append((self.local, len(q), s.cached - before))
            _held_consistently(s.node.cache)
            if len(checked) % 5:
                return
            for layer in range(cc.layers):
                kv = s.kv[layer, ids].double().cpu().numpy()
                qv = s.q[layer, int(ids[-1])].double().cpu().numpy()
                ro, _, err, _ = kv_model.attend(qv, kv[:, 0], kv[:, 1], cc.head_dim ** -0.5)
                o = s.answer[layer].double().cpu().numpy()
                assert (np.abs(o - ro) <= err + 2.0 ** -8 * (np.abs(ro) + err)).all()

    announce(f"closed loop with KV caches: {variant}")
    nodes = [Checked(cfg.nodes, i, cache=cc, kv_tokens=cfg.kv_tokens) for i in range(cfg.nodes)]
    with_cache = simulate(cfg, nodes)
    announce("the same loop without")
    without = simulate(cfg)
    assert with_cache["trace"] == without["trace"] and with_cache["sim_ms"] == without["sim_ms"]
    assert [c[0] for c in checked] == [r["target"] for r in without["trace"]]
    for (_, n, cached), r in zip(checked, without["trace"]):
        assert n == r["len"] and cached <= r["actual"]
        if variant != "few_slots":  # every sequence of the tree is in the cache
            assert cached == r["actual"]
    assert sum(nd.cache.given_up for nd in nodes) > 0
    # new sequences take the lowest free pages, so a period may end without a hole
    assert sum(nd.cache.moved for nd in nodes) > 0 or variant != "routed"
    for nd in nodes:
        held = int((nd.cache.node.cache.refs > 0).sum())
        assert held <= -(-cfg.kv_tokens // 16) + cc.slots
        nd.close()


def test_admit_gives_up_what_is_oldest():
    import torch
    from paper_2606_17059_amd import Forest, KVCache, NodeCache
    announce("admissions to a full cache")
    f = Forest(2)
    c = KVCache.create(1, 1, 64, 16, 8, 4, 8, torch.bfloat16, device())
    node = NodeCache(f, 0, c)
    rng = np.random.default_rng(0)
    a, b, d = (rng.integers(0, 1000, n).astype(np.int32) for n in (40, 33, 50))
    assert node.admit(a)[:2] == (0, 0) and node.admit(b)[:2] == (1, 0)      # 3 and 3 pages
    assert node.admit(np.concatenate([a[:20], b[:9]]))[:2] == (2, 20)       # shares one page, copies one
    assert c.refs.sum().item() == 8 and list(node.tokens) == [1, 0, 2]
    again = node.admit(a[:17])  # all of it is there: no row, no page
    assert again.slot == 3 and again.cached == 17 and again.place.numel() == 0 and int((c.refs > 0).sum()) == 7
    node.drop([3])
    assert node.lookup(b[:5]) == (1, 5) and node.lookup(d) == (-1, 0) and node.lookup([]) == (-1, 0)
    got = node.admit(d)  # 4 pages: the oldest leaves, then the next
    assert got.cached == 0 and list(node.tokens)[-1] == got.slot and 1 not in list(node.tokens)[:-1]
    _held_consistently(c)
    got = node.admit(np.arange(128, dtype=np.int32))  # the whole cache
    assert list(node.tokens) == [got.slot] and int((c.refs > 0).sum()) == 8
    got = node.admit(np.concatenate([np.arange(100), [7] * 28]).astype(np.int32))  # its prefix would not fit beside it
    assert got.cached == 0 and int(c.lengths[got.slot]) == 128
    for bad in (np.zeros(129, np.int32), []):
        with pytest.raises(ValueError):
            node.admit(bad)
    c.check()
    node.drop([got.slot, 3])
    assert not node.tokens and int((c.refs > 0).sum()) == 0 and node.follow() == 0
    node.close()
    f.close()

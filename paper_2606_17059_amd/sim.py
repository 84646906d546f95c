"""Closed-loop simulation of the decentralized router (Algorithm 1) on N nodes.

Every node owns one forest: its own tree (the local peer, with access times)
and its estimates of the other nodes' trees.  Requests arrive one at a time,
round robin over the nodes, and each runs to completion before the next starts
(the paper's batching-free setup, Section "Experimental Setup").  For request
r arriving at node i:

  * node i routes r: k = the peer with the longest match in i's forest
    (pr_route_select; on equal match its own tree first);
  * if k = i, i runs r; otherwise r is forwarded (a round trip of 2 * comm
    with jitter), k runs it, and i inserts r into its estimate of k
    (UpdateTrieEstimate);
  * running r at node k: serving r refreshes the prefix it reuses (pr_touch),
    then least-recently-used tokens are evicted (pr_evict_lru) until the new
    tokens fit the node's KV budget, and r is inserted into k's own tree
    (UpdateTrie);
  * every poll period each node exports its own tree (sendTrie) and every
    other node replaces its estimate with it (anti-entropy, Section
    "Trie-broadcast loss").

The cost model is synthetic: latency = base + prefill_ms_per_token * (tokens
not cached at the processing node) + the forward's round trip.  The hit of a
request is the match at the processing node's own tree ("actual") and at the
routing node's estimate of it ("expected"), as fractions of the prompt.

The routing itself is the library's; the simulator only drives it through a
backend (RouterBackend below), so that the same trace can be replayed against
another implementation of the calls.

With a CacheConfig a node also has the KV cache whose index its own tree is
(node_cache.py): a request is admitted to it as a fork of its longest cached
prefix, keys and values of the other tokens are written on every layer, its last
token attends to all of them (the paper's workload has one output token), and
the cached sequences follow the tree's evictions.  There is no model: keys, values
and queries come from fixed random tables by token and position.
"""
from __future__ import annotations

import argparse
import json
import time
from dataclasses import dataclass, field, asdict
from typing import Dict, List, Optional

import numpy as np


@dataclass
class SimConfig:
    nodes: int = 4
    requests: int = 4000
    topics: int = 57
    prefix_len: tuple = (380, 520)     # few-shot prefix tokens per topic, U{a..b}
    question_len: tuple = (40, 140)    # fresh question tokens per request, U{a..b}
    vocab: int = 32000
    skew: Optional[float] = None       # None: uniform topics; else Zipf exponent over topic ranks
    comm_ms: float = 2.0               # one-way communication latency
    jitter_ms: float = 0.5             # uniform jitter added to each one-way delay
    poll_ms: float = 500.0             # anti-entropy period
    kv_tokens: int = 20000             # KV-cache budget of one node, in tokens
    base_ms: float = 20.0              # fixed cost of a request
    prefill_ms_per_token: float = 0.5  # cost of every token not found in the processing node's cache
    route: bool = True                 # False: every request runs where it arrives (no-routing baseline)
    seed: int = 20261202


@dataclass
class CacheConfig:
    """A node's KV cache; the heads are those of the paper's 0.5B model."""
    layers: int = 4
    kv_heads: int = 2
    q_heads: int = 14
    head_dim: int = 64
    page_tokens: int = 16
    slots: int = 256        # sequences kept at once
    max_tokens: int = 1024  # of a sequence
    seed: int = 20261202


class ServedCache:
    """A node's KV cache in the simulation: it admits requests, writes their rows and takes their last token's
    attention, rows coming from tables in place of a model."""

    TABLE = 4096

    def __init__(self, forest, local: int, cfg: CacheConfig, kv_tokens: int, device):
        import torch
        from .kvcache import KVCache
        from .node_cache import NodeCache
        T = cfg.page_tokens
        # full pages of kv_tokens distinct tokens, and a partly filled one of each sequence
        pages = -(-kv_tokens // T) + cfg.slots + -(-cfg.max_tokens // T)
        cache = KVCache.create(cfg.layers, cfg.kv_heads, cfg.head_dim, T, pages, cfg.slots, -(-cfg.max_tokens // T),
                               torch.bfloat16, device)
        self.node = NodeCache(forest, local, cache)
        g = torch.Generator(device=device).manual_seed(cfg.seed)
        shape = (cfg.layers, self.TABLE, 2, cfg.kv_heads, cfg.head_dim)
        self.kv = torch.empty(shape, dtype=torch.bfloat16, device=device).normal_(generator=g)
        self.q = torch.empty((cfg.layers, self.TABLE, cfg.q_heads, cfg.head_dim), dtype=torch.bfloat16,
                             device=device).normal_(generator=g)
        self.cached, self.admitted, self.given_up, self.moved = 0, 0, 0, 0
        self.answer = None  # the last request's attention, [layers, heads, head_dim]

    def row_ids(self, tokens, first: int = 0):
        """Row of the tables for each token at its position."""
        t = np.asarray(tokens, np.int64)
        return (t * 31 + np.arange(first, first + len(t)) * 7) % self.TABLE

    def serve(self, tokens) -> None:
        import torch
        a = self.node.admit(tokens)
        c = self.node.cache
        ids = torch.from_numpy(self.row_ids(tokens[a.cached:], a.cached)).to(c.device)
        last = int(self.row_ids(tokens)[-1])
        slot = torch.tensor([a.slot], dtype=torch.int32, device=c.device)
        out = []
        for layer in range(c.layers):
            rows = self.kv[layer, ids]
            c.write(layer, a.place, rows[:, 0], rows[:, 1])
            out.append(c.attend(layer, slot, self.q[layer, last:last + 1])[0])
        self.answer = torch.stack(out)
        self.admitted += len(tokens)
        self.cached += a.cached

    def follow(self) -> None:
        self.given_up += self.node.follow()

    def compact(self) -> None:
        self.moved += self.node.compact()[0]

    def close(self) -> None:
        self.node.cache.check()
        self.node.close()


class RouterBackend:
    """One node's router: the calls the simulation makes, on the library.  With `cache` (and the node's budget of
    tokens) it also serves what it inserts into its own tree from a KV cache."""

    def __init__(self, num_peers: int, local: int, device=None, cache: Optional[CacheConfig] = None,
                 kv_tokens: int = 0):
        import torch
        from .router import Forest
        self.dev = device if device is not None else torch.device("cuda", torch.cuda.current_device())
        self.f = Forest(num_peers)
        self.local = local
        self.f.set_local_peer(local)
        self.cache = ServedCache(self.f, local, cache, kv_tokens, self.dev) if cache is not None else None

    def _csr(self, seqs):
        import torch
        t = np.concatenate([np.asarray(s, np.int32) for s in seqs]) if seqs else np.zeros(0, np.int32)
        o = np.zeros(len(seqs) + 1, np.int64)
        o[1:] = np.cumsum([len(s) for s in seqs])
        return torch.from_numpy(t).to(self.dev), torch.from_numpy(o).to(self.dev)

    def set_time(self, t: int) -> None:
        self.f.set_time(t)

    def route(self, q):
        import torch
        t, o = self._csr([q])
        m, b1, b2 = self.f.route_select(t, o, None, self.local, True)
        torch.cuda.synchronize()
        return m.cpu().numpy()[0], int(b1.cpu()[0]), int(b2.cpu()[0])

    def touch(self, q) -> None:
        t, o = self._csr([q])
        self.f.touch(t, o)

    def tree_tokens(self) -> int:
        return self.f.tree_tokens(self.local)

    def evict(self, n: int) -> int:
        ev = self.f.evict_lru(n)
        if self.cache is not None:
            self.cache.follow()
        return ev

    def insert(self, peer: int, q) -> None:
        import torch
        t, o = self._csr([q])
        self.f.merge(torch.tensor([peer], dtype=torch.int32, device=self.dev), t, o)
        if peer == self.local and self.cache is not None:
            self.cache.serve(q)

    def export_local(self):
        if self.cache is not None:
            self.cache.compact()
        return self.f.export_snapshot(self.local)

    def load_estimate(self, peer: int, snapshot) -> None:
        t, o = snapshot
        self.f.load_snapshot_device(peer, t.contiguous(), o)

    def close(self) -> None:
        if self.cache is not None:
            self.cache.close()
        self.f.close()


def make_workload(cfg: SimConfig):
    """Seeded synthetic prompts: topic prefixes plus fresh questions."""
    rng = np.random.default_rng(np.random.SeedSequence([cfg.seed, 4]))
    heads = [rng.integers(0, cfg.vocab, size=int(rng.integers(cfg.prefix_len[0], cfg.prefix_len[1] + 1)),
                          dtype=np.int32) for _ in range(cfg.topics)]
    if cfg.skew is None:
        p = np.full(cfg.topics, 1.0 / cfg.topics)
    else:
        w = 1.0 / np.power(np.arange(1, cfg.topics + 1, dtype=np.float64), cfg.skew)
        p = (w / w.sum())[rng.permutation(cfg.topics)]
    topic = rng.choice(cfg.topics, size=cfg.requests, p=p)
    qlen = rng.integers(cfg.question_len[0], cfg.question_len[1] + 1, size=cfg.requests)
    prompts = [np.concatenate([heads[t], rng.integers(0, cfg.vocab, size=int(n), dtype=np.int32)])
               for t, n in zip(topic, qlen)]
    jitter = rng.uniform(-cfg.jitter_ms, cfg.jitter_ms, size=(cfg.requests, 2))
    return prompts, topic, jitter


def simulate(cfg: SimConfig, backends: Optional[List] = None, make_backend=None) -> Dict:
    """Run the closed loop.  backends: one RouterBackend-like object per node
    (created with make_backend(num_peers, local) if not given)."""
    N = cfg.nodes
    mk = make_backend or (lambda P, local: RouterBackend(P, local))
    nodes = backends or [mk(N, i) for i in range(N)]
    prompts, topic, jitter = make_workload(cfg)
    clock = 0.0
    next_poll = cfg.poll_ms
    trace = []
    t_calls = 0.0

    def stamp():
        return int(round(clock * 1000))  # microseconds

    def run_at(k, q, hit):
        nonlocal t_calls
        nd = nodes[k]
        t0 = time.perf_counter()
        nd.set_time(stamp())
        nd.touch(q)
        need = max(0, len(q) - hit)
        have = nd.tree_tokens()
        ev = 0
        if have + need > cfg.kv_tokens:
            ev = nd.evict(have + need - cfg.kv_tokens)
        nd.insert(nd.local, q)
        t_calls += time.perf_counter() - t0
        return ev

    for j, q in enumerate(prompts):
        i = j % N
        while clock >= next_poll:  # anti-entropy rounds due before this request
            t0 = time.perf_counter()
            snaps = [nodes[a].export_local() for a in range(N)]
            for b in range(N):
                for a in range(N):
                    if a != b:
                        nodes[b].load_estimate(a, snaps[a])
            t_calls += time.perf_counter() - t0
            next_poll += cfg.poll_ms
        t0 = time.perf_counter()
        for nd in nodes:
            nd.set_time(stamp())
        m_row, best, second = nodes[i].route(q)
        t_calls += time.perf_counter() - t0
        k = best if cfg.route else i
        expected = int(m_row[k])
        delay = 0.0
        if k != i:
            delay = 2 * cfg.comm_ms + jitter[j, 0] + jitter[j, 1]
            t0 = time.perf_counter()
            actual = int(nodes[k].route(q)[0][k])  # the processing node's own tree
            t_calls += time.perf_counter() - t0
        else:
            actual = int(m_row[i])
        ev = run_at(k, q, actual)
        if k != i:
            t0 = time.perf_counter()
            nodes[i].insert(k, q)  # UpdateTrieEstimate after a successful forward
            t_calls += time.perf_counter() - t0
        lat = cfg.base_ms + cfg.prefill_ms_per_token * (len(q) - actual) + delay
        clock += lat
        trace.append({"origin": i, "target": k, "second": second, "topic": int(topic[j]), "len": len(q),
                      "expected": expected, "actual": actual, "evicted": ev, "latency_ms": lat})
    if backends is None:
        for nd in nodes:
            nd.close()
    return {"config": asdict(cfg), "trace": trace, "library_seconds": t_calls, "sim_ms": clock}


def summarize(res: Dict, window: int = 300, stride: int = 30) -> Dict:
    tr = res["trace"]
    N = res["config"]["nodes"]
    tgt = np.array([r["target"] for r in tr])
    ln = np.array([r["len"] for r in tr], np.float64)
    share = np.bincount(tgt, minlength=N) / len(tr)
    tops = np.array([r["topic"] for r in tr])
    # per-topic specialisation: the share of a topic's requests its busiest node takes, per window
    spec = []
    for t in np.unique(tops):
        idx = np.nonzero(tops == t)[0]
        if len(idx) >= window:
            for s in range(0, len(idx) - window + 1, stride):
                spec.append(np.bincount(tgt[idx[s:s + window]], minlength=N).max() / window)
    return {
        "requests": len(tr),
        "hotspot_share": float(share.max()),
        "node_share": share.tolist(),
        "forwarded": float(np.mean([r["origin"] != r["target"] for r in tr])),
        "expected_hit": float(np.sum([r["expected"] for r in tr]) / ln.sum()),
        "actual_hit": float(np.sum([r["actual"] for r in tr]) / ln.sum()),
        "mean_latency_ms": float(np.mean([r["latency_ms"] for r in tr])),
        "evicted_tokens": int(np.sum([r["evicted"] for r in tr])),
        "topic_window_top_share": float(np.mean(spec)) if spec else None,
        "library_seconds": res["library_seconds"],
        "library_us_per_request": res["library_seconds"] / len(tr) * 1e6,
    }


def main() -> int:
    ap = argparse.ArgumentParser(description="closed-loop simulation of Algorithm 1 on the library")
    ap.add_argument("--nodes", type=int, default=4)
    ap.add_argument("--requests", type=int, default=4000)
    ap.add_argument("--skew", type=float, default=None)
    ap.add_argument("--comm-ms", type=float, default=2.0)
    ap.add_argument("--poll-ms", type=float, default=500.0)
    ap.add_argument("--kv-tokens", type=int, default=20000)
    ap.add_argument("--no-route", action="store_true")
    ap.add_argument("--seed", type=int, default=20261202)
    ap.add_argument("--kv-cache", action="store_true",
                    help="each node serves its requests from a KV cache that follows its tree")
    ap.add_argument("--kv-slots", type=int, default=256, help="sequences a node's KV cache keeps")
    a = ap.parse_args()
    cfg = SimConfig(nodes=a.nodes, requests=a.requests, skew=a.skew, comm_ms=a.comm_ms, poll_ms=a.poll_ms,
                    kv_tokens=a.kv_tokens, route=not a.no_route, seed=a.seed)
    if a.kv_cache:
        cache = CacheConfig(slots=a.kv_slots, max_tokens=cfg.prefix_len[1] + cfg.question_len[1], seed=cfg.seed)
        nodes = [RouterBackend(cfg.nodes, i, cache=cache, kv_tokens=cfg.kv_tokens) for i in range(cfg.nodes)]
        out = summarize(simulate(cfg, nodes))
        served = [nd.cache for nd in nodes]
        out["kv_cached"] = sum(s.cached for s in served) / max(1, sum(s.admitted for s in served))
        out["kv_given_up"] = sum(s.given_up for s in served)
        out["kv_pages_moved"] = sum(s.moved for s in served)
        out["kv_pages_held"] = [int((s.node.cache.refs > 0).sum()) for s in served]
        out["kv_config"] = asdict(cache)
        for nd in nodes:
            nd.close()
    else:
        out = summarize(simulate(cfg))
    out["config"] = asdict(cfg)
    print(json.dumps(out))
    return 0


if __name__ == "__main__":
    raise SystemExit(main())

"""A node's KV cache kept in step with its own tree.

Algorithm 1 pairs every change of the local tree with one of the cache's memory:
updateTrie with updateKVCache, EvictLRUTrie with evictKVCache.  NodeCache makes the
second halves from the library's calls:

  * `admit` finds the cached sequence with the longest common prefix (a forest of its
    own, one tree per cache slot, routed like a forest of peers), forks it (pr_kv_fork)
    and makes room for the rest (pr_kv_extend);
  * `follow`, after pr_evict_lru, routes the cached sequences against the node's forest:
    the match lengths in the local tree are what each may keep, and go to pr_kv_trim as
    they are, on the device.

Keys and values are the caller's to write (KVCache.write) and to use (KVCache.attend).
"""
from __future__ import annotations

from typing import Dict, List, NamedTuple

import numpy as np

from .kvcache import KVCache
from .router import Forest


class Admission(NamedTuple):
    slot: int     # the cache slot that holds the sequence
    cached: int   # its first tokens whose keys and values are there already
    place: object  # int32 CUDA tensor: where the rows of the others go


class NodeCache:
    """forest: the node's, on the cache's device; local: its own tree's peer id there; cache: an empty KVCache with at
    most PR_MAX_PEERS slots.  Calls are host-synchronous and run on the current stream of that device, whichever device
    is current.  The rows of an admission have to be written before the next call, which may share or copy them."""

    SPARE = 1 << 16  # nodes and label tokens out of use that the index may have beside as many as it had in use

    def __init__(self, forest: Forest, local: int, cache: KVCache):
        self.forest, self.local, self.cache = forest, int(local), cache
        self.slots = cache.lengths.shape[0]
        self.index = Forest(self.slots)
        self.tokens: Dict[int, np.ndarray] = {}  # per slot in use, least recently used first
        self._least = 0  # size of the index after its last compaction

    def _ints(self, x):
        import torch
        return torch.tensor(x, dtype=torch.int32, device=self.cache.device)

    def _csr(self, seqs: List[np.ndarray]):
        import torch
        t = np.concatenate(seqs) if seqs else np.zeros(0, np.int32)
        o = np.zeros(len(seqs) + 1, np.int64)
        o[1:] = np.cumsum([len(s) for s in seqs])
        return torch.from_numpy(t).to(self.cache.device), torch.from_numpy(o).to(self.cache.device)

    def _set(self, slot: int, tokens: np.ndarray) -> None:
        """The slot's sequence, in the index and here (an empty one: the slot is free)."""
        import torch
        with torch.cuda.device(self.cache.device):  # a forest is of the device that is current at its first call
            self.index.load_snapshot_device(slot, *self._csr([tokens] if len(tokens) else []))
        self.tokens.pop(slot, None)
        if len(tokens):
            self.tokens[slot] = tokens
        # a slot's next sequence leaves its last one's nodes and labels behind (3,000 admissions to six slots: 453,036
        # nodes of which 12 were in use)
        if self._size() > 2 * self._least + self.SPARE:
            with torch.cuda.device(self.cache.device):
                self.index.compact()
            self._least = self._size()

    def _size(self) -> int:
        info = self.index.info()
        return info["num_nodes"] + info["pool_tokens"]

    def drop(self, slots) -> None:
        """Give up the sequences of these slots (evictKVCache)."""
        slots = [s for s in slots if s in self.tokens]
        if slots:
            self.cache.trim(self._ints(slots))
            for s in slots:
                self._set(s, np.zeros(0, np.int32))

    def lookup(self, tokens) -> tuple:
        """(slot, tokens) of the longest cached prefix; (-1, 0) if there is none."""
        t = np.ascontiguousarray(tokens, dtype=np.int32)
        if not self.tokens or len(t) == 0:
            return -1, 0
        m, best = self.index.route(*self._csr([t]))
        slot = int(best[0])
        n = int(m[0, slot])
        return (slot, n) if n else (-1, 0)

    def admit(self, tokens) -> Admission:
        """Put a sequence of one token or more into the cache: a fork of its longest cached prefix, with room for
        the rest.  Where no slot or too few pages are free, the least recently used sequences are given up.  Raises
        ValueError if the sequence does not fit an empty cache."""
        t = np.array(tokens, dtype=np.int32)  # kept: not the caller's, who may fill it anew
        c, T = self.cache, self.cache.page_tokens
        pages = -(-len(t) // T)
        if len(t) == 0 or pages > min(c.table.shape[1], c.pages):
            raise ValueError(f"a sequence of {len(t)} tokens does not fit the cache")
        src, cached = self.lookup(t)
        if src >= 0:
            self.tokens[src] = self.tokens.pop(src)  # used now
        while True:
            # a shared page that is partly filled is copied when it is appended to
            need = pages - cached // T if cached < len(t) else 0
            if len(self.tokens) < self.slots and int((c.refs == 0).sum()) >= need:
                break
            oldest = next(iter(self.tokens))
            if oldest == src:  # nothing else is left
                src, cached = -1, 0
            self.drop([oldest])
        slot = next(s for s in range(self.slots) if s not in self.tokens)
        if cached:
            c.fork(self._ints([src]), self._ints([slot]), self._ints([cached]))
        import torch
        rest = len(t) - cached
        place = c.extend(self._ints([slot]), torch.tensor([0, rest], device=c.device), rest)
        self._set(slot, t)
        return Admission(slot, cached, place)

    def follow(self) -> int:
        """Trim every cached sequence to what the local tree still holds of it; the tokens given up."""
        slots = list(self.tokens)
        if not slots:
            return 0
        m, _ = self.forest.route(*self._csr([self.tokens[s] for s in slots]))
        keep = m[:, self.local]
        self.cache.trim(self._ints(slots), keep)
        gone = 0
        order = list(self.tokens)
        for s, k in zip(slots, keep.tolist()):
            if k < len(self.tokens[s]):
                gone += len(self.tokens[s]) - k
                self._set(s, self.tokens[s][:k])
        self.tokens = {s: self.tokens[s] for s in order if s in self.tokens}  # trimming is no use
        return gone

    def compact(self) -> tuple:
        """Move the held pages to the lowest ids: (pages moved, pages held)."""
        return tuple(self.cache.compact().tolist())

    def close(self) -> None:
        self.index.close()

"""A plain model of the paged KV cache (test infrastructure): the rules of
include/prefix_router.h in Python lists, and attention in 64 bits from the pages'
numbers.  Shares no code with the library."""
import math

import numpy as np


class Pages:
    """Who holds which page, and which rows lie there: content[page][t] is the id of the row written at token t."""

    def __init__(self, page_tokens, num_pages, num_slots, slot_pages):
        self.T, self.P, self.S, self.M = page_tokens, num_pages, num_slots, slot_pages
        self.table = [[] for _ in range(num_slots)]
        self.length = [0] * num_slots
        self.refs = [0] * num_pages
        self.content = [[None] * page_tokens for _ in range(num_pages)]
        self.skipped = 0

    def _up(self, n):
        return -(-n // self.T)

    def extend(self, slots, offsets, rows):
        place = [-1] * rows
        free = [p for p in range(self.P) if self.refs[p] == 0]
        refs = list(self.refs)
        seen, dry, used, plan = set(), False, 0, []
        for i, s in enumerate(slots):
            a, b = offsets[i], offsets[i + 1]
            if s == -1:
                continue
            if not (0 <= s < self.S) or a < 0 or b < a or b > rows:
                self.skipped += 1
                continue
            if b > a:
                if s in seen:
                    self.skipped += 1
                    continue
                seen.add(s)
            n = b - a
            if n == 0:  # changes nothing, also where another entry appends to the slot
                continue
            start = self.length[s]
            if start + n > self.M * self.T:
                self.skipped += 1
                continue
            shared = start % self.T > 0 and refs[self.table[s][-1]] > 1
            need = self._up(start + n) - self._up(start) + shared
            if need and (dry or used + need > len(free)):
                dry = True
                self.skipped += 1
                continue
            plan.append((s, a, n, start, shared, free[used:used + need]))
            used += need
        for s, a, n, start, shared, new in plan:
            new = list(new)
            for p in new:
                self.refs[p] = 1
            if shared:
                old, mine = self.table[s][-1], new.pop(0)
                self.content[mine][:start % self.T] = self.content[old][:start % self.T]
                self.refs[old] -= 1
                self.table[s][-1] = mine
            self.table[s] += new
            self.length[s] = start + n
            for r in range(n):
                place[a + r] = self.table[s][(start + r) // self.T] * self.T + (start + r) % self.T
        return place

    def write(self, place, ids):
        for p, x in zip(place, ids):
            if 0 <= p < self.P * self.T:
                self.content[p // self.T][p % self.T] = x

    def fork(self, src, dst, tokens):
        length = list(self.length)
        for i, (a, b, n) in enumerate(zip(src, dst, tokens)):
            if b == -1:
                continue
            if (not (0 <= a < self.S) or not (0 <= b < self.S) or a in dst or b in dst[:i] or length[b] or n < 0 or
                    n > length[a]):
                self.skipped += 1
                continue
            self.table[b] = self.table[a][:self._up(n)]
            self.length[b] = n
            for p in self.table[b]:
                self.refs[p] += 1

    def trim(self, slots, keep):
        for s, n in zip(slots, keep):
            if s == -1:
                continue
            if not (0 <= s < self.S) or n < 0:
                self.skipped += 1
                continue
            if n >= self.length[s]:
                continue
            for p in self.table[s][self._up(n):]:
                self.refs[p] -= 1
            self.table[s] = self.table[s][:self._up(n)]
            self.length[s] = n

    def compact(self):
        held = sum(r > 0 for r in self.refs)
        holes = [p for p in range(held) if not self.refs[p]]
        movers = [p for p in range(held, self.P) if self.refs[p]]
        to = dict(zip(movers, holes))
        for a, b in to.items():
            self.content[b] = list(self.content[a])
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.table = [[to.get(p, p) for p in row] for row in self.table]
        return [len(holes), held]

    def rows(self, slot):
        """Ids of a sequence's rows in order."""
        n = self.length[slot]
        return [self.content[self.table[slot][t // self.T]][t % self.T] for t in range(n)]

    def table_array(self):
        t = np.full((self.S, self.M), -1, np.int32)
        for s, row in enumerate(self.table):
            t[s, :len(row)] = row
        return t

    def free_words(self):
        w = np.zeros((self.P + 63) // 64, np.uint64)
        for p, r in enumerate(self.refs):
            if not r:
                w[p // 64] |= np.uint64(1) << np.uint64(p % 64)
        return w.view(np.int64)


def e4m3(x):
    """The nearest e4m3 value of float64 numbers: ties to even, at most 448 (3 bits behind the leading one, exponents
    from -6)."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(x), 448.0)
    step = np.exp2(np.floor(np.log2(np.maximum(a, 2.0 ** -6))) - 3)
    return np.sign(x) * np.minimum(np.round(a / step) * step, 448.0)


def attend(q, k, v, scale):
    """Heads q [heads, D] over keys and values [tokens, kv_heads, D] in float64: out, lse, and the error a pass in 32
    bits may have (absolute, per output number), with the lse's.

    A score is a sum of D products in float32: off by at most D 2^-24 sum |q k| scale, times 2 for the scaling and the
    subtraction of the maximum (|x| 2^-24 each, |x| <= sum |q k| scale).  A weight's relative error is twice that (its
    own score's and the normalising sum's), plus what 2^x and the rounding in two 16-bit parts leave: 2^-16 together.
    An output is off by that times the weights' sum of |v|."""
    heads, D = q.shape
    n, H, _ = k.shape
    out, lse = np.zeros((heads, D)), np.full(heads, -math.inf)
    err, lerr = np.zeros((heads, D)), np.zeros(heads)
    if n == 0:
        return out, lse, err, lerr
    for h in range(heads):
        g = h // (heads // H)
        x = scale * (k[:, g] @ q[h])
        top = x.max()
        p = np.exp(x - top)
        lse[h] = top + np.log(p.sum())
        p /= p.sum()
        out[h] = p @ v[:, g]
        off = 2 * D * 2.0 ** -24 * (abs(scale) * (np.abs(k[:, g]) @ np.abs(q[h]))).max()
        err[h] = (2 * off + 2.0 ** -16) * (p @ np.abs(v[:, g]))
        lerr[h] = off + 2.0 ** -21 * (1 + abs(lse[h]))
    return out, lse, err, lerr

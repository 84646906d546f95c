"""The KV-cache operators: their cases, plain forms, and what a pass cannot do without.

A node's KV cache is paged memory next to the node's own radix tree:

  k        [layers, pages, kv_heads, head_dim / 8, page_tokens, 8]
  v        [layers, pages, kv_heads, page_tokens / 4, head_dim, 4]
  table    int32 [slots, pages a slot]: the pages of a slot's sequence, -1 past its last
  lengths  int32 [slots]: tokens of a slot's sequence
  refs     int32 [pages]: slots whose sequence holds the page
  free     int64 words: bit p % 64 of word p / 64 is set if page p is held by none

A case names such a cache and what a program does with it:

  attend   one new token a sequence attends to its cached tokens (KVCache.attend)
  append   sequences are cut back to their accepted tokens, get room for new ones, and the new tokens' rows are
           written in every layer (KVCache.trim, extend, write)
  share    sequences start as forks of cached prefixes and get their first tokens of their own; the slots' earlier
           forks are freed first (KVCache.trim, fork, extend)
  compact  the live pages move to the lowest ids (KVCache.compact); every pass starts from the same tables
  step     a whole decode step: room for one token a sequence, then in every layer its rows and its attention
"""
import math
import random

import torch

own = False
DEVICE = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}


def _case(name, do, n, lo, hi, kv_heads, group, dim, page, kind="bf16", io="bf16", layers=1, window=0, new=(1, 1),
          parents=0, empty=0, lse=False):
    return dict(name=name, do=do, n=n, lo=lo, hi=hi, kv_heads=kv_heads, group=group, dim=dim, page=page, kind=kind,
                io=io, layers=layers, window=window, new_lo=new[0], new_hi=new[1], parents=parents, empty=empty,
                lse=lse)


def listed():
    return [
        # one request at a time, a few-shot prompt and one answer token, on the paper's 0.5B model's heads
        _case("attend one 611", "attend", 1, 611, 611, 2, 7, 64, 16),
        # one long-context request: few rows, everything comes from splitting its length
        _case("attend one 131072", "attend", 1, 131072, 131072, 8, 4, 128, 64),
        # a front end's ragged batch with rows that hold nothing yet
        _case("attend ragged 64", "attend", 64, 1, 8192, 8, 4, 128, 16, "fp16", "fp16", empty=3, lse=True),
        # the largest batch: long contexts, eight query heads a key head
        _case("attend 128 long", "attend", 128, 4096, 16384, 8, 8, 128, 64),
        # an 8-bit cache of one key head shared by all query heads, the last tokens only
        _case("attend window e4m3", "attend", 96, 500, 12000, 1, 48, 192, 32, "e4m3", "bf16", window=4096),
        # a decode step's rows on all layers of the 0.5B model
        _case("append 256 tokens", "append", 256, 100, 1500, 2, 7, 64, 16, layers=24),
        # prompts that arrive with part of their prefix cached
        _case("append 16 prompts", "append", 16, 0, 900, 8, 4, 128, 64, layers=4, new=(300, 4000)),
        # answers sampled side by side from shared prompts: each child copies its prompt's last page
        _case("share 64 of 8", "share", 64, 380, 660, 2, 7, 64, 16, layers=24, parents=8),
        # many short questions on a few long documents
        _case("share 256 of 3 long", "share", 256, 20000, 100000, 4, 4, 128, 32, layers=2, parents=3, new=(8, 120)),
        # a small node's cache after evictions
        _case("compact 57", "compact", 57, 380, 660, 2, 7, 64, 16, layers=24),
        # a large cache after evictions
        _case("compact 400", "compact", 400, 200, 4000, 8, 4, 128, 64, layers=1),
        # a whole decode step on an 8-bit cache
        _case("step 48 e4m3", "step", 48, 200, 6000, 8, 5, 128, 32, "e4m3", "bf16", layers=6),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    do = rng.choice(["attend"] * 5 + ["append", "share", "compact", "step", "step"])
    dim = rng.choice([64, 96, 128, 128, 192, 256])
    page = rng.choice([16, 16, 32, 64, 128, 256])
    kind = rng.choice(["bf16", "bf16", "fp16", "e4m3"])
    io = kind if kind != "e4m3" else rng.choice(["bf16", "fp16"])
    kv_heads, group = rng.choice([1, 2, 3, 4, 8, 8, 16]), rng.choice([1, 2, 4, 5, 7, 8, 16, 24, 48])
    token = 2 * kv_heads * dim * (1 if kind == "e4m3" else 2)
    if do == "attend":
        n = _log_int(rng, 1, 256)
        hi = max(2, min(_log_int(rng, 16, 131072), int(2.5e9 / token / n), int(6e8 / n / kv_heads / max(1, group / 8))))
        lo = rng.randint(1, hi)
        window = rng.choice([0, 0, 0, rng.randint(1, hi)])
        return _case("", do, n, lo, hi, kv_heads, group, dim, page, kind, io, window=window,
                     empty=rng.randint(0, n // 8), lse=rng.random() < 0.5)
    layers = rng.randint(1, 8)
    if do == "step":
        n = _log_int(rng, 1, 96)
        hi = max(2, min(_log_int(rng, 32, 8000), int(1e9 / token / n / layers)))
        return _case("", do, n, rng.randint(1, hi), hi, kv_heads, group, dim, page, kind, io, layers=layers)
    kind = io = rng.choice(["bf16", "fp16"])  # what is returned here is the cache itself
    token = 2 * kv_heads * dim * 2
    if do == "append":
        n = _log_int(rng, 1, 300)
        new_hi = rng.choice([1, rng.randint(2, 9), max(2, min(_log_int(rng, 16, 4000), int(1e9 / token / n / layers)))])
        hi = max(2, min(_log_int(rng, 16, 4000), int(1e9 / token / n / layers)))
        return _case("", do, n, rng.randint(0, hi), hi, kv_heads, group, dim, page, kind, io, layers=layers,
                     new=(1, new_hi))
    if do == "share":
        n, parents = _log_int(rng, 1, 300), rng.randint(1, 12)
        hi = max(2, min(_log_int(rng, 16, 60000), int(1e9 / token / parents / layers)))
        return _case("", do, n, rng.randint(1, hi), hi, kv_heads, group, dim, page, kind, io, layers=layers,
                     parents=parents, new=(1, rng.choice([1, 2, 40])))
    n = _log_int(rng, 4, 500)
    hi = max(2, min(_log_int(rng, 32, 4000), int(2e9 / token / n / layers)))
    return _case("", do, n, rng.randint(1, hi), hi, kv_heads, group, dim, page, kind, io, layers=layers)


# ---- sizes: the same for every seed, so that a case's work is one number --------------------------------------
def _sizes(case):
    """(tokens each sequence holds, new tokens each gets) of a case."""
    rng = random.Random(case["n"] * 1000003 + case["hi"])
    many = case["parents"] if case["do"] == "share" else case["n"]
    held = [rng.randint(case["lo"], case["hi"]) for _ in range(many)]
    for i in range(case["empty"]):
        held[(i * 7 + 1) % many] = 0
    new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(case["n"])]
    return held, new


def _up(a, b):
    return -(-a // b)


def _forked(case, held):
    """Tokens of its parent each child starts with, in the order of the children."""
    rng = random.Random(case["n"] + 5)
    return [max(1, held[i % len(held)] - rng.randint(0, held[i % len(held)] // 3)) for i in range(case["n"])]


def _heads(case):
    return case["kv_heads"] * case["group"]


def work(case):
    held, new = _sizes(case)
    b = 1 if case["kind"] == "e4m3" else 2
    T, L = case["page"], case["layers"]
    token = 2 * case["kv_heads"] * case["dim"] * b  # a token's key and value in one layer
    rows = 2 * case["kv_heads"] * case["dim"] * 2   # ... as they arrive
    qo = 2 * _heads(case) * case["dim"] * 2         # a query and its output
    if case["do"] in ("attend", "step"):
        one = case["do"] == "step"
        seen = sum(min(x + one, case["window"] or x + one) for x in held)
        flops = 4 * seen * _heads(case) * case["dim"] * L
        moved = L * (seen * token + case["n"] * (qo + (rows if one else 0)))
        return {"bytes": moved + 4 * sum(_up(x, T) for x in held), "flops": flops}
    if case["do"] == "append":
        return {"bytes": sum(new) * (L * (rows + token) + 4) + 4 * sum(_up(x + y, T) - _up(x, T)
                                                                      for x, y in zip(held, new)), "flops": 0}
    if case["do"] == "share":
        start = _forked(case, held)
        copied = sum(x % T for x in start) * L * token
        pages = sum(_up(x, T) for x in start)
        return {"bytes": 2 * copied + 24 * pages + 4 * sum(new), "flops": 0}
    _, moves = _holes(case, held)
    return {"bytes": 2 * moves * T * L * token + 8 * sum(_up(x, T) for x in held), "flops": 0}


def _holes(case, held):
    """(pages that were taken, pages that move) of a compaction: every third sequence's pages are free."""
    each = [_up(x, case["page"]) for x in held]
    live = sum(p for i, p in enumerate(each) if i % 3 != 1)
    at, moves = 0, 0
    for i, p in enumerate(each):
        if i % 3 == 1:
            moves += max(0, min(live, at + p) - at)
        at += p
    return at, moves


# ---- inputs ---------------------------------------------------------------------------------------------------
def _pool(shape, dtype, gen):
    x = torch.empty(shape, dtype=torch.bfloat16 if dtype == torch.float8_e4m3fn else dtype, device=DEVICE)
    x.normal_(generator=gen)
    return x.to(dtype)


def _words(taken):
    """The free bits of pages: set where `taken` is not."""
    P = taken.numel()
    bits = torch.zeros(_up(P, 64) * 64, dtype=torch.int64, device=taken.device)
    bits[:P] = (~taken).to(torch.int64)
    return (bits.view(-1, 64) << torch.arange(64, device=taken.device)).sum(1)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    cpu = torch.Generator().manual_seed(int(seed))
    held, new = _sizes(case)
    do, n, T, L, H, D = (case[x] for x in ("do", "n", "page", "layers", "kv_heads", "dim"))
    kind, io = DTYPES[case["kind"]], DTYPES[case["io"]]
    first = [_up(x, T) for x in held]
    if do == "share":
        children = _forked(case, held)
        room = sum(_up(x + y, T) - x // T for x, y in zip(children, new))
        most = max([_up(x, T) for x in held] + [_up(x + y, T) for x, y in zip(children, new)])
    else:
        add = new if do in ("append", "step") else [0] * n
        room = sum(_up(x + y, T) - _up(x, T) for x, y in zip(held, add))
        most = max(1, max(_up(x + y, T) for x, y in zip(held, add)))
    P = sum(first) + room + 3
    S = len(held) + (n if do == "share" else 0) + 2
    # a service that has run for a while: a sequence's pages lie anywhere, its slot too
    ids = torch.randperm(P, generator=cpu)[:sum(first)] if do != "compact" else torch.arange(sum(first))
    rows = torch.randperm(S, generator=cpu)
    meta = torch.zeros(2 * _up(P, 64) + S * most + S + P, dtype=torch.int32, device=DEVICE)
    W = 2 * _up(P, 64)
    free, table = meta[:W].view(torch.int64), meta[W:W + S * most].view(S, most)
    lengths, refs = meta[W + S * most:W + S * most + S], meta[W + S * most + S:]
    host = torch.full((S, most), -1, dtype=torch.int32)
    size = torch.zeros(S, dtype=torch.int32)
    count = torch.zeros(P, dtype=torch.int32)
    at = 0
    for i, p in enumerate(first):
        if not (do == "compact" and i % 3 == 1):
            host[rows[i], :p] = ids[at:at + p].to(torch.int32)
            size[rows[i]] = held[i]
            count[ids[at:at + p]] = 1
        at += p
    table.copy_(host)
    lengths.copy_(size)
    refs.copy_(count)
    free.copy_(_words(refs > 0))
    s = {"case": case, "table": table, "lengths": lengths, "refs": refs, "free": free, "meta": meta,
         "k": _pool((L, P, H, D // 8, T, 8), kind, gen), "v": _pool((L, P, H, T // 4, D, 4), kind, gen),
         "k_scale": 0.75 if case["kind"] == "e4m3" else 1.0, "v_scale": 0.05 if case["kind"] == "e4m3" else 1.0,
         "scale": D ** -0.5, "window": case["window"]}
    slot = rows.to(torch.int32).to(DEVICE)
    s["slots"] = slot[:len(held)].contiguous()
    if do == "share":
        s["src"] = slot[torch.arange(n, device=DEVICE) % len(held)].contiguous()
        s["slots"] = slot[len(held):len(held) + n].contiguous()
        s["tokens"] = torch.tensor(children, dtype=torch.int32, device=DEVICE)
        s["none"] = torch.zeros(n, dtype=torch.int32, device=DEVICE)
    if do in ("append", "share", "step"):
        off = torch.zeros(n + 1, dtype=torch.int64)
        off[1:] = torch.cumsum(torch.tensor(new), 0)
        s["offsets"], s["rows"] = off.to(DEVICE), int(off[-1])
    if do in ("append", "step"):
        s["keep"] = torch.tensor(held, dtype=torch.int32, device=DEVICE)
        # rows as a fused projection leaves them: keys and values of one token side by side
        s["kv"] = torch.empty((L, s["rows"], 2, H, D), dtype=io, device=DEVICE).normal_(generator=gen)
    if do in ("attend", "step"):
        s["q"] = torch.empty((L, n, _heads(case), D), dtype=io, device=DEVICE).normal_(0, 3.0, generator=gen)
    if do == "compact":
        s["before"] = meta.clone()
    if own:
        from paper_2606_17059_amd import KVCache
        s["cache"] = KVCache(s["k"], s["v"], table, lengths, refs, free, k_scale=s["k_scale"], v_scale=s["v_scale"])
    return s


def _take(pool, layer, pages):
    return pool.view(torch.uint8)[layer][pages].view(pool.dtype)


# ---- plain forms ----------------------------------------------------------------------------------------------
def _attend(s, layer, q):
    """(out, log of the sum of exponentials) of one new token a sequence."""
    n, heads, D = q.shape
    H, T = s["k"].shape[2], s["k"].shape[4]
    size = s["lengths"][s["slots"].long()].long()
    pages = s["table"][s["slots"].long()].clamp(min=0).long()
    ctx = pages.shape[1] * T
    k = _take(s["k"], layer, pages).float().permute(0, 2, 1, 4, 3, 5).reshape(n, H, ctx, D)
    x = torch.matmul(q.float().view(n, H, heads // H, D), k.transpose(2, 3)) * (s["scale"] * s["k_scale"])
    del k
    at = torch.arange(ctx, device=q.device)
    seen = at < size[:, None]
    if s["window"]:
        seen &= at >= (size - s["window"])[:, None]
    x = x.masked_fill(~seen[:, None, None], -math.inf)
    top = x.amax(3, keepdim=True)
    top = top.masked_fill(top == -math.inf, 0.0)
    p = torch.exp(x - top)
    total = p.sum(3, keepdim=True)
    v = _take(s["v"], layer, pages).float().permute(0, 2, 1, 3, 5, 4).reshape(n, H, ctx, D)
    out = torch.matmul(p, v) * s["v_scale"] / total.masked_fill(total == 0, 1.0)
    return out.view(n, heads, D).to(q.dtype), (top + torch.log(total)).view(n, heads)


def _extend(s):
    """Room for the new tokens: where each row goes (page * page_tokens + place in the page)."""
    T = s["k"].shape[4]
    slots, table, refs = s["slots"].long(), s["table"], s["refs"]
    off = s["offsets"]
    start = s["lengths"][slots].long()
    add = off[1:] - off[:-1]
    old = (start + T - 1) // T
    last = table[slots, (old - 1).clamp(min=0)].clamp(min=0).long()
    # the last page is partly filled and not the sequence's alone
    copy = (start % T > 0) & (refs[last] > 1) & (add > 0)
    need = (start + add + T - 1) // T - old + copy
    rank = torch.cumsum(need, 0) - need
    pages = torch.sort(refs > 0, stable=True).indices
    row = torch.arange(s["rows"], device=DEVICE)
    i = torch.searchsorted(off, row, right=True) - 1
    pos = start[i] + row - off[i]
    col = pos // T
    fresh = col >= old[i] - copy[i].long()
    page = torch.where(fresh, pages[(rank[i] + col - old[i] + copy[i]).clamp(min=0)], table[slots[i], col].long())
    refs.index_add_(0, last, -copy.to(torch.int32))
    # a sequence's own copy of its partly filled last page
    some = torch.nonzero(copy)[:, 0]
    src, dst = last[some], pages[rank[some]]
    inside = torch.arange(T, device=DEVICE) < (start % T)[some, None]
    k, v = s["k"], s["v"]
    k[:, dst] = torch.where(inside[None, :, None, None, :, None], k[:, src], k[:, dst])
    v[:, dst] = torch.where(inside.view(1, -1, 1, T // 4, 1, 4), v[:, src], v[:, dst])
    table[slots[i], col] = page.to(torch.int32)
    refs[page[fresh]] = 1
    s["lengths"][slots] = (start + add).to(torch.int32)
    s["free"].copy_(_words(refs > 0))
    return (page * T + pos % T).to(torch.int32)


def _write(s, layer, place, rows):
    """Rows [r, 2, kv_heads, head_dim] into their places."""
    T, kind = s["k"].shape[4], s["k"].dtype
    page, t = place.long() // T, place.long() % T
    x = rows.float()
    if kind == torch.float8_e4m3fn:
        top = torch.finfo(kind).max
        x = (x / torch.tensor([s["k_scale"], s["v_scale"]], device=DEVICE)[:, None, None]).clamp(-top, top)
    x = x.to(kind).view(torch.uint8 if kind == torch.float8_e4m3fn else torch.int16)
    k, v = s["k"].view(x.dtype), s["v"].view(x.dtype)
    k[layer, page, :, :, t] = x[:, 0].reshape(x.shape[0], x.shape[2], -1, 8)
    v[layer, page, :, t // 4, :, t % 4] = x[:, 1]


def _trim(s, keep):
    T = s["k"].shape[4]
    slots = s["slots"].long()
    to = torch.minimum(s["lengths"][slots], keep)
    rows = s["table"][slots]
    gone = (torch.arange(rows.shape[1], device=DEVICE) >= ((to.long() + T - 1) // T)[:, None]) & (rows >= 0)
    s["refs"].index_add_(0, rows.clamp(min=0).long().flatten(), -gone.flatten().to(torch.int32))
    s["table"][slots] = rows.masked_fill(gone, -1)
    s["lengths"][slots] = to
    s["free"].copy_(_words(s["refs"] > 0))


def _fork(s):
    T = s["k"].shape[4]
    rows = s["table"][s["src"].long()]
    got = torch.arange(rows.shape[1], device=DEVICE) < ((s["tokens"].long() + T - 1) // T)[:, None]
    s["table"][s["slots"].long()] = rows.masked_fill(~got, -1)
    s["refs"].index_add_(0, rows.clamp(min=0).long().flatten(), got.flatten().to(torch.int32))
    s["lengths"][s["slots"].long()] = s["tokens"]
    s["free"].copy_(_words(s["refs"] > 0))


def _compact(s):
    refs, P = s["refs"], s["refs"].numel()
    ids = torch.arange(P, device=DEVICE)
    live = refs > 0
    count = live.sum()
    dst, src = torch.nonzero(~live & (ids < count))[:, 0], torch.nonzero(live & (ids >= count))[:, 0]
    s["k"][:, dst] = s["k"][:, src]
    s["v"][:, dst] = s["v"][:, src]
    to = torch.arange(P, dtype=torch.int32, device=DEVICE)
    to[src] = dst.to(torch.int32)
    table = s["table"]
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()], table))
    refs[dst] = refs[src]
    refs[src] = 0
    s["free"].copy_(_words(refs > 0))
    return torch.stack([dst.new_tensor(dst.numel()), count]).to(torch.int32)


# ---- one pass -------------------------------------------------------------------------------------------------
def _state(s):
    return {x: s[x] for x in ("k", "v", "table", "lengths", "refs", "free")}


def run(s):
    case, c = s["case"], s.get("cache")
    do = case["do"]
    if do == "attend":
        if own:
            lse = torch.empty(s["q"].shape[1:3], dtype=torch.float32, device=DEVICE) if case["lse"] else None
            out = c.attend(0, s["slots"], s["q"][0], s["scale"], window=s["window"], lse=lse)
        else:
            out, lse = _attend(s, 0, s["q"][0])
        return {"out": out, "lse": lse} if case["lse"] else {"out": out}
    if do == "append":
        if own:
            c.trim(s["slots"], s["keep"])
            place = c.extend(s["slots"], s["offsets"], s["rows"])
            for layer in range(case["layers"]):
                c.write(layer, place, s["kv"][layer, :, 0], s["kv"][layer, :, 1])
        else:
            _trim(s, s["keep"])
            place = _extend(s)
            for layer in range(case["layers"]):
                _write(s, layer, place, s["kv"][layer])
        return {"place": place, **_state(s)}
    if do == "share":
        if own:
            c.trim(s["slots"], s["none"])
            c.fork(s["src"], s["slots"], s["tokens"])
            place = c.extend(s["slots"], s["offsets"], s["rows"])
        else:
            _trim(s, s["none"])
            _fork(s)
            place = _extend(s)
        return {"place": place, **_state(s)}
    if do == "compact":
        s["meta"].copy_(s["before"])
        moved = c.compact() if own else _compact(s)
        return {"moved": moved, **_state(s)}
    out = []
    if own:
        c.trim(s["slots"], s["keep"])
        place = c.extend(s["slots"], s["offsets"], s["rows"])
        for layer in range(case["layers"]):
            c.write(layer, place, s["kv"][layer, :, 0], s["kv"][layer, :, 1])
            out.append(c.attend(layer, s["slots"], s["q"][layer], s["scale"]))
    else:
        _trim(s, s["keep"])
        place = _extend(s)
        for layer in range(case["layers"]):
            _write(s, layer, place, s["kv"][layer])
            out.append(_attend(s, layer, s["q"][layer])[0])
    return {"out": out, "place": place, "table": s["table"], "lengths": s["lengths"]}


# ---- in 64 bits -----------------------------------------------------------------------------------------------
def _e4m3(x):
    """The nearest e4m3 value, ties to the even one: 3 bits behind the leading one, exponents from -6, at most 448."""
    a = x.abs().clamp(max=448.0)
    step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)
    return torch.sign(x) * (torch.round(a / step) * step).clamp(max=448.0)


def exact(case, seed):
    """Attention one sequence at a time from its pages' numbers, in double precision."""
    if case["do"] not in ("attend", "step"):
        return None  # these outputs are whole numbers and numbers that were moved
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    T, D, H = case["page"], case["dim"], case["kv_heads"]
    outs, lses = [], []
    for layer in range(case["layers"]):
        out = torch.zeros(s["q"].shape[1:], dtype=torch.float64, device=DEVICE)
        lse = torch.full(s["q"].shape[1:3], -math.inf, dtype=torch.float64, device=DEVICE)
        for i, slot in enumerate(s["slots"].tolist()):
            size = int(s["lengths"][slot])
            if not size and case["do"] == "attend":
                continue
            held = s["table"][slot, :_up(size, T)].long()
            k = _take(s["k"], layer, held).double().transpose(2, 3).reshape(len(held), H, T, D)
            v = _take(s["v"], layer, held).double().transpose(3, 4).reshape(len(held), H, T, D)
            k = k.transpose(0, 1).reshape(H, -1, D)[:, :size] * s["k_scale"]
            v = v.transpose(0, 1).reshape(H, -1, D)[:, :size] * s["v_scale"]
            if case["do"] == "step":
                new = s["kv"][layer, i].double()
                if case["kind"] == "e4m3":
                    unit = torch.tensor([s["k_scale"], s["v_scale"]], dtype=torch.float64, device=DEVICE)[:, None, None]
                    new = _e4m3(new / unit) * unit
                k, v = torch.cat([k, new[0][:, None]], 1), torch.cat([v, new[1][:, None]], 1)
            if case["window"]:
                k, v = k[:, -case["window"]:], v[:, -case["window"]:]
            q = s["q"][layer, i].double().view(H, -1, D)
            x = torch.bmm(q, k.transpose(1, 2).contiguous()) * s["scale"]
            lse[i] = torch.logsumexp(x, 2).flatten()
            out[i] = torch.bmm(torch.softmax(x, 2), v.contiguous()).reshape(-1, D)
        outs.append(out)
        lses.append(lse)
    if case["do"] == "step":
        return {"out": outs, "place": None, "table": None, "lengths": None}
    return {"out": outs[0], "lse": lses[0]} if case["lse"] else {"out": outs[0]}

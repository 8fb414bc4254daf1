"""Performance cases of the prefix cache's operators: what a serving worker runs below the plan.

Each case is one call that a user of this library makes, on seeded synthetic inputs:

  tables  block tables and slot maps of a batch, from the resident chunks, the requests' prefix
          nodes and their lengths
  write   new keys and values into the pages that the slot map names
  attend  attention of the batch's new tokens over the paged cache, single tokens included

`own` False computes the same in plain torch operations, in 32 bits, rounded once at the end.
"""

import math
import random

import numpy as np
import torch

own = False

HOP = 14    # ancestors a line of the prefix table moves up by; its last two are the next hop and the depth
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
E4M3_MAX = 448.0


# ------------------------------------------------------------------ cases ---

def _tables(name, n, depth, chain, slots, requests, starts, suffix, tick, most, page, chunk=512):
    """`starts` of the requests begin in this step, with up to `suffix` tokens of their own behind the
    prefix; the others go on by `tick` tokens.  No request gets more than `most` tokens."""
    c = dict(kind="tables", n=n, depth=depth, chain=chain, slots=slots, requests=requests, starts=starts,
             suffix=suffix, tick=tick, most=most, page=page, chunk=chunk)
    return c if name is None else dict(c, name=name)


def _write(name, tokens, heads, dim, dtype, cache, page):
    c = dict(kind="write", tokens=tokens, heads=heads, dim=dim, dtype=dtype, cache=cache, page=page)
    return c if name is None else dict(c, name=name)


def _attend(name, requests, singles, new, len_lo, len_hi, heads, kv_heads, dim, dtype, cache, page, window=0):
    """`singles` of the requests have one new token, the others up to `new`."""
    c = dict(kind="attend", requests=requests, singles=singles, new=new, len_lo=len_lo, len_hi=len_hi, heads=heads,
             kv_heads=kv_heads, dim=dim, dtype=dtype, cache=cache, page=page, window=window)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # a decode step of a small batch: nothing but latency
        _tables("tables_tick64", 2_000, 12, 0.2, 256, 64, 0, 700, 1, 1, 16),
        # a burst of new requests over a document pool, all looked up in the tree
        _tables("tables_admit257", 10_000, 8, 0.2, 1_024, 257, 257, 1_000, 1, 1_021, 32),
        # a large worker in the middle of long conversations, one request in eight new
        _tables("tables_step4096", 50_000, 64, 0.9, 4_096, 4_096, 512, 2_048, 1, 512, 16),
        # the keys and values of a decode step
        _write("write_tick61", 61, 2, 128, "bf16", "bf16", 16),
        # a prefill step into an 8-bit cache, odd number of tokens
        _write("write_8191_e4m3", 8_191, 8, 128, "f16", "e4m3", 32),
        # the largest step: a budget of 65,536 tokens
        _write("write_65536", 65_536, 8, 128, "bf16", "bf16", 16),
        # one user's next token behind a chunked prefix
        _attend("attend_one", 1, 1, 1, 4_097, 4_097, 16, 2, 128, "bf16", "bf16", 16),
        # a decode batch, lengths spread, seven query heads to a key head
        _attend("attend_tick64", 64, 64, 1, 500, 8_190, 28, 4, 128, "bf16", "bf16", 16),
        # a large decode batch over an 8-bit cache
        _attend("attend_tick256_e4m3", 256, 256, 1, 1_024, 16_384, 40, 8, 128, "bf16", "e4m3", 32),
        # one missing chunk of 512 tokens recomputed behind a long resident prefix
        _attend("attend_chunk512", 1, 0, 512, 33_280, 33_280, 16, 2, 128, "bf16", "bf16", 16),
        # prefill chunks among decoding requests, a sliding window, odd sizes
        _attend("attend_mixed33", 33, 29, 509, 700, 9_001, 28, 4, 64, "f16", "f16", 16, window=4_096),
        # the largest: long prompts in chunks of 2,048
        _attend("attend_prefill4", 4, 0, 2_048, 8_192, 16_384, 32, 8, 128, "bf16", "bf16", 64),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["tables", "write", "attend", "attend", "attend"])
    page = rng.choice([16, 16, 32, 64])
    if kind == "tables":
        n = log_int(200, 50_000)
        depth = log_int(4, 64)
        requests = log_int(1, 4_096)
        starts = rng.choice([0, requests, requests // 8, rng.randint(0, requests)])
        return _tables(None, n, depth, rng.choice([0.2, 0.6, 0.9]), max(1, min(n, log_int(16, 4_096))), requests, starts,
                       log_int(16, 2_048), rng.choice([1, 1, 4]), log_int(4, 2_048 if requests < 1_024 else 512), page)
    heads, kv_heads = rng.choice([(8, 8), (16, 2), (28, 4), (32, 8), (40, 8), (12, 1)])
    dim = rng.choice([64, 128, 128, 256])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    cache = rng.choice([dtype, dtype, "e4m3"])
    if kind == "write":
        return _write(None, min(log_int(1, 65_536), 65_536 * 1_024 // (kv_heads * dim)), kv_heads, dim, dtype, cache, page)
    requests = log_int(1, 128)
    form = rng.choice(["singles", "few", "chunks", "mixed"])
    new = {"singles": 1, "few": rng.randint(2, 8)}.get(form) or log_int(16, 2_048)
    singles = {"singles": requests, "mixed": rng.randint(0, requests)}.get(form, 0)
    if form in ("chunks", "mixed"):
        requests = min(requests, 24)
        singles = min(singles, requests)
    hi = max(log_int(64, 16_384), new)
    lo = min(hi, max(1, int(hi * rng.uniform(0.05, 1.0))))
    window = rng.choice([0, 0, 0, log_int(64, 4_096)])
    largest = work(listed()[-1])["flops"]
    while True:  # the plain form pads every request to the longest and the newest
        c = _attend(None, requests, singles, new, lo, hi, heads, kv_heads, dim, dtype, cache, page, window)
        padded = requests * new * hi * heads
        if work(c)["flops"] <= largest / 2 and padded <= 2.5e9 and requests * hi * kv_heads * dim <= 2.2e9:
            return c
        if requests > 1:
            requests = max(1, requests // 2)
            singles = min(singles, requests)
        else:
            new = max(1, new // 2)
            hi = max(new, hi * 3 // 4)
            lo = min(lo, hi)


def _spread(lo, hi, count):
    """`count` whole numbers from lo to hi, even over their logarithm."""
    if count <= 0:
        return []
    if count == 1:
        return [int(hi)]
    return [int(round(math.exp(math.log(lo) + (math.log(hi) - math.log(lo)) * i / (count - 1)))) for i in range(count)]


def _batch(case):
    """(new tokens, length) of an attend case's requests, before the seed shuffles them."""
    many = case["requests"] - case["singles"]
    new = [1] * case["singles"] + _spread(max(1, case["new"] // 2), case["new"], many)
    length = _spread(case["len_lo"], case["len_hi"], case["requests"])
    order = list(range(case["requests"]))
    random.Random(7).shuffle(order)
    length = [length[i] for i in order]
    return [(min(a, b), b) for a, b in zip(new, length)]


def work(case):
    if case["kind"] == "tables":
        R, page = case["requests"], case["page"]
        begun, gone_on = case["starts"], case["requests"] - case["starts"]
        path = case["depth"] / 2                      # chunks looked up, about half of them resident
        tokens = begun * min(case["most"], path * case["chunk"] / 2) + gone_on * min(case["tick"], case["most"])
        placed = tokens / page + begun * path / 2 * case["chunk"] / page
        return {"bytes": int(R * 24 + begun * path * 8 + placed * 8 + tokens * 12), "flops": int(R * 8 + tokens * 4)}
    if case["kind"] == "write":
        values = 2 * case["tokens"] * case["heads"] * case["dim"]
        return {"bytes": values * (2 + (1 if case["cache"] == "e4m3" else 2)) + 8 * case["tokens"], "flops": values}
    w, pairs, rows, keys = case["window"], 0, 0, 0
    for new, length in _batch(case):
        first = length - new
        if w:
            pairs += sum(min(w, p + 1) for p in range(first, length))
            keys += min(length, new + w - 1)
        else:
            pairs += new * first + new * (new + 1) // 2
            keys += length
        rows += new
    size = 1 if case["cache"] == "e4m3" else 2
    return {"bytes": 2 * keys * case["kv_heads"] * case["dim"] * size + rows * case["heads"] * (4 * case["dim"] + 4),
            "flops": 4 * case["dim"] * case["heads"] * pairs}


# ----------------------------------------------------------------- inputs ---

def _tree(case, rng):
    """parent, depth: a forest where a node continues the last one's chain, or branches off an earlier node."""
    n, most = case["n"], case["depth"]
    go_on = rng.random(n) < case["chain"]
    pick = rng.random(n)
    parent = [-1] * n
    depth = [0] * n
    inner = [0]                                        # nodes that may have children
    for v in range(1, n):
        p = v - 1 if go_on[v] and depth[v - 1] < most - 1 else inner[int(pick[v] * len(inner))]
        parent[v] = p
        depth[v] = depth[p] + 1
        if depth[v] < most - 1:
            inner.append(v)
    return np.array(parent, np.int32), np.array(depth, np.int32)


def _lines(parent, depth):
    """The prefix table: line v holds v, its parent and so on, 15 in all (-1 past the root), and v's depth."""
    n = parent.shape[0]
    up = np.concatenate([parent, [-1]]).astype(np.int32)   # up[-1] = -1
    lines = np.empty((n, HOP + 2), np.int32)
    lines[:, 0] = np.arange(n)
    for j in range(1, HOP + 1):
        lines[:, j] = up[lines[:, j - 1]]
    lines[:, HOP + 1] = depth
    return lines


def _prepare_tables(case, seed):
    rng = np.random.default_rng(seed)
    R, page, chunk = case["requests"], case["page"], case["chunk"]
    parent, depth = _tree(case, rng)
    n = parent.shape[0]
    held = np.zeros(n, bool)                            # closed under parents, as a plan's target is
    count = 0
    for v in rng.permutation(n):
        path = []
        while v >= 0 and not held[v]:
            path.append(v)
            v = parent[v]
        if count + len(path) > case["slots"]:
            break
        held[path] = True
        count += len(path)
    slot = np.full(n, -1, np.int32)
    slot[held] = rng.permutation(case["slots"])[:count]
    resident_pages = case["slots"] * (chunk // page)

    leaf = rng.integers(0, n, R).astype(np.int32)
    known = np.flatnonzero(held)
    if known.size:                                      # half the requests ask for what is popular
        popular = rng.random(R) < 0.5
        leaf[popular] = rng.choice(known, int(popular.sum()))
    leaf[rng.random(R) < 0.05] = -1                     # no shared prefix
    begins = np.zeros(R, bool)
    begins[rng.permutation(R)[:case["starts"]]] = True
    prefix = np.where(leaf >= 0, (depth[np.maximum(leaf, 0)] + 1) * chunk, 0)
    own_tokens = np.zeros(R, np.int64)
    own_tokens[begins] = rng.permutation(_spread(1, case["suffix"], case["starts"]))
    length = prefix + own_tokens
    short = begins & (rng.random(R) < 0.1)              # prompts that end inside the path
    length[short] = np.maximum(1, (length[short] * rng.random(int(short.sum()))).astype(np.int64))
    cached = np.full(R, -1, np.int64)
    cached[~begins] = prefix[~begins] + rng.integers(1, case["suffix"] + 1, int((~begins).sum()))
    length[~begins] = cached[~begins] + case["tick"]
    max_blocks = int(-(-(case["depth"] * chunk + case["suffix"] + case["tick"]) // page))

    # what the requests that go on have in their rows, and the pages that are free
    table = np.full((R, max_blocks), -1, np.int32)
    have = np.where(begins, 0, -(-cached // page))
    order = rng.permutation(int(have.sum())).astype(np.int32) + resident_pages
    table[np.arange(max_blocks)[None, :] < have[:, None]] = order
    tokens = case["starts"] * min(case["most"], max_blocks * page) + (R - case["starts"]) * min(case["tick"], case["most"])   # the step's budget
    free = resident_pages + int(have.sum()) + rng.permutation(tokens // page + R + 64).astype(np.int32)
    d = torch.device("cuda")

    def put(a, dtype=np.int32):
        return torch.from_numpy(np.ascontiguousarray(a.astype(dtype))).to(d)

    return dict(case=case, leaf=put(leaf), length=put(length), cached=put(cached), lines=put(_lines(parent, depth)), slot=put(slot),
                free=put(free), block_table=put(table),
                query_start=torch.empty(R + 1, dtype=torch.int32, device=d), start=torch.empty(R, dtype=torch.int32, device=d),
                end=torch.empty(R, dtype=torch.int32, device=d),
                slot_map=torch.empty(tokens, dtype=torch.int64, device=d), position=torch.empty(tokens, dtype=torch.int32, device=d),
                taken=torch.empty(1, dtype=torch.int32, device=d))


def _prepare_write(case, seed):
    d = torch.device("cuda")
    g = torch.Generator(device=d).manual_seed(seed)
    T, H, D, page = case["tokens"], case["heads"], case["dim"], case["page"]
    dtype, cache = DTYPES[case["dtype"]], DTYPES[case["cache"]]
    # the projection's output holds queries, keys and values side by side
    rows = torch.randn((T, 3 * H, D), generator=g, device=d, dtype=dtype)
    pages = -(-T // page) + 7
    pool = torch.zeros((2, pages, H, page, D), device=d, dtype=cache)
    places = torch.randperm(pages * page, generator=g, device=d)[:T]
    if T > 8:
        places[T - 3:] = -1                              # the batch is padded
    s = dict(case=case, k=rows[:, H:2 * H], v=rows[:, 2 * H:], slot_map=places, k_cache=pool[0], v_cache=pool[1], k_scale=None, v_scale=None)
    if case["cache"] == "e4m3":
        s["k_scale"] = 0.01 + 0.02 * torch.rand(H, generator=g, device=d)
        s["v_scale"] = 0.01 + 0.02 * torch.rand(H, generator=g, device=d)
    return s


def _prepare_attend(case, seed):
    d = torch.device("cuda")
    g = torch.Generator(device=d).manual_seed(seed)
    batch = _batch(case)
    random.Random(seed).shuffle(batch)
    page, D, Hq, Hkv = case["page"], case["dim"], case["heads"], case["kv_heads"]
    dtype, cache = DTYPES[case["dtype"]], DTYPES[case["cache"]]
    blocks = [-(-length // page) for _, length in batch]
    max_blocks = max(blocks)
    pages = sum(blocks) + 5
    new = torch.tensor([a for a, _ in batch], dtype=torch.int64)
    T = int(new.sum())
    rows = torch.randn((T, Hq + 2 * Hkv, D), generator=g, device=d, dtype=dtype)
    k = torch.randn((pages, Hkv, page, D), generator=g, device=d, dtype=dtype)
    k += torch.randn((1, Hkv, 1, D), generator=g, device=d, dtype=dtype)    # keys have channels that stand out
    v = torch.randn((pages, Hkv, page, D), generator=g, device=d, dtype=dtype)
    s = dict(case=case, k_scale=None, v_scale=None)
    if case["cache"] == "e4m3":
        s["k_scale"] = 0.5 + torch.rand(Hkv, generator=g, device=d)
        s["v_scale"] = 0.5 + torch.rand(Hkv, generator=g, device=d)
        k, v = k.to(cache), v.to(cache)
    table = torch.full((len(batch), max_blocks), -1, dtype=torch.int32)
    order = torch.randperm(pages, generator=g, device=d).cpu().to(torch.int32)
    at = 0
    for r, b in enumerate(blocks):
        table[r, :b] = order[at:at + b]
        at += b
    s.update(q=rows[:, :Hq], k_cache=k, v_cache=v, block_table=table.to(d),
             query_start=torch.cat([torch.zeros(1, dtype=torch.int64), new.cumsum(0)]).to(torch.int32).to(d),
             length=torch.tensor([b for _, b in batch], dtype=torch.int32).to(d),
             out=torch.empty((T, Hq, D), dtype=dtype, device=d), lse=torch.empty((T, Hq), dtype=torch.float32, device=d),
             scale=1.0 / math.sqrt(D), window=case["window"], max_new=int(new.max()), max_len=max(b for _, b in batch))
    return s


def prepare(case, seed):
    return {"tables": _prepare_tables, "write": _prepare_write, "attend": _prepare_attend}[case["kind"]](case, seed)


# -------------------------------------------------------------------- run ---

def _run_tables(s):
    case = s["case"]
    page, chunk = case["page"], case["chunk"]
    if own:
        from paper_2608_01655_amd import binding as B

        B.pp_block_tables(s["leaf"], s["length"], s["cached"], s["lines"], s["slot"], s["free"], s["block_table"], s["query_start"],
                          s["start"], s["end"], s["slot_map"], s["position"], s["taken"], page_size=page, chunk_tokens=chunk,
                          n_slots=case["slots"], max_new=case["most"])
        return {k: s[k] for k in ("block_table", "query_start", "start", "end", "slot_map", "position", "taken")}
    leaf, length, cached, lines, slot, free, old = (s[k].long() for k in ("leaf", "length", "cached", "lines", "slot", "free", "block_table"))
    R, max_blocks = old.shape
    d = leaf.device
    begins = cached < 0
    at = torch.where(begins, leaf, -1)
    deep = torch.where(at >= 0, lines[at.clamp(min=0), HOP + 1] + 1, 0)
    ups = []
    for _ in range((case["depth"] - 1) // HOP + 1):      # line by line up the path
        line = torch.where((at >= 0)[:, None], lines[at.clamp(min=0)], -1)
        ups.append(line[:, :HOP])
        at = line[:, HOP]
    up = torch.cat(ups, 1)                               # leaf to root
    i = torch.arange(up.shape[1], device=d)[None, :]
    path = torch.gather(up, 1, (deep[:, None] - 1 - i).clamp(min=0))   # root to leaf
    there = torch.where(i < deep[:, None], slot[path.clamp(min=0)], -1)
    ok = (there >= 0) & (there < case["slots"])
    hit = ok.long().cumprod(1).sum(1)
    start = torch.where(begins, chunk * torch.minimum(hit, (length - 1).clamp(min=0) // chunk), torch.minimum(cached, length))
    end = torch.minimum(length, start + case["most"])
    new = end - start
    query_start = torch.cat([new.new_zeros(1), new.cumsum(0)])
    first_block = (start + page - 1) // page
    need = (end + page - 1) // page - first_block
    first_page = need.cumsum(0) - need
    b = torch.arange(max_blocks, device=d)[None, :]
    per = chunk // page
    shared = torch.gather(there, 1, (b // per).clamp(max=there.shape[1] - 1).expand(R, -1)) * per + b % per
    taken = first_page[:, None] + b - first_block[:, None]
    fresh = torch.where(taken < free.shape[0], free[taken.clamp(0, free.shape[0] - 1)], -1)
    table = torch.where(begins[:, None] & (b < first_block[:, None]), shared, old)
    table = torch.where((b >= first_block[:, None]) & (b < first_block[:, None] + need[:, None]), fresh, table)
    t = torch.arange(s["slot_map"].shape[0], device=d)
    r = (torch.searchsorted(query_start, t, right=True) - 1).clamp(max=R - 1)
    live = t < query_start[-1]
    position = torch.where(live, start[r] + t - query_start[r], 0)
    on = table[r, position // page]
    place = torch.where(live & (on >= 0), on * page + position % page, -1)
    return {"block_table": table.int(), "query_start": query_start.int(), "start": start.int(), "end": end.int(), "slot_map": place,
            "position": position.int(), "taken": need.sum().int().reshape(1)}


def _run_write(s):
    if own:
        from paper_2608_01655_amd import binding as B

        B.pp_kv_write(s["k"], s["v"], s["slot_map"], s["k_cache"], s["v_cache"], k_scale=s["k_scale"], v_scale=s["v_scale"])
        return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    page = s["case"]["page"]
    place = s["slot_map"]
    from_row = torch.where(place >= 0, torch.arange(place.shape[0], device=place.device), 0)   # padding repeats token 0
    to = place[from_row]
    for x, cache, scale in ((s["k"], s["k_cache"], s["k_scale"]), (s["v"], s["v_cache"], s["v_scale"])):
        x = x[from_row].float()
        if scale is not None:
            x = (x / scale[None, :, None]).clamp(-E4M3_MAX, E4M3_MAX)
        x = x.to(cache.dtype)
        bits = torch.uint8 if cache.dtype == torch.float8_e4m3fn else torch.int16
        cache.view(bits)[to // page, :, to % page] = x.view(bits)
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _rows(cache, table):
    """The cache rows of every request in order, padded: [requests][heads][blocks * page][dim], 32 bits."""
    bits = torch.uint8 if cache.dtype == torch.float8_e4m3fn else torch.int16
    x = cache.view(bits)[table].view(cache.dtype)        # [R][blocks][H][page][D]
    R, n, H, page, D = x.shape
    return x.permute(0, 2, 1, 3, 4).float().reshape(R, H, n * page, D)


def _run_attend(s):
    if own:
        from paper_2608_01655_amd import binding as B

        B.pp_paged_attention(s["q"], s["k_cache"], s["v_cache"], s["block_table"], s["query_start"], s["length"], s["out"], s["lse"],
                             scale=s["scale"], window=s["window"], max_new=s["max_new"], max_len=s["max_len"], k_scale=s["k_scale"],
                             v_scale=s["v_scale"])
        return {"out": s["out"], "lse": s["lse"]}
    q, length, begin = s["q"], s["length"].long(), s["query_start"].long()
    T, Hq, D = q.shape
    Hkv = s["k_cache"].shape[1]
    G = Hq // Hkv
    new = begin[1:] - begin[:-1]
    R, N = new.shape[0], s["max_new"]
    d = q.device
    i = torch.arange(N, device=d)
    x = q[(begin[:-1, None] + i[None, :]).clamp(max=T - 1)].float()              # [R][N][Hq][D]
    x = x.reshape(R, N, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(R, Hkv, N * G, D) * s["scale"]
    if s["k_scale"] is not None:
        x = x * s["k_scale"][None, :, None, None]
    table = s["block_table"].long().clamp(min=0)
    k = _rows(s["k_cache"], table).transpose(2, 3).contiguous()
    p = torch.matmul(x, k)                                                       # [R][Hkv][N * G][keys]
    del k
    j = torch.arange(p.shape[3], device=d)
    at = (length - new)[:, None] + i[None, :]                                    # [R][N]
    seen = (j <= at[:, :, None]) & (j < length[:, None, None])
    if s["window"]:
        seen &= j > at[:, :, None] - s["window"]
    p = p.view(R, Hkv, N, G, -1).masked_fill_(~seen[:, None, :, None, :], -math.inf).view(R, Hkv, N * G, -1)
    m = p.amax(3, keepdim=True)
    p = p.sub_(torch.where(m > -math.inf, m, 0.0)).exp_()
    l = p.sum(3, keepdim=True)
    v = _rows(s["v_cache"], table)
    v *= (j < length[:, None])[:, None, :, None]
    o = torch.matmul(p, v) / torch.where(l > 0, l, 1.0)
    if s["v_scale"] is not None:
        o = o * s["v_scale"][None, :, None, None]
    lse = (m + l.log()).reshape(R, Hkv, N, G)
    o = o.reshape(R, Hkv, N, G, D)
    t = torch.arange(T, device=d)
    r = torch.searchsorted(begin, t, right=True) - 1
    n = t - begin[r]
    return {"out": o[r, :, n].reshape(T, Hq, D).to(q.dtype), "lse": lse[r, :, n].reshape(T, Hq)}


def run(s):
    return {"tables": _run_tables, "write": _run_write, "attend": _run_attend}[s["case"]["kind"]](s)


# ------------------------------------------------------------------ exact ---

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "tables":
        return _exact_tables(s)
    if case["kind"] == "write":
        return _exact_write(s)
    return _exact_attend(s)


def _exact_tables(s):
    """Request by request, as the definition reads."""
    case = s["case"]
    page, chunk = case["page"], case["chunk"]
    per = chunk // page
    leaf, length, cached, slot, free = (s[k].cpu().tolist() for k in ("leaf", "length", "cached", "slot", "free"))
    parent = s["lines"][:, 1].cpu().tolist()
    table = s["block_table"].cpu().numpy().copy()
    query_start, starts, ends, places, positions, taken = [0], [], [], [], [], 0
    for r in range(len(leaf)):
        if cached[r] < 0:
            path, v = [], leaf[r]
            while v >= 0:
                path.insert(0, v)
                v = parent[v]
            start = 0
            for v in path:
                if not 0 <= slot[v] < case["slots"] or start + chunk >= length[r]:
                    break
                table[r, start // page:start // page + per] = slot[v] * per + np.arange(per)
                start += chunk
        else:
            start = min(cached[r], length[r])
        end = min(length[r], start + case["most"])
        for b in range(-(-start // page), -(-end // page)):
            table[r, b] = free[taken]
            taken += 1
        pos = np.arange(start, end)
        places.append(table[r, pos // page].astype(np.int64) * page + pos % page)
        positions.append(pos)
        starts.append(start)
        ends.append(end)
        query_start.append(query_start[-1] + end - start)
    pad = s["slot_map"].shape[0] - query_start[-1]
    return {"block_table": table, "query_start": np.array(query_start, np.int32), "start": np.array(starts, np.int32), "end": np.array(ends, np.int32),
            "slot_map": np.concatenate(places + [np.full(pad, -1, np.int64)]),
            "position": np.concatenate(positions + [np.zeros(pad, np.int64)]).astype(np.int32), "taken": np.array([taken], np.int32)}


def _exact_write(s):
    """The value that each place stands for before it is rounded to the cache's type."""
    page = s["case"]["page"]
    got = {}
    place = s["slot_map"].cpu()
    live = place >= 0
    for name, x, scale in (("k_cache", s["k"], s["k_scale"]), ("v_cache", s["v"], s["v_scale"])):
        full = s[name].cpu().to(torch.float64)
        y = x.cpu().to(torch.float64)
        if scale is not None:
            y = torch.clamp(y / scale.cpu().to(torch.float64)[None, :, None], -E4M3_MAX, E4M3_MAX)
        by_token = full.permute(0, 2, 1, 3).reshape(-1, full.shape[1], full.shape[3]).clone()
        by_token[place[live]] = y[live]
        got[name] = by_token.reshape(full.shape[0], page, full.shape[1], full.shape[3]).permute(0, 2, 1, 3).contiguous()
    return got


def _exact_attend(s):
    """Request by request and key head by key head, on its own keys only."""
    page, w = s["case"]["page"], s["window"]
    begin, length = s["query_start"].tolist(), s["length"].tolist()
    T, Hq, D = s["q"].shape
    Hkv = s["k_cache"].shape[1]
    G = Hq // Hkv
    out = torch.zeros((T, Hq, D), dtype=torch.float64, device=s["q"].device)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64, device=s["q"].device)
    for r, n in enumerate(length):
        pages = s["block_table"][r:r + 1, :-(-n // page)].long()
        rows = slice(begin[r], begin[r + 1])
        at = torch.arange(n - (begin[r + 1] - begin[r]), n, device=out.device)
        j = torch.arange(n, device=out.device)
        hidden = j[None, :] > at[:, None]
        if w:
            hidden |= j[None, :] <= at[:, None] - w
        for h in range(Hkv):
            k, v = (_rows(s[c][:, h:h + 1], pages)[0, 0, :n].to(torch.float64) for c in ("k_cache", "v_cache"))
            ks = 1.0 if s["k_scale"] is None else s["k_scale"][h].to(torch.float64)
            vs = 1.0 if s["v_scale"] is None else s["v_scale"][h].to(torch.float64)
            for head in range(h * G, h * G + G):
                e = (s["q"][rows, head].to(torch.float64) @ k.T) * (s["scale"] * ks)
                e[hidden] = -math.inf
                lse[rows, head] = torch.logsumexp(e, 1)
                out[rows, head] = (torch.softmax(e, 1) @ v) * vs
    return {"out": out, "lse": lse}

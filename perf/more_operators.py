"""Performance cases of the operators around a worker's pages: what brings rows into them, what reads
pages of latent rows, and what moves, shares and frees pages.

Each case is one call that a user of this library makes, on seeded synthetic inputs:

  rotary  norms of queries and keys for each head, rotation by position, and the write into the pages
  latent  attention of new tokens over pages of one latent row a token, which all heads share
  copy    pages copied from place to place, in the pools of all layers
  fork    block table rows of beams or samples from their parents' rows
  free    the pages that no row names

`own` False computes the same in plain torch operations, in 32 bits, rounded once at the end.
"""

import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
BITS = {"bf16": torch.int16, "f16": torch.int16, "e4m3": torch.uint8}
E4M3_MAX = 448.0
EPS = 1e-6


# ------------------------------------------------------------------ cases ---

def _named(name, c):
    return c if name is None else dict(c, name=name)


def _rotary(name, tokens, heads, kv_heads, dim, rot, interleaved, norm, far, factor, dtype, cache, page, latent=0):
    """Positions below `far`, frequencies scaled by `factor`.  With `latent`, the key rows are one a token of
    latent + rot elements, the latent normed and the rest rotated, and there are no values."""
    return _named(name, dict(kind="rotary", tokens=tokens, heads=heads, kv_heads=kv_heads, dim=dim, rot=rot, interleaved=interleaved,
                             norm=norm, far=far, factor=factor, dtype=dtype, cache=cache, page=page, latent=latent))


def _latent(name, requests, singles, new, len_lo, len_hi, heads, latent, rot, dtype, cache, page, window=0):
    """`singles` of the requests have one new token, the others up to `new`."""
    return _named(name, dict(kind="latent", requests=requests, singles=singles, new=new, len_lo=len_lo, len_hi=len_hi, heads=heads,
                             latent=latent, rot=rot, dtype=dtype, cache=cache, page=page, window=window))


def _copy(name, moves, pools, heads, dim, dtype, page, partial):
    """`partial` of the moves copy the first tokens of a page only, and some name no page."""
    return _named(name, dict(kind="copy", moves=moves, pools=pools, heads=heads, dim=dim, dtype=dtype, page=page, partial=partial))


def _fork(name, groups, beams, len_lo, len_hi, page):
    """`groups` requests of `beams` rows each, whose new rows come from any row of the request."""
    return _named(name, dict(kind="fork", groups=groups, beams=beams, len_lo=len_lo, len_hi=len_hi, page=page))


def _free(name, requests, len_lo, len_hi, page, shared, spare):
    """Rows share the pages of their first `shared` blocks among four; `spare` more pages than the rows name."""
    return _named(name, dict(kind="free", requests=requests, len_lo=len_lo, len_hi=len_hi, page=page, shared=shared, spare=spare))


def listed():
    return [
        # a decode step's queries and keys, normed and rotated whole: nothing but latency
        _rotary("rotary_tick61", 61, 28, 4, 128, 128, False, True, 8_190, 1.0, "bf16", "bf16", 16),
        # the largest step, a budget of 65,536 tokens far into long contexts, half of each head rotated, 8-bit pages
        _rotary("rotary_65536_e4m3", 65_536, 32, 8, 128, 64, True, False, 1_000_000, 8.0, "bf16", "e4m3", 32),
        # one user's next token behind a chunked prefix
        _latent("latent_one", 1, 1, 1, 4_097, 4_097, 16, 512, 64, "bf16", "bf16", 16),
        # a decode batch over 8-bit latents, lengths spread, the heads of one GPU of eight
        _latent("latent_tick64_e4m3", 64, 64, 1, 500, 16_383, 16, 512, 64, "bf16", "e4m3", 32),
        # a decode batch with all heads on one GPU
        _latent("latent_tick48_all", 48, 48, 1, 500, 8_190, 128, 512, 64, "bf16", "bf16", 16),
        # the largest: prompts in chunks of up to 2,048 among decoding requests, behind long resident prefixes
        _latent("latent_prefill5", 5, 1, 2_048, 4_096, 16_384, 16, 512, 64, "f16", "f16", 64),
        # the open pages of a few forked requests, in four layers' pools
        _copy("copy_open29", 29, 8, 2, 128, "bf16", 16, 1.0),
        # 16 chunks of 512 tokens from requests' pages into slots, 16 layers
        _copy("copy_chunks512", 512, 32, 8, 128, "bf16", 16, 0.0),
        # a beam step of a small batch
        _fork("fork_beams8x8", 8, 8, 300, 5_001, 16),
        # a beam step of a large batch of long conversations
        _fork("fork_beams512x8", 512, 8, 512, 16_384, 16),
        # a small batch between two steps
        _free("free_64", 64, 300, 8_190, 16, 32, 4_099),
        # a large worker
        _free("free_4096", 4_096, 512, 16_384, 16, 64, 100_003),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["rotary", "rotary", "latent", "latent", "latent", "copy", "fork", "free"])
    page = rng.choice([16, 16, 32, 64])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    cache = rng.choice([dtype, dtype, "e4m3"])
    if kind == "rotary":
        far, factor, interleaved = log_int(64, 1_000_000), rng.choice([1.0, 1.0, 8.0, 40.0]), rng.choice([False, True])
        if rng.random() < 0.3:
            heads = rng.choice([16, 20, 128])
            return _rotary(None, min(log_int(1, 65_536), 4_000_000 // (heads * 64)), heads, 1, 64, 64, interleaved, False, far, factor,
                           dtype, cache, page, latent=rng.choice([256, 512]))
        heads, kv_heads = rng.choice([(8, 8), (16, 2), (28, 4), (32, 8), (40, 8), (12, 1)])
        dim = rng.choice([64, 128, 128, 256])
        rot = rng.choice([dim, dim, dim // 2, dim // 4])
        tokens = min(log_int(1, 65_536), 65_536 * 40 * 128 // ((heads + kv_heads) * dim))
        return _rotary(None, tokens, heads, kv_heads, dim, rot, interleaved, rng.choice([False, True]), far, factor, dtype, cache, page)
    if kind == "copy":
        pools, heads, dim = rng.randint(1, 32), rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 256])
        moves = max(1, min(log_int(1, 4_096), 512 * 32 * 16 * 1_024 // (pools * heads * dim * page)))
        return _copy(None, moves, pools, heads, dim, cache, page, rng.choice([0.0, 0.0, 0.3, 1.0]))
    if kind == "fork":
        beams = rng.randint(1, 16)
        hi = log_int(16, 16_384)
        return _fork(None, max(1, log_int(1, 4_096) // beams), beams, max(1, int(hi * rng.uniform(0.05, 1.0))), hi, page)
    if kind == "free":
        hi = log_int(16, 16_384)
        return _free(None, log_int(1, 4_096), max(1, int(hi * rng.uniform(0.05, 1.0))), hi, page, rng.choice([0, 32, 64]), log_int(1, 100_000))
    requests = log_int(1, 128)
    heads = rng.choice([5, 8, 16, 16, 32, 128])
    latent = rng.choice([512, 512, 256])
    form = rng.choice(["singles", "few", "chunks", "mixed"])
    new = {"singles": 1, "few": rng.randint(2, 8)}.get(form) or log_int(16, 2_048)
    singles = {"singles": requests, "mixed": rng.randint(0, requests)}.get(form, 0)
    if form in ("chunks", "mixed"):
        requests = min(requests, 24)
        singles = min(singles, requests)
    hi = max(log_int(64, 16_384), new)
    lo = min(hi, max(1, int(hi * rng.uniform(0.05, 1.0))))
    window = rng.choice([0, 0, 0, log_int(64, 4_096)])
    largest = max(work(c)["flops"] for c in listed())
    while True:  # the plain form pads every request to the longest and the newest
        c = _latent(None, requests, singles, new, lo, hi, heads, latent, 64, dtype, cache, page, window)
        padded = requests * new * hi * heads
        if work(c)["flops"] <= largest / 2 and padded <= 2.5e9 and requests * hi * (latent + 64) <= 2.2e9:
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
    """(new tokens, length) of a latent case's requests, before the seed shuffles them."""
    many = case["requests"] - case["singles"]
    new = [1] * case["singles"] + _spread(max(1, case["new"] // 2), case["new"], many)
    length = _spread(case["len_lo"], case["len_hi"], case["requests"])
    order = list(range(case["requests"]))
    random.Random(7).shuffle(order)
    length = [length[i] for i in order]
    return [(min(a, b), b) for a, b in zip(new, length)]


def _size(dtype):
    return 1 if dtype == "e4m3" else 2


def work(case):
    kind = case["kind"]
    if kind == "rotary":
        row = case["latent"] + case["rot"] if case["latent"] else 2 * case["kv_heads"] * case["dim"]
        q = case["heads"] * case["dim"]
        return {"bytes": case["tokens"] * (4 * q + (2 + _size(case["cache"])) * row + 12), "flops": 6 * case["tokens"] * (q + row)}
    if kind == "copy":
        share = 1 - case["partial"] / 2
        row = case["heads"] * case["dim"] * _size(case["dtype"])
        return {"bytes": int(2 * case["moves"] * share * case["pools"] * case["page"] * row), "flops": case["moves"]}
    if kind in ("fork", "free"):
        rows = case["groups"] * case["beams"] if kind == "fork" else case["requests"]
        blocks = sum(-(-n // case["page"]) for n in _spread(case["len_lo"], case["len_hi"], rows))
        return {"bytes": 8 * blocks + 28 * rows if kind == "fork" else 4 * (blocks + rows + case["spare"]), "flops": blocks}
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
    C, D = case["latent"], case["latent"] + case["rot"]
    return {"bytes": keys * D * _size(case["cache"]) + rows * case["heads"] * (2 * D + 2 * C + 4), "flops": 2 * (C + D) * case["heads"] * pairs}


# ----------------------------------------------------------------- inputs ---

def _frequencies(case):
    """Radians a token of the rotated pairs.  With a factor above 1, pairs that turn fewer than once in the 4,096
    tokens a model has been trained on slow down by it, those of 32 turns and more keep their pace, and in between
    the two are mixed evenly over the turns."""
    w = 10_000.0 ** (-np.arange(0, case["rot"], 2, dtype=np.float64) / case["rot"])
    if case["factor"] == 1.0:
        return w
    keep = np.clip((4_096 * w / (2 * math.pi) - 1.0) / 31.0, 0.0, 1.0)
    return keep * w + (1 - keep) * w / case["factor"]


def _amplitude(case):
    return 1.0 if case["factor"] == 1.0 else 0.1 * math.log(case["factor"]) + 1.0


def _prepare_rotary(case, seed):
    d = torch.device("cuda")
    g = torch.Generator(device=d).manual_seed(seed)
    T, H, Hk, D, page, C = (case[k] for k in ("tokens", "heads", "kv_heads", "dim", "page", "latent"))
    dtype, cache = DTYPES[case["dtype"]], DTYPES[case["cache"]]
    row = C + case["rot"] if C else D
    s = dict(case=case, v=None, v_cache=None, k_scale=None, v_scale=None, q_weight=None, k_weight=None)
    pages = -(-T // page) + 7
    if C:                                                # queries and latent rows come of two products
        q = torch.randn((T, H, 2 * D + D), generator=g, device=d, dtype=dtype)
        s["q"] = q[:, :, 2 * D:]
        s["k"] = torch.randn((T, 1, row), generator=g, device=d, dtype=dtype) * 3
        s["k_cache"] = torch.zeros((pages, 1, page, row), device=d, dtype=cache)
        s["k_weight"] = (0.5 + torch.rand(C, generator=g, device=d)).to(dtype)
    else:                                                # one product's output: queries, keys and values side by side
        rows = torch.randn((T, H + 2 * Hk, D), generator=g, device=d, dtype=dtype)
        s["q"], s["k"], s["v"] = rows[:, :H], rows[:, H:H + Hk], rows[:, H + Hk:]
        pool = torch.zeros((2, pages, Hk, page, D), device=d, dtype=cache)
        s["k_cache"], s["v_cache"] = pool[0], pool[1]
        if case["norm"]:
            s["q_weight"], s["k_weight"] = ((0.5 + torch.rand(D, generator=g, device=d)).to(dtype) for _ in range(2))
    s["q_out"] = torch.empty((T, H, D), device=d, dtype=dtype)
    if case["cache"] == "e4m3":
        s["k_scale"] = 0.01 + 0.02 * torch.rand(Hk, generator=g, device=d)
        s["v_scale"] = None if C else 0.01 + 0.02 * torch.rand(Hk, generator=g, device=d)
    places = torch.randperm(pages * page, generator=g, device=d)[:T]
    if T > 8:
        places[T - 3:] = -1                              # the batch is padded
    s["slot_map"] = places
    s["position"] = torch.randint(0, case["far"], (T,), generator=g, device=d, dtype=torch.int32)
    if own:                                              # a program lays these out once
        from paper_2608_01655_amd import binding as B

        scaled = {} if case["factor"] == 1.0 else dict(factor=case["factor"], original=4_096, slow=1.0, fast=32.0)
        s["turns"] = torch.from_numpy(B.pp_rotary_turns(case["rot"], 10_000.0, **scaled)).to(d)
    else:
        s["frequency"] = torch.from_numpy(_frequencies(case)).to(d)
    return s


def _prepare_latent(case, seed):
    d = torch.device("cuda")
    g = torch.Generator(device=d).manual_seed(seed)
    batch = _batch(case)
    random.Random(seed).shuffle(batch)
    page, H, C, D = case["page"], case["heads"], case["latent"], case["latent"] + case["rot"]
    dtype, cache = DTYPES[case["dtype"]], DTYPES[case["cache"]]
    blocks = [-(-length // page) for _, length in batch]
    pages = sum(blocks) + 5
    new = torch.tensor([a for a, _ in batch], dtype=torch.int64)
    T = int(new.sum())
    c = torch.randn((pages, 1, page, D), generator=g, device=d, dtype=dtype)
    c += torch.randn((1, 1, 1, D), generator=g, device=d, dtype=dtype)      # channels that stand out
    s = dict(case=case, k_scale=None)
    if case["cache"] == "e4m3":
        s["k_scale"] = 0.5 + torch.rand(1, generator=g, device=d)
        c = c.to(cache)
    table = torch.full((len(batch), max(blocks)), -1, dtype=torch.int32)
    order = torch.randperm(pages, generator=g, device=d).cpu().to(torch.int32)
    at = 0
    for r, b in enumerate(blocks):
        table[r, :b] = order[at:at + b]
        at += b
    s.update(q=torch.randn((T, H, D), generator=g, device=d, dtype=dtype), cache=c, block_table=table.to(d),
             query_start=torch.cat([torch.zeros(1, dtype=torch.int64), new.cumsum(0)]).to(torch.int32).to(d),
             length=torch.tensor([b for _, b in batch], dtype=torch.int32).to(d),
             out=torch.empty((T, H, C), dtype=dtype, device=d), lse=torch.empty((T, H), dtype=torch.float32, device=d),
             scale=1.0 / math.sqrt(128 + case["rot"]), window=case["window"], max_new=int(new.max()), max_len=max(b for _, b in batch))
    return s


def _prepare_copy(case, seed):
    d = torch.device("cuda")
    g = torch.Generator(device=d).manual_seed(seed)
    n, page = case["moves"], case["page"]
    pages = 2 * n + 3
    dtype = DTYPES[case["dtype"]]
    pool = torch.randn((case["pools"], pages, case["heads"], page, case["dim"]), generator=g, device=d, dtype=torch.bfloat16).to(dtype)
    order = torch.randperm(pages, generator=g, device=d).to(torch.int32)
    source, target = order[:n].clone(), order[n:2 * n].clone()
    if n > 8:                                            # rows that keep their pages have no move
        source[5] = -1
        target[7] = -1
    tokens = None
    if case["partial"]:
        part = torch.rand(n, generator=g, device=d) < case["partial"]
        tokens = torch.where(part, torch.randint(0, page + 1, (n,), generator=g, device=d), page).to(torch.int32)
    return dict(case=case, pools=list(pool), source=source, target=target, tokens=tokens)


def _tables(rng, length, page, first, spare=0):
    """(block table of rows of `length` tokens with pages of their own from `first` on, pages past them)."""
    blocks = -(-length // page)
    table = np.full((length.shape[0], max(1, int(blocks.max()))), -1, np.int32)
    total = int(blocks.sum())
    order = (first + rng.permutation(total + spare)).astype(np.int32)
    table[np.arange(table.shape[1])[None, :] < blocks[:, None]] = order[:total]
    return table, order[total:]


def _put(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a.astype(dtype))).to("cuda")


def _prepare_fork(case, seed):
    rng = np.random.default_rng(seed)
    R = case["groups"] * case["beams"]
    length = rng.permutation(np.array(_spread(case["len_lo"], case["len_hi"], R), np.int64))
    table, free = _tables(rng, length, case["page"], 1_000, spare=R + 3)
    parent = np.arange(R) // case["beams"] * case["beams"] + rng.integers(0, case["beams"], R)
    parent[rng.random(R) < 0.02] = -1                    # rows that are through
    d = torch.device("cuda")

    def empty(n):
        return torch.empty(n, dtype=torch.int32, device=d)

    return dict(case=case, parent=_put(parent), length=_put(length), block_table=_put(table), free=_put(free),
                out_table=torch.full(table.shape, -1, dtype=torch.int32, device=d), out_length=empty(R), source=empty(R), target=empty(R),
                tokens=empty(R), taken=empty(1))


def _prepare_free(case, seed):
    rng = np.random.default_rng(seed)
    R, first = case["requests"], 8_192
    length = rng.permutation(np.array(_spread(case["len_lo"], case["len_hi"], R), np.int64))
    table, _ = _tables(rng, length, case["page"], first, spare=case["spare"])
    total = int((-(-length // case["page"])).sum()) + case["spare"]
    shared = min(case["shared"], table.shape[1])
    for r in range(R):
        full = min(shared, int(length[r]) // case["page"])
        q = r // 4 * 4
        full = min(full, int(length[q]) // case["page"])
        if r % 8 < 4:                                    # four rows of one request
            table[r, :full] = table[q, :full]
        else:                                            # behind the same resident chunks
            table[r, :full] = np.arange(full) + int(rng.integers(0, 16)) * shared
    d = torch.device("cuda")
    n_pages = first + total
    return dict(case=case, block_table=_put(table), length=_put(length), first=first, n_pages=n_pages,
                marks=torch.empty(n_pages, dtype=torch.uint8, device=d), free=torch.full((n_pages - first,), -1, dtype=torch.int32, device=d),
                count=torch.empty(1, dtype=torch.int32, device=d))


def prepare(case, seed):
    return {"rotary": _prepare_rotary, "latent": _prepare_latent, "copy": _prepare_copy, "fork": _prepare_fork,
            "free": _prepare_free}[case["kind"]](case, seed)


# -------------------------------------------------------------------- run ---

def _results(s, *names):
    return {k: s[k] for k in names if s[k] is not None}


def _normed(x, weight):
    if weight is None:
        return x
    n = weight.shape[0]
    y = x[..., :n]
    y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * weight.float()
    return torch.cat([y, x[..., n:]], -1)


def _turned(x, first, cos, sin, interleaved):
    """x with the elements from `first` on rotated; cos, sin [tokens][1][pairs]."""
    n = 2 * cos.shape[-1]
    y = x[..., first:first + n]
    a, b = (y[..., 0::2], y[..., 1::2]) if interleaved else (y[..., :n // 2], y[..., n // 2:])
    a, b = a * cos - b * sin, a * sin + b * cos
    y = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([x[..., :first], y, x[..., first + n:]], -1)


def _run_rotary(s):
    case = s["case"]
    C, page = case["latent"], case["page"]
    if own:
        from paper_2608_01655_amd import binding as B

        B.pp_rotary_write(s["position"], s["turns"], q=s["q"], q_out=s["q_out"], k=s["k"], v=s["v"], slot_map=s["slot_map"],
                          k_cache=s["k_cache"], v_cache=s["v_cache"], k_scale=s["k_scale"], v_scale=s["v_scale"], q_weight=s["q_weight"],
                          k_weight=s["k_weight"], eps=EPS, k_first=C, interleaved=case["interleaved"], amplitude=_amplitude(case))
        return _results(s, "q_out", "k_cache", "v_cache")
    angle = s["position"].double()[:, None] * s["frequency"]
    cos, sin = ((f(angle) * _amplitude(case)).float()[:, None] for f in (torch.cos, torch.sin))
    s["q_out"].copy_(_turned(_normed(s["q"].float(), s["q_weight"]), 0, cos, sin, case["interleaved"]))
    k = _turned(_normed(s["k"].float(), s["k_weight"]), C, cos, sin, case["interleaved"])
    place = s["slot_map"]
    from_row = torch.where(place >= 0, torch.arange(place.shape[0], device=place.device), 0)   # padding repeats token 0
    to = place[from_row]
    bits = BITS[case["cache"]]
    for x, cache, scale in ((k, s["k_cache"], s["k_scale"]), (s["v"], s["v_cache"], s["v_scale"])):
        if x is None:
            continue
        x = x[from_row].float()
        if scale is not None:
            x = (x / scale[None, :, None]).clamp(-E4M3_MAX, E4M3_MAX)
        cache.view(bits)[to // page, :, to % page] = x.to(cache.dtype).view(bits)
    return _results(s, "q_out", "k_cache", "v_cache")


def _run_latent(s):
    if own:
        from paper_2608_01655_amd import binding as B

        B.pp_latent_attention(s["q"], s["cache"], s["block_table"], s["query_start"], s["length"], s["out"], s["lse"], scale=s["scale"],
                              window=s["window"], max_new=s["max_new"], max_len=s["max_len"], k_scale=s["k_scale"])
        return {"out": s["out"], "lse": s["lse"]}
    case = s["case"]
    C, D = case["latent"], case["latent"] + case["rot"]
    q, length, begin = s["q"], s["length"].long(), s["query_start"].long()
    T, H, _ = q.shape
    new = begin[1:] - begin[:-1]
    R, N = new.shape[0], s["max_new"]
    d = q.device
    i = torch.arange(N, device=d)
    x = q[(begin[:-1, None] + i[None, :]).clamp(max=T - 1)].float().reshape(R, N * H, D) * s["scale"]
    if s["k_scale"] is not None:
        x = x * s["k_scale"]
    c = s["cache"].view(BITS[case["cache"]])[s["block_table"].long().clamp(min=0)].view(s["cache"].dtype).float()
    c = c.reshape(R, -1, D)                                                      # rows in order, padded
    p = torch.matmul(x, c.transpose(1, 2).contiguous())                          # [R][N * H][keys]
    j = torch.arange(p.shape[2], device=d)
    at = (length - new)[:, None] + i[None, :]                                    # [R][N]
    seen = (j <= at[:, :, None]) & (j < length[:, None, None])
    if s["window"]:
        seen &= j > at[:, :, None] - s["window"]
    p = p.view(R, N, H, -1).masked_fill_(~seen[:, :, None, :], -math.inf).view(R, N * H, -1)
    m = p.amax(2, keepdim=True)
    p = p.sub_(torch.where(m > -math.inf, m, 0.0)).exp_()
    l = p.sum(2, keepdim=True)
    v = c[:, :, :C].contiguous()
    v *= (j < length[:, None])[:, :, None]
    o = torch.matmul(p, v) / torch.where(l > 0, l, 1.0)
    if s["k_scale"] is not None:
        o = o * s["k_scale"]
    lse = (m + l.log()).reshape(R, N, H)
    o = o.reshape(R, N, H, C)
    t = torch.arange(T, device=d)
    r = torch.searchsorted(begin, t, right=True) - 1
    n = t - begin[r]
    return {"out": o[r, n].to(q.dtype), "lse": lse[r, n]}


def _run_copy(s):
    if own:
        from paper_2608_01655_amd import binding as B

        B.pp_page_copy(s["pools"], s["source"], s["target"], s["tokens"])
        return s["pools"]
    bits, page = BITS[s["case"]["dtype"]], s["case"]["page"]
    source, target = s["source"].long(), s["target"].long()
    n = source.shape[0]
    ok = (source >= 0) & (target >= 0)
    move = torch.where(ok, torch.arange(n, device=ok.device), 0)                  # what names no page repeats move 0
    source, target = source[move], target[move]
    j = torch.arange(page, device=ok.device)
    for pool in s["pools"]:
        pool = pool.view(bits)
        rows = pool[source]
        if s["tokens"] is not None:
            rows = torch.where((j < s["tokens"][move, None])[:, None, :, None], rows, pool[target])
        pool[target] = rows
    return s["pools"]


def _run_fork(s):
    case = s["case"]
    page = case["page"]
    names = ("out_table", "out_length", "source", "target", "tokens", "taken")
    if own:
        from paper_2608_01655_amd import binding as B

        B.pp_fork_tables(s["parent"], s["length"], s["block_table"], s["free"], *(s[k] for k in names), page_size=page)
        return {k: s[k] for k in names}
    parent, length, table, free = (s[k].long() for k in ("parent", "length", "block_table", "free"))
    R, blocks = table.shape
    row = torch.arange(R, device=parent.device)
    live = parent >= 0
    at = parent.clamp(min=0)
    n = torch.where(live, length[at], 0)
    first = torch.full((R + 1,), R, dtype=torch.int64, device=parent.device)      # a parent's first new row
    first.scatter_reduce_(0, torch.where(live, parent, R), row, "amin")
    copied = live & (n % page > 0) & (first[at] != row)
    rank = copied.long().cumsum(0) - copied.long()
    fresh = free[rank.clamp(max=free.shape[0] - 1)]
    b = torch.arange(blocks, device=parent.device)[None, :]
    old = s["out_table"].long()
    new = torch.where(b < ((n + page - 1) // page)[:, None], table[at], old)
    last = b == (n // page)[:, None]
    new = torch.where(last & copied[:, None], fresh[:, None], new)
    source = torch.where(copied, torch.gather(table[at], 1, (n // page).clamp(max=blocks - 1)[:, None])[:, 0], -1)
    out = (new, n, source, torch.where(copied, fresh, -1), torch.where(copied, n % page, 0), copied.sum().reshape(1))
    return {k: x.int() for k, x in zip(names, out)}


def _run_free(s):
    page, first, n_pages = s["case"]["page"], s["first"], s["n_pages"]
    if own:
        from paper_2608_01655_amd import binding as B

        B.pp_free_pages(s["block_table"], s["length"], s["free"], s["count"], s["marks"], page_size=page, first=first)
        return {"free": s["free"], "count": s["count"]}
    table, length = s["block_table"].long(), s["length"].long()
    b = torch.arange(table.shape[1], device=table.device)[None, :]
    named = (b < ((length + page - 1) // page)[:, None]) & (table >= 0)
    mark = torch.zeros(n_pages + 1, dtype=torch.int64, device=table.device)
    mark[torch.where(named, table, n_pages)] = 1
    here = 1 - mark[first:n_pages]
    to = torch.where(here > 0, here.cumsum(0) - 1, n_pages - first)
    free = torch.full((n_pages - first + 1,), -1, dtype=torch.int32, device=table.device)
    free[to] = torch.arange(first, n_pages, dtype=torch.int32, device=table.device)
    free[n_pages - first] = -1
    return {"free": free[:n_pages - first], "count": here.sum().int().reshape(1)}


def run(s):
    return {"rotary": _run_rotary, "latent": _run_latent, "copy": _run_copy, "fork": _run_fork, "free": _run_free}[s["case"]["kind"]](s)


# ------------------------------------------------------------------ exact ---

def exact(case, seed):
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "latent": _exact_latent, "copy": _exact_copy, "fork": _exact_fork, "free": _exact_free}[case["kind"]](s)


def _exact_rotary(s):
    """Pairs as complex numbers, and the values that places stand for before they are rounded to the cache's type."""
    case = s["case"]
    C, page, rot = case["latent"], case["page"], case["rot"]
    w = torch.from_numpy(_frequencies(case)).to(s["q"].device)
    turn = torch.polar(torch.full_like(w, _amplitude(case)).expand(case["tokens"], -1).contiguous(), s["position"].double()[:, None] * w)[:, None]

    def rows(x, weight, first):
        x = x.double()
        if weight is not None:
            head = x[..., :weight.shape[0]]
            rms = (head.square().sum(-1, keepdim=True) / weight.shape[0] + EPS).sqrt()
            x[..., :weight.shape[0]] = head / rms * weight.double()
        part = x[..., first:first + rot]
        shape = part.shape[:-1]
        pairs = part.reshape(*shape, rot // 2, 2) if case["interleaved"] else part.reshape(*shape, 2, rot // 2).transpose(-1, -2)
        z = torch.view_as_real(torch.complex(pairs[..., 0], pairs[..., 1]) * turn)
        x[..., first:first + rot] = (z if case["interleaved"] else z.transpose(-1, -2)).reshape(*shape, rot)
        return x

    got = {"q_out": rows(s["q"], s["q_weight"], 0)}
    live = s["slot_map"] >= 0
    for name, x, scale in (("k_cache", rows(s["k"], s["k_weight"], C), s["k_scale"]), ("v_cache", s["v"], s["v_scale"])):
        if x is None:
            continue
        y = x.double()
        if scale is not None:
            y = torch.clamp(y / scale.double()[None, :, None], -E4M3_MAX, E4M3_MAX)
        P, H, _, D = s[name].shape
        by_token = torch.zeros((P * page, H, D), dtype=torch.float64, device=y.device)
        by_token[s["slot_map"][live]] = y[live]
        got[name] = by_token.reshape(P, page, H, D).permute(0, 2, 1, 3).contiguous()
    return got


def _exact_latent(s):
    """Request by request and head by head, on its own rows only."""
    case = s["case"]
    page, w, C = case["page"], s["window"], case["latent"]
    begin, length = s["query_start"].tolist(), s["length"].tolist()
    T, H, D = s["q"].shape
    out = torch.zeros((T, H, C), dtype=torch.float64, device=s["q"].device)
    lse = torch.full((T, H), -math.inf, dtype=torch.float64, device=s["q"].device)
    for r, n in enumerate(length):
        pages = s["block_table"][r, :-(-n // page)].long()
        c = s["cache"].view(BITS[case["cache"]])[pages].view(s["cache"].dtype).reshape(-1, D)[:n].to(torch.float64)
        if s["k_scale"] is not None:
            c = c * s["k_scale"].to(torch.float64)
        rows = slice(begin[r], begin[r + 1])
        at = torch.arange(n - (begin[r + 1] - begin[r]), n, device=out.device)
        j = torch.arange(n, device=out.device)
        hidden = j[None, :] > at[:, None]
        if w:
            hidden |= j[None, :] <= at[:, None] - w
        for h in range(H):
            e = (s["q"][rows, h].to(torch.float64) @ c.T) * s["scale"]
            e[hidden] = -math.inf
            lse[rows, h] = torch.logsumexp(e, 1)
            out[rows, h] = torch.softmax(e, 1) @ c[:, :C]
    return {"out": out, "lse": lse}


def _exact_copy(s):
    """Move by move."""
    case = s["case"]
    n = case["moves"]
    source, target = s["source"].tolist(), s["target"].tolist()
    tokens = [case["page"]] * n if s["tokens"] is None else s["tokens"].tolist()
    pools = [p.view(BITS[case["dtype"]]).clone() for p in s["pools"]]
    for a, b, t in zip(source, target, tokens):
        if a >= 0 and b >= 0:
            for p in pools:
                p[b, :, :t] = p[a, :, :t]
    return [p.view(DTYPES[case["dtype"]]).to(torch.float64) for p in pools]


def _exact_fork(s):
    page = s["case"]["page"]
    parent, length, free = (s[k].tolist() for k in ("parent", "length", "free"))
    table, out = s["block_table"].cpu().numpy(), s["out_table"].cpu().numpy().copy()
    R = len(parent)
    got = {k: np.full(R, v, np.int32) for k, v in (("out_length", 0), ("source", -1), ("target", -1), ("tokens", 0))}
    kept, taken = set(), 0
    for r, p in enumerate(parent):
        if p < 0:
            continue
        n = length[p]
        got["out_length"][r] = n
        blocks = -(-n // page)
        out[r, :blocks] = table[p, :blocks]
        if n % page and p in kept:
            got["source"][r], got["target"][r], got["tokens"][r] = table[p, blocks - 1], free[taken], n % page
            out[r, blocks - 1] = free[taken]
            taken += 1
        kept.add(p)
    return dict(out_table=out, **got, taken=np.array([taken], np.int32))


def _exact_free(s):
    page, first, n_pages = s["case"]["page"], s["first"], s["n_pages"]
    named = np.zeros(n_pages, bool)
    table = s["block_table"].cpu().numpy()
    for r, n in enumerate(s["length"].tolist()):
        named[table[r, :-(-n // page)]] = True
    pages = first + np.flatnonzero(~named[first:])
    return {"free": np.concatenate([pages, np.full(n_pages - first - pages.size, -1)]).astype(np.int32), "count": np.array([pages.size], np.int32)}

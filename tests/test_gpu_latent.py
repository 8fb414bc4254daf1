"""Attention over pages of latent rows on the GPU against a plain 64-bit implementation
(tests/rows_ref.py, where the tolerances are derived)."""

import math

import numpy as np
import pytest
import torch

from paper_2608_01655_amd import binding as B
from tests import rows_ref as R

pytestmark = pytest.mark.gpu
BF, HF, E4 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


@pytest.fixture(autouse=True)
def _say_case(request):
    print(f"\n[case] {request.node.name}", flush=True)
    yield


def close(got, want, tol):
    got = got.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    same = (got == want) | torch.isnan(want)               # infinities
    bad = ~(same | ((got - want).abs() <= tol))
    assert not bool(bad.any()), (int(bad.sum()), float((got - want).abs().nan_to_num().max()), bad.nonzero()[:4].tolist())


def case(new, length, heads, *, latent=512, dtype=BF, cache=BF, page=16, seed=0, spread=1.0, spare=3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    D = latent + 64
    blocks = [-(-n // page) if n > 0 else 0 for n in length]
    pages = sum(blocks) + spare
    rows = torch.randn((pages, 1, page, D), generator=g, device="cuda") + torch.randn(D, generator=g, device="cuda")
    scale = None
    if cache == E4:
        scale = 0.5 + torch.rand(1, generator=g, device="cuda")
    table = torch.full((len(new), max(max(blocks), 1)), -1, dtype=torch.int32)
    order = torch.randperm(pages, generator=g, device="cuda").cpu().to(torch.int32)
    at = 0
    for r, b in enumerate(blocks):
        table[r, :b] = order[at:at + b]
        at += b
    T = sum(new)
    q = (torch.randn((T, heads, D), generator=g, device="cuda") * spread).to(dtype)
    return dict(q=q, cache=rows.to(cache), table=table.cuda(), begin=torch.tensor([0, *np.cumsum(new)], dtype=torch.int32, device="cuda"),
                length=torch.tensor(length, dtype=torch.int32, device="cuda"), latent=latent, scale=192 ** -0.5, ks=scale,
                max_new=max(new), max_len=max(max(length), 0), out=torch.full((T, heads, latent), 7.0, dtype=dtype, device="cuda"),
                lse=torch.full((T, heads), 7.0, device="cuda"), window=0)


def attend(c, **kw):
    a = {k: c[k] for k in ("scale", "max_new", "max_len", "window")}
    B.pp_latent_attention(c["q"], c["cache"], c["table"], c["begin"], c["length"], c["out"], c["lse"], k_scale=c["ks"], **{**a, **kw})
    return c["out"], c["lse"]


def check(c, **kw):
    out, lse = attend(c, **kw)
    torch.cuda.synchronize()
    want, want_lse, tol, tol_lse = R.latent(c["q"], c["cache"], c["table"], c["begin"], c["length"], c["latent"], scale=c["scale"],
                                            window=c["window"], k_scale=c["ks"])
    close(out, want, tol)
    close(lse, want_lse, tol_lse)


TYPES = [(BF, BF), (HF, HF), (BF, E4), (HF, E4)]


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("latent", [512, 256])
@pytest.mark.parametrize("heads", [1, 5, 16, 20, 32, 33, 128])
def test_single_tokens(heads, latent, dtype, cache):
    length = [1, 2, 15, 16, 17, 63, 64, 65, 130, 700]
    check(case([1] * len(length), length, heads, latent=latent, dtype=dtype, cache=cache, seed=heads))


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("latent", [512, 256])
@pytest.mark.parametrize("new,heads", [(2, 8), (2, 16), (3, 11), (7, 16), (40, 16), (65, 4), (130, 2)])
def test_new_tokens(new, heads, latent, dtype, cache):
    length = [new, new + 1, 100 + new, 333 + new]
    check(case([new] * 4, length, heads, latent=latent, dtype=dtype, cache=cache, seed=new))


@pytest.mark.parametrize("dtype,cache,page,latent", [(BF, BF, 16, 512), (HF, E4, 32, 512), (BF, E4, 64, 256), (HF, HF, 1024, 256)])
@pytest.mark.parametrize("window", [0, 1, 50, 200])
def test_mixed_batches(window, dtype, cache, page, latent):
    new = [1, 33, 1, 0, 5, 1, 80, 1]
    length = [400, 433, 1, 77, 205, 64, 80, 900]
    c = case(new, length, 16, latent=latent, dtype=dtype, cache=cache, page=page, seed=window)
    c["window"] = window
    check(c)


@pytest.mark.parametrize("dtype,cache,page,latent", [(BF, BF, 16, 512), (HF, E4, 32, 512), (BF, E4, 64, 256), (HF, HF, 1024, 256)])
@pytest.mark.parametrize("window", [0, 1, 50, 200])
@pytest.mark.parametrize("heads", [16, 7])
def test_mixed_batches_that_may_be_long(heads, window, dtype, cache, page, latent):
    """Where the requests of few rows may have many keys they have launches of their own."""
    new = [1, 33, 1, 0, 5, 1, 80, 2, 1]
    length = [400, 433, 1, 77, 205, 64, 80, 300, 900]
    c = case(new, length, heads, latent=latent, dtype=dtype, cache=cache, page=page, seed=window)
    c["window"] = window
    wide = torch.full((len(new), 200_000 // page), -1, dtype=torch.int32, device="cuda")
    wide[:, :c["table"].shape[1]] = c["table"]
    c["table"] = wide
    check(c, max_len=200_000)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("new,heads,n", [(1, 16, 9000), (1, 128, 5000), (2, 20, 6001), (30, 16, 5000)])
def test_long_requests_in_parts(new, heads, n, dtype, cache):
    c = case([new, new], [n, n // 3], heads, dtype=dtype, cache=cache, seed=n)
    assert B.pp_latent_workspace(c["q"], c["cache"], c["table"], c["latent"], max_new=new, max_len=n) > 0
    check(c)


@pytest.mark.parametrize("dtype,cache,latent", [(BF, BF, 512), (HF, E4, 512), (BF, E4, 256)])
@pytest.mark.parametrize("new,heads", [(1, 16), (1, 64)])
def test_long_requests_in_one_part(new, heads, dtype, cache, latent):
    """A bound on the lengths that is too low makes one part of what is longer: a wave goes through more tiles
    than it has page numbers of at a time, and its ring comes round."""
    c = case([new] * 2, [9000, 4097], heads, latent=latent, dtype=dtype, cache=cache, seed=heads)
    check(c, max_len=100)


def put(c, r, keys, value, dims=slice(None)):
    page = c["cache"].shape[2]
    for j in keys:
        bits = c["cache"].view(torch.uint8) if c["cache"].dtype == E4 else c["cache"]
        at = bits[int(c["table"][r, j // page]), 0, j % page]
        at[dims] = 0x7f if c["cache"].dtype == E4 else value


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("latent", [512, 256])
@pytest.mark.parametrize("new,heads", [(1, 16), (3, 5), (50, 16), (1, 128)])
def test_what_is_not_seen_may_hold_anything(new, heads, latent, dtype, cache):
    """NaN and infinities behind the last token, in other pages, in keys only later rows see, and before a window."""
    n = 150 + new
    c = case([new, new], [n, new + 20], heads, latent=latent, dtype=dtype, cache=cache, seed=3)
    want = [x.clone() for x in attend(c)]
    page = c["cache"].shape[2]
    bad = c["cache"].view(torch.uint8) if cache == E4 else c["cache"]
    named = set(c["table"].flatten().tolist())
    for p in range(bad.shape[0]):
        if p not in named:
            bad[p] = 0x7f if cache == E4 else math.nan
    for r, k in ((0, n), (1, new + 20)):                  # the rest of the last page
        put(c, r, range(k, -(-k // page) * page), math.inf)
    got = [x.clone() for x in attend(c)]
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    c["window"] = 40
    want = [x.clone() for x in attend(c)]
    put(c, 0, range(0, n - new - 39), -math.inf)
    got = [x.clone() for x in attend(c)]
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    c["window"] = 0
    if new > 1:                                           # the last key: the rows before it stay as they are
        c = case([new], [n], heads, latent=latent, dtype=dtype, cache=cache, seed=4)
        want = [x.clone() for x in attend(c)]
        put(c, 0, [n - 1], math.nan, slice(3, 9))
        got = attend(c)
        assert torch.equal(got[0][:-1], want[0][:-1]) and torch.equal(got[1][:-1], want[1][:-1])
        assert bool(torch.isnan(got[0][-1]).all())


@pytest.mark.parametrize("latent", [512, 256])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("new,heads,n", [(2, 8, 60), (40, 16, 300), (40, 16, 6000), (3, 8, 9000)])
def test_infinities_that_are_seen(new, heads, n, dtype, latent):
    """A key that scores -infinity from an infinite element: weight 0, and that element is NaN (0 times it)."""
    c = case([new], [n], heads, latent=latent, dtype=dtype, cache=dtype, seed=5)
    c["q"].abs_().add_(0.01)
    at = n - 2
    page = c["cache"].shape[2]
    c["cache"][int(c["table"][0, at // page]), 0, at % page, [5, latent - 1]] = -math.inf
    check(c)


@pytest.mark.parametrize("latent", [512, 256])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("new,n", [(1, 40), (5, 90), (100, 100), (100, 4000)])
def test_rows_of_minus_infinity(new, n, dtype, latent):
    """A row whose seen keys all score -infinity is empty, whatever their values."""
    c = case([new], [n], 8, latent=latent, dtype=dtype, cache=dtype, seed=6)
    c["q"].abs_().add_(0.01)
    dead = new - new // 4
    put(c, 0, range(n - new + dead), -math.inf, slice(2, 3))
    out, lse = attend(c)
    torch.cuda.synchronize()
    assert bool((out[:dead] == 0).all()) and bool((lse[:dead] == -math.inf).all())
    assert bool(torch.isfinite(lse[dead:]).all())


@pytest.mark.parametrize("heads", [4, 16, 128])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_empty_rows_and_tokens_of_nobody(heads, dtype):
    """Lengths of 0 and below, more new tokens than the length, rows behind the last request."""
    c = case([2, 3, 1, 4, 2], [0, 1, -5, 2, 30], heads, dtype=dtype, cache=dtype, seed=7)
    T = c["q"].shape[0]
    c["begin"][-1] = T - 1                                # one token is nobody's
    c["max_new"] = 4
    check_part = c["out"].clone()
    out, lse = attend(c)
    torch.cuda.synchronize()
    assert torch.equal(out[-1], check_part[-1]) and bool((lse[-1] == 7).all())
    want, want_lse, tol, tol_lse = R.latent(c["q"][:-1], c["cache"], c["table"], c["begin"], c["length"], c["latent"], scale=c["scale"])
    close(out[:-1], want, tol)
    close(lse[:-1], want_lse, tol_lse)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("new,heads,n", [(1, 16, 2000), (1, 128, 2000), (60, 16, 2000)])
def test_maxima_that_grow(new, heads, n, dtype, cache):
    """Scores that rise along the keys, so that what was summed is scaled down many times; a key far above."""
    c = case([new], [n], heads, dtype=dtype, cache=cache, seed=8, spread=0.25)
    page = c["cache"].shape[2]
    c["q"][..., 0] = 4.0
    for j in range(n):
        c["cache"][int(c["table"][0, j // page]), 0, j % page, 0] = j / 40 if j != n // 2 else 100.0
    check(c)


@pytest.mark.parametrize("scale", [-0.1, 0.0, 1.5, -2.0])
@pytest.mark.parametrize("new,heads", [(1, 16), (30, 16)])
def test_scales(new, heads, scale):
    c = case([new] * 2, [200, 300], heads, seed=9, spread=0.5)
    c["scale"] = scale
    check(c)


@pytest.mark.parametrize("new,heads", [(1, 16), (30, 12), (1, 40)])
@pytest.mark.parametrize("dtype,cache", [(BF, BF), (HF, E4)])
def test_strides(new, heads, dtype, cache):
    """Rows in wider rows, pages with gaps, a block table inside a wider one, an output head by head."""
    c = case([new] * 3, [150, 77, 30 + new], heads, dtype=dtype, cache=cache, seed=10)
    T = c["q"].shape[0]
    q = torch.zeros((T, heads + 2, 640), device="cuda", dtype=dtype)[:, 1:-1, 32:608]
    q.copy_(c["q"])
    P, _, page, D = c["cache"].shape
    if cache == E4:
        store = torch.full((P, page, 640), 0x7f, device="cuda", dtype=torch.uint8)
        store[:, :, 16:592] = c["cache"][:, 0].view(torch.uint8)
        pages = store[:, None, :, 16:592].view(E4)
    else:
        store = torch.full((P, page, 640), math.nan, device="cuda", dtype=dtype)
        store[:, :, 16:592] = c["cache"][:, 0]
        pages = store[:, None, :, 16:592]
    table = torch.full((3, c["table"].shape[1] + 9), -1, dtype=torch.int32, device="cuda")[:, 4:-5]
    table.copy_(c["table"])
    out = torch.zeros((heads, T, 520), device="cuda", dtype=dtype).transpose(0, 1)[..., :512]
    check(dict(c, q=q, cache=pages, table=table, out=out))


def test_without_lse_and_bad_pages():
    """Page numbers below 0 act as 0, above the last as the last; tokens past the block table do not exist."""
    c = case([1, 20], [300, 320], 16, seed=11)
    c["table"][0, 3], c["table"][1, 5] = -9, 10 ** 6
    want = R.latent(c["q"], c["cache"], c["table"], c["begin"], c["length"], 512, scale=c["scale"])
    out = c["out"]
    B.pp_latent_attention(c["q"], c["cache"], c["table"], c["begin"], c["length"], out, scale=c["scale"], max_new=20, max_len=320)
    torch.cuda.synchronize()
    close(out, want[0], want[2])
    c["table"] = c["table"][:, :7].contiguous()
    check(c)


def test_expanded_tensors_that_are_read():
    c = case([1, 1, 1], [70, 70, 70], 16, seed=12)
    c["table"][1:] = c["table"][:1]
    q = c["q"][:1, :1].expand(3, 16, 576)
    want = [x.clone() for x in attend(dict(c, q=q.contiguous()))]
    got = attend(dict(c, q=q, table=c["table"][:1].expand(3, -1)))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    with pytest.raises(B.PPError):
        attend(dict(c, out=c["out"][:, :1].expand(3, 16, 512)))


@pytest.mark.parametrize("requests", [65, 300])
def test_many_requests(requests):
    """More of them than a wave has lanes, some without new tokens."""
    new = [0 if r % 7 == 2 else 1 if r % 3 else 2 + r * 5 % 19 for r in range(requests)]
    length = [n + r * 37 % 60 for r, n in enumerate(new)]
    length[requests // 2], length[-1] = 1500, 1400
    check(case(new, length, 16, seed=13))


def check_requests(c, which):
    """Requests `which` of the call against the 64-bit implementation, one at a time."""
    out, lse = attend(c)
    torch.cuda.synchronize()
    begin = c["begin"].tolist()
    cache = c["cache"].cpu()
    for r in which:
        rows = slice(begin[r], begin[r + 1])
        sub = torch.tensor([0, begin[r + 1] - begin[r]], dtype=torch.int32)
        want, want_lse, tol, tol_lse = R.latent(c["q"][rows], cache, c["table"][r:r + 1], sub, c["length"][r:r + 1], c["latent"],
                                                scale=c["scale"], window=c["window"], k_scale=c["ks"])
        close(out[rows], want, tol)
        close(lse[rows], want_lse, tol_lse)


@pytest.mark.parametrize("window", [0, 700])
@pytest.mark.parametrize("dtype,cache,latent", [(BF, BF, 512), (HF, E4, 512), (BF, E4, 256)])
@pytest.mark.parametrize("requests,heads", [(1030, 20), (520, 200)])
def test_more_slots_than_are_cut(requests, heads, dtype, cache, latent, window):
    """So many rows that each block takes 128 of them whole, some of them over more keys than it has page numbers of
    at a time."""
    length = [1 + r % 50 for r in range(requests)]
    long = {3: 4097, 100: 2300, 515: 5000, requests - 1: 2048}
    for r, n in long.items():
        length[r] = n
    c = case([1] * requests, length, heads, latent=latent, dtype=dtype, cache=cache, seed=requests)
    c["window"] = window
    assert B.pp_latent_workspace(c["q"], c["cache"], c["table"], latent, max_new=1, max_len=5000, window=window) == 0
    check_requests(c, [*long, 0, 49, 300])


@pytest.mark.parametrize("window", [0, 300])
@pytest.mark.parametrize("heads,new", [(16, 8200), (40, 3400)])
def test_prompts_of_more_slots_than_are_cut(heads, new, window):
    c = case([new, 3], [new, 600], heads, seed=heads)
    c["window"] = window
    out, lse = attend(c)
    torch.cuda.synchronize()
    cache = c["cache"].cpu()
    for i in (0, 1, 37, new // 2, new - 1):               # single tokens of the prompt
        sub = torch.tensor([0, 1], dtype=torch.int32)
        want, want_lse, tol, tol_lse = R.latent(c["q"][i:i + 1], cache, c["table"][:1], sub, torch.tensor([i + 1]), 512, scale=c["scale"], window=window)
        close(out[i:i + 1], want, tol)
        close(lse[i:i + 1], want_lse, tol_lse)


@pytest.mark.parametrize("requests", [1, 3, 700])
@pytest.mark.parametrize("heads", [16, 128])
def test_shares_of_any_lengths(requests, heads):
    """Blocks whose share is of many requests, of a part of one, or begins and ends inside them."""
    g = np.random.default_rng(requests)
    length = g.integers(0, 40, requests).tolist()
    length[requests // 2] = 3000 if requests > 1 else 130
    length[-1] = 1111
    new = [1 if n else 0 for n in length]
    new[0], length[0] = 1, max(length[0], 1)
    c = case(new, length, heads, seed=requests)
    which = sorted({0, requests // 2, requests - 1, *range(0, requests, 41)})
    check_requests(c, which)


def test_starts_that_are_out_of_order():
    """Requests whose tokens overlap, or lie outside: nothing else is written, and nothing fails."""
    c = case([2] * 40, [70] * 40, 128, seed=19)
    want = [x.clone() for x in attend(c)]
    bad = c["begin"].clone()
    bad[5:35:2] = 0
    bad[6:36:2] = 10 ** 6
    attend(dict(c, begin=bad, out=torch.empty_like(c["out"]), lse=torch.empty_like(c["lse"])), max_new=80)
    torch.cuda.synchronize()
    got = attend(c)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("new,heads", [(1, 16), (24, 16)])
def test_same_bits_again(new, heads):
    c = case([new] * 5, [5000, 4000, 37, 100, 2000], heads, seed=14)
    want = [x.clone() for x in attend(c)]
    for _ in range(3):
        got = attend(c)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("new,heads", [(1, 16), (1, 128), (24, 16)])
def test_captured_and_replayed(new, heads):
    """Two graphs with a workspace each, replayed in turn with eager calls between."""
    graphs = []
    for seed in range(2):
        c = case([new] * 4, [3000, 700, new, 45 + new], heads, seed=seed)
        c["ws"] = torch.empty(B.pp_latent_workspace(c["q"], c["cache"], c["table"], 512, max_new=new, max_len=3000), dtype=torch.uint8, device="cuda")
        attend(c, workspace=c["ws"])
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            attend(c, workspace=c["ws"])
        graphs.append((c, g))
    for turn in range(3):
        for i, (c, g) in enumerate(graphs):
            c["q"].copy_(case([new] * 4, [3000, 700, new, 45 + new], heads, seed=10 * turn + i)["q"])
            c["out"].fill_(3)
            g.replay()
            torch.cuda.synchronize()
            got = c["out"].clone(), c["lse"].clone()
            want = attend(c)
            torch.cuda.synchronize()
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    check(graphs[0][0])


def test_on_another_stream():
    c = case([1, 40], [4000, 4100], 16, seed=15)
    want = [x.clone() for x in attend(c)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = attend(c, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_workspace_that_does_not_do():
    c = case([1], [30_000], 16, seed=16)
    need = B.pp_latent_workspace(c["q"], c["cache"], c["table"], 512, max_new=1, max_len=30_000)
    kept = torch.zeros(need + 256, dtype=torch.uint8, device="cuda")
    for bad in (kept[:64], kept[:need - 1], kept[16:need + 16]):
        with pytest.raises(B.PPError) as e:
            attend(c, workspace=bad)
        assert e.value.code == B.PP_E_ARG
    want = [x.clone() for x in attend(c)]
    got = attend(c, workspace=kept[:need])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_offsets_past_32_bits():
    """Pages and queries whose offsets need more than 32 bits."""
    pages = 2 ** 32 // (16 * 576 * 2) + 100
    cache = torch.zeros((pages, 1, 16, 576), device="cuda", dtype=BF)
    c = case([1, 20], [200, 150], 16, seed=17)
    n = c["cache"].shape[0]
    cache[pages - n:] = c["cache"]
    c["table"] = torch.where(c["table"] >= 0, c["table"] + pages - n, c["table"])
    check(dict(c, cache=cache))


def test_refusals_of_the_binding():
    c = case([1, 3], [70, 80], 16, seed=18)
    for kw in (dict(cache=c["cache"][:, 0]), dict(cache=c["cache"].expand(-1, 2, -1, -1)), dict(q=c["q"][..., :512]), dict(q=c["q"][0]),
               dict(out=c["out"].to(HF)), dict(out=c["out"][:, :8]), dict(table=c["table"].long()), dict(length=c["length"].long()),
               dict(begin=c["begin"][:2]), dict(lse=c["lse"].double()), dict(ks=torch.ones(2, device="cuda")), dict(cache=c["cache"].float()),
               dict(q=c["q"].cpu())):
        with pytest.raises(ValueError):
            attend(dict(c, **kw))
    for kw in (dict(out=c["out"][..., :256]), dict(ks=torch.ones(1, device="cuda")), dict(scale=math.nan), dict(window=-1)):
        with pytest.raises(B.PPError):
            attend(dict(c, **kw))
    D = torch.zeros((9, 1, 16, 640), device="cuda", dtype=BF)
    with pytest.raises(B.PPError):
        attend(dict(c, cache=D, q=torch.zeros((4, 16, 640), device="cuda", dtype=BF)))

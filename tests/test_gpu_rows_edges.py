"""Attention over pages of latent rows where keys that are not finite meet the cuts of a batch."""

import math

import pytest
import torch

from paper_2608_01655_amd import binding as B
from tests import rows_ref as R
from tests.test_gpu_latent import attend, case, check, check_requests, close, put

pytestmark = pytest.mark.gpu
BF, HF, E4 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


@pytest.fixture(autouse=True)
def _say_case(request):
    print(f"\n[case] {request.node.name}", flush=True)
    yield


@pytest.mark.parametrize("latent", [512, 256])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("others", [0, 5])
@pytest.mark.parametrize("new,heads,n,first,dead", [
    (1, 16, 128, 0, 32), (1, 16, 128, 96, 32), (1, 16, 100, 96, 4), (1, 16, 9000, 0, 128), (1, 16, 9000, 512, 16), (3, 5, 60, 0, 48),
    (1, 128, 3000, 0, 256), (1, 128, 3000, 300, 900), (1, 128, 3000, 2990, 10), (40, 16, 6000, 0, 700), (40, 16, 6000, 5950, 20),
    (100, 16, 100, 0, 40), (100, 16, 700, 600, 70)])
def test_runs_of_minus_infinity(new, heads, n, first, dead, others, dtype, latent):
    """Keys that score -infinity from an infinite element, whole tiles, waves' shares and parts of them: the element
    is 0 times an infinity and so NaN in every row that sees one and another key, wherever the batch is cut; rows that
    see no other key are 0."""
    c = case([new] + [1] * others, [n] + [400] * others, heads, latent=latent, dtype=dtype, cache=dtype, seed=20)
    c["q"].abs_().add_(0.01)
    put(c, 0, range(first, first + dead), -math.inf, slice(5, 6))
    want = R.latent(c["q"], c["cache"], c["table"], c["begin"], c["length"], latent, scale=c["scale"])[0]
    assert bool(torch.isnan(want[new - 1, :, 5]).all()) and int(torch.isnan(want).sum()) <= new * heads
    check(c)


@pytest.mark.parametrize("new,heads,n,window", [(1, 16, 9000, 300), (2, 128, 3000, 700), (40, 16, 6000, 500)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_runs_of_minus_infinity_in_a_window(dtype, new, heads, n, window):
    """The same at a window's edge: rows whose window is past them are finite."""
    c = case([new], [n], heads, dtype=dtype, cache=dtype, seed=21)
    c["q"].abs_().add_(0.01)
    c["window"] = window
    put(c, 0, range(n - window - 200, n - window + 1), -math.inf, slice(5, 6))
    check(c)


@pytest.mark.parametrize("scale,k_scale", [(0.0, 1e-8), (0.0, 1e-38), (1e-30, 1e-20), (-1e-36, 1e-9)])
@pytest.mark.parametrize("new,heads", [(1, 16), (30, 16)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_scales_whose_product_vanishes(dtype, new, heads, scale, k_scale):
    """Scores of next to nothing: every key that is seen has the same weight, others none."""
    c = case([new] * 2, [200, 3000], heads, dtype=dtype, cache=E4, seed=22)
    c["scale"], c["ks"] = scale, torch.full((1,), k_scale, device="cuda")
    check(c)


def least_time(c, calls=10):
    """Microseconds of a call, the least of a few turns."""
    ws = torch.empty(B.pp_latent_workspace(c["q"], c["cache"], c["table"], c["latent"], max_new=c["max_new"], max_len=c["max_len"],
                                           window=c["window"]), dtype=torch.uint8, device="cuda")
    least = math.inf
    for _ in range(6):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        for _ in range(calls):
            attend(c, workspace=ws)
        b.record()
        torch.cuda.synchronize()
        least = min(least, a.elapsed_time(b) / calls * 1e3)
    return least


@pytest.mark.parametrize("cache", [BF, E4])
@pytest.mark.parametrize("new,heads,n,requests,window", [(1, 16, 16_001, 64, 0), (1, 128, 6001, 48, 0), (200, 16, 8_203, 6, 0),
                                                         (1, 16, 16_001, 64, 9_000), (200, 16, 8_203, 6, 3_000)])
def test_what_is_not_seen_costs_no_time(new, heads, n, requests, window, cache):
    """NaN behind the last token and before a window is not looked at key by key: a call takes what it takes
    without (a walk over all keys of a share took many times as long)."""
    c = case([new] * requests, [n] * requests, heads, cache=cache, seed=23)
    c["window"] = window
    clean = least_time(c)
    want = [x.clone() for x in attend(c)]
    for r in range(requests):
        hidden = list(range(n, -(-n // 16) * 16))
        if window:
            hidden += range(n - new - window - 100, n - new - window + 1)
        put(c, r, hidden, math.nan)
    spoilt = least_time(c)
    got = attend(c)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    print(f"{clean:.1f} us, {spoilt:.1f} with NaN", flush=True)
    assert spoilt < 2 * clean + 20


def many(seed, requests, lo, hi, heads, *, latent, dtype, cache, window=0, page=16, pages=2048):
    """Single tokens of long requests, whose rows of the block table share a pool that is much smaller."""
    c = case([1] * 4, [pages * page // 4] * 4, heads, latent=latent, dtype=dtype, cache=cache, page=page, seed=seed, spare=0)
    g = torch.Generator().manual_seed(seed)
    length = torch.randint(lo, hi + 1, (requests,), generator=g)
    c["table"] = torch.randint(0, pages, (requests, -(-hi // page)), generator=g).int().cuda()
    c["length"], c["begin"] = length.int().cuda(), torch.arange(requests + 1, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(seed)
    c["q"] = torch.randn((requests, heads, latent + 64), generator=g, device="cuda", dtype=dtype)
    c["out"] = torch.full((requests, heads, latent), 7.0, dtype=dtype, device="cuda")
    c["lse"] = torch.full((requests, heads), 7.0, device="cuda")
    return dict(c, max_new=1, max_len=hi, window=window), length.tolist()


def share(length, window, tile, start, least):
    """Tiles of a block's share: all requests' tiles and starts over 256 blocks."""
    tiles = [-(-(n - (max(0, n - window) & ~63 if window else 0)) // tile) for n in length]
    return max(least, -(-sum(t + start for t in tiles) // 256))


@pytest.mark.parametrize("dtype,cache", [(BF, BF), (HF, HF), (BF, E4), (HF, E4)])
@pytest.mark.parametrize("latent", [512, 256])
@pytest.mark.parametrize("requests,lo,hi,window,page", [(140, 8000, 16_384, 0, 16), (200, 9000, 12_000, 7001, 64)])
def test_waves_of_many_tiles(requests, lo, hi, window, page, latent, dtype, cache):
    """Each wave goes through more tiles than it has page numbers of at a time (64 of 16 keys, 32 of 32), and its ring
    comes round many times."""
    c, length = many(requests, requests, lo, hi, 16, latent=latent, dtype=dtype, cache=cache, window=window, page=page)
    tile = 32 if cache == E4 else 16
    assert share(length, window, tile, 16, 8) / 4 > 1.2 * 1024 / tile
    check_requests(c, [0, 1, requests // 2, requests - 1])


@pytest.mark.parametrize("dtype,cache,latent", [(BF, BF, 512), (HF, HF, 256), (HF, E4, 512), (BF, E4, 256)])
@pytest.mark.parametrize("window", [0, 11_003])
def test_blocks_of_many_tiles(window, dtype, cache, latent):
    """The same of blocks of 128 rows whose shares begin and end inside requests: 64 tiles of 32 keys, or of 64."""
    requests = 130 if cache == E4 else 70
    c, length = many(requests, requests, 12_000, 16_384, 128, latent=latent, dtype=dtype, cache=cache, window=window)
    tile, start = (64, 8) if cache == E4 else (32, 16)
    assert share(length, window, tile, start, start // 2) > 1.2 * 64
    check_requests(c, [0, 1, requests // 2])


@pytest.mark.parametrize("wild", [False, True])
@pytest.mark.parametrize("requests,heads,overlap", [(40, 128, range(5, 35)), (40, 128, range(5, 9)), (40, 16, range(5, 9)), (1100, 20, range(50, 900))])
def test_requests_that_overlap_write_nothing_else(requests, heads, overlap, wild):
    """Starts out of order or outside: what stands around out, lse and the workspace and the rows that no request names stay as
    they are, and requests that overlap no other have their rows, or are left out whole where all requests together have more
    tiles of 128 rows than starts in order can have."""
    c = case([2] * requests, [70] * requests, heads, seed=24)
    T = 2 * requests
    begin = c["begin"].tolist()
    for r in overlap:
        begin[r] = [0, 10 ** 6, -7, 2 * r][r % 4] if wild else 2 * r + [-8, 6, -3, 0][r % 4]
    begin[0] = 1                                      # a row of nobody, but where a request begins at 0
    named = [0] * (T + 1)
    clip = lambda x: min(max(x, 0), T)  # noqa: E731
    ranges = [(clip(a), max(clip(a), clip(b))) for a, b in zip(begin, begin[1:])]
    for a, b in ranges:
        for t in range(a, b):
            named[t] += 1
    alone = [t for r, (a, b) in enumerate(ranges) if (a, b) == (2 * r, 2 * r + 2) and named[a] == named[a + 1] == 1 for t in (a, a + 1)]
    assert max(named) > 1 and (wild or len(alone) > 4 and not named[0])
    bad = dict(c, begin=torch.tensor(begin, dtype=torch.int32, device="cuda"))
    need = B.pp_latent_workspace(c["q"], c["cache"], c["table"], c["latent"], max_new=T, max_len=c["max_len"])
    guard = 1 << 20
    space = torch.full((need + 2 * guard,), 0x5a, dtype=torch.uint8, device="cuda")
    outs = torch.full((T + 64, heads, c["latent"]), 7.0, dtype=BF, device="cuda")
    lses = torch.full((T + 64, heads), 7.0, device="cuda")
    got = attend(dict(bad, out=outs[32:-32], lse=lses[32:-32]), max_new=T, workspace=space[guard:guard + need])
    torch.cuda.synchronize()
    assert bool((space[:guard] == 0x5a).all()) and bool((space[guard + need:] == 0x5a).all())
    for x in (outs, lses):
        assert bool((x[:32] == 7).all()) and bool((x[-32:] == 7).all())
    nobody = [t for t in range(T) if not named[t]]
    for x in got:
        assert bool((x[nobody] == 7).all())
    if wild:
        return
    if sum(-(-(b - a) * heads // 128) for a, b in ranges) > T * heads // 128 + requests:
        out = [t for t in alone if bool((got[0][t] == 7).all()) and bool((got[1][t] == 7).all())]
        assert len(out) < len(alone)
        alone = [t for t in alone if t not in out]
    wanted, want_lse, tol, tol_lse = R.latent(c["q"], c["cache"], c["table"], c["begin"], c["length"], c["latent"], scale=c["scale"])
    close(got[0][alone], wanted[alone], tol[alone])
    close(got[1][alone], want_lse[alone], tol_lse[alone])

"""Edges of the paged attention: what the ordinary cases do not reach."""

import math

import pytest
import torch

from paper_2608_01655_amd import binding as B
from tests import serve_ref as S
from tests.test_gpu_serve import BF, E4, HF, attend, attend_case, close

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _say_case(request):
    print(f"\n[case] {request.node.name}", flush=True)
    yield


def put(c, name, r, at, x):
    """Sets tokens `at` of request r in the pages of c[name] to x (a value or rows [tokens][heads][dim])."""
    page = c[name].shape[2]
    at = torch.as_tensor(at, device="cuda")
    c[name][c["table"][r].long()[at // page], :, at % page] = x


@pytest.mark.parametrize("gap", [14.0, 16.0, 18.0, 20.0])
@pytest.mark.parametrize("new", [1, 5, 100])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype,cache", [(HF, HF), (HF, E4), (BF, BF)])
def test_small_weights_beside_large_ones(dtype, cache, dim, new, gap):
    """Every 32nd key takes nearly all the weight and has V = 0, so that the output is what the others
    add, `gap` below in the exponent: their weights keep the type's precision.

    Tolerance: serve_ref's, but for f16 with weights held in units of 2^-10 of the largest (or smaller
    ones): a weight below the normal range is off by 2^-25 of that unit, 2^-35 |v| a key, over a sum of
    at least 1; the output's own subnormal rounding is 2^-25."""
    n, heads, kv_heads = 1100, 8, 2
    c = attend_case(3, [new], [n], heads, kv_heads, dim, dtype, cache, scale=1.0)
    c["ks"] = c["vs"] = None
    g = torch.Generator(device="cuda").manual_seed(int(gap))
    c["q"][...] = 0
    c["q"][..., 0] = 1
    sink = torch.arange(0, n, 32)
    v = (128 + 128 * torch.rand((n, kv_heads, dim), generator=g, device="cuda")).to(dtype).to(cache)
    put(c, "k", 0, range(n), torch.zeros((), device="cuda").to(cache))
    put(c, "v", 0, range(n), v)
    gap_key = torch.zeros(dim, device="cuda")
    gap_key[0] = gap
    put(c, "k", 0, sink, gap_key.to(cache))
    put(c, "v", 0, sink, torch.zeros((), device="cuda").to(cache))
    out, lse = attend(c)
    torch.cuda.synchronize()
    v = v.double().cpu()
    v[sink] = 0
    v = v.repeat_interleave(heads // kv_heads, 1)
    w = torch.full((n,), math.exp(-gap), dtype=torch.float64)
    w[sink] = 1
    u = S.UNIT[dtype]
    for i in range(new):
        e = n - new + i + 1
        total = w[:e].sum()
        o = torch.einsum("j,jhd->hd", w[:e], v[:e]) / total
        tol = 2 * u * o + ((dim + 8) * 2.0 ** -24 * gap * 2 + (e + 64) * 2.0 ** -23) * o
        if dtype == HF:
            tol += 2.0 ** -35 * v[:e].sum(0) + 2.0 ** -25
        close(out[i], o, tol)
        want = torch.full((heads,), float(gap + total.log()), dtype=torch.float64)
        close(lse[i], want, torch.full_like(want, (dim + 8) * 2.0 ** -24 * gap + (e + 64) * 2.0 ** -23 + 2.0 ** -22 * float(want[0])))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("new,n", [(1, 40), (5, 90), (100, 100), (100, 400), (100, 9000)])
def test_rows_of_minus_infinity_whatever_the_values(new, n, dim, dtype):
    """A row whose seen keys all score -infinity is empty, also where their values are infinite or NaN."""
    c = attend_case(4, [new], [n], 8, 2, dim, dtype, dtype)
    c["q"].abs_().add_(0.01)
    dead = new - new // 4                                 # new tokens that see nothing else
    last = n - new + dead                                 # the first key that scores
    k = torch.zeros(dim, device="cuda", dtype=dtype)
    k[0] = -math.inf
    put(c, "k", 0, range(last), k)
    for at, x in ((0, math.inf), (last // 2, math.nan), (max(last - 2, 0), -math.inf), (last - 1, math.inf)):
        put(c, "v", 0, [at], x)
    out, lse = attend(c)
    torch.cuda.synchronize()
    assert bool((out[:dead] == 0).all()) and bool((lse[:dead] == -math.inf).all())
    assert bool(torch.isfinite(lse[dead:]).all())


@pytest.mark.parametrize("requests,new,heads,kv_heads", [(512, 1, 8, 8), (64, 128, 64, 8), (80, 3, 16, 2)])
@pytest.mark.parametrize("wide", [False, True])
def test_no_bound_at_all(requests, new, heads, kv_heads, wide):
    """max_len as large as its type, behind block tables of a few pages and of as many as there may be:
    the same as with a bound that fits, but for the rounding where the latter takes parts."""
    c = attend_case(6, [new] * requests, [new + r % 7 for r in range(requests)], heads, kv_heads, 128, BF, BF)
    out, lse = attend(c)
    want, want_lse = out.double().cpu(), lse.double().cpu()
    if wide:                                              # rows may overlap where they are only read
        blocks, row = (1 << 27) - 1, c["table"].shape[1]
        table = torch.zeros(blocks + requests * row, dtype=torch.int32, device="cuda")
        table[:requests * row] = c["table"].flatten()
        c["table"] = table.as_strided((requests, blocks), (row, 1))
    out, lse = attend(c, max_len=2 ** 31 - 1)
    torch.cuda.synchronize()
    close(out, want, 2 ** -7 * want.abs() + 2 ** -12)
    close(lse, want_lse, 2 ** -18 * want_lse.abs() + 2 ** -18)


@pytest.mark.parametrize("dtype,cache", [(BF, BF), (HF, E4)])
def test_write_to_a_place_named_twice(dtype, cache):
    """Such a place holds elements of either row, in any mix; the others are whole."""
    T, heads, dim, page = 40, 4, 128, 16
    rows = torch.randn((2, T, heads, dim), device="cuda", dtype=dtype).clamp(-400, 400)
    pages = torch.zeros((2, 3, heads, page, dim), device="cuda", dtype=cache)
    place = torch.arange(T, device="cuda")
    place[::2] = 0
    B.pp_kv_write(rows[0], rows[1], place, pages[0], pages[1])
    got = pages.permute(0, 1, 3, 2, 4).reshape(2, -1, heads, dim)[:, :T].float()
    want = rows.to(cache).float()
    assert torch.equal(got[:, 1::2], want[:, 1::2])
    assert bool((got[:, :1] == want[:, ::2]).any(1).all())
    assert bool((got[:, 2::2] == 0).all())


def test_a_workspace_that_does_not_do():
    c = attend_case(10, [1], [30_000], 16, 2, 128, BF, BF)
    need = B.pp_attention_workspace(c["q"], c["k"], c["table"], max_new=1, max_len=30_000)
    assert need > 64
    kept = torch.zeros(need + 256, dtype=torch.uint8, device="cuda")
    for bad in (kept[:64], kept[:need - 1], kept[16:need + 16]):
        with pytest.raises(B.PPError) as e:
            attend(c, workspace=bad)
        assert e.value.code == B.PP_E_ARG
    want = [x.clone() for x in attend(c)]
    got = attend(c, workspace=kept[:need])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("R", [3, 100])
def test_tables_without_a_tree(R):
    """No chunk at all: nothing is found, whatever the requests ask for."""
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    leaf = torch.arange(R, dtype=torch.int32, device="cuda") - 1
    length = torch.arange(R, dtype=torch.int32, device="cuda") * 3
    T = int(length.sum())
    i32 = lambda *s: torch.full(s, -7, dtype=torch.int32, device="cuda")  # noqa: E731
    table, begin, start, end, position, taken = i32(R, 20), i32(R + 1), i32(R), i32(R), i32(T), i32(1)
    slot_map = torch.empty(T, dtype=torch.int64, device="cuda")
    free = torch.arange(100, 100 + 20 * R, dtype=torch.int32, device="cuda")
    B.pp_block_tables(leaf, length, torch.full_like(leaf, -1), e.view(0, 16), e, free, table, begin, start, end, slot_map,
                      position, taken, page_size=16, chunk_tokens=32, n_slots=0)
    assert bool((start == 0).all()) and torch.equal(end, length) and begin[1:].tolist() == length.cumsum(0).tolist()
    need = -(-length // 16)
    assert int(taken) == int(need.sum())
    for r in range(R):
        first = 100 + int(need[:r].sum())
        n, a, b = int(need[r]), int(begin[r]), int(begin[r + 1])
        assert table[r].tolist() == list(range(first, first + n)) + [-7] * (20 - n)
        assert slot_map[a:b].tolist() == list(range(first * 16, first * 16 + b - a))
        assert position[a:b].tolist() == list(range(b - a))


def check_requests(c, which, window=0):
    """Requests `which` of the call against the 64-bit implementation, one at a time."""
    out, lse = attend(c, window)
    torch.cuda.synchronize()
    k, v, begin = c["k"].cpu(), c["v"].cpu(), c["begin"].tolist()
    for r in which:
        rows = slice(begin[r], begin[r + 1])
        sub = torch.tensor([0, begin[r + 1] - begin[r]], dtype=torch.int32)
        want, want_lse, tol, tol_lse = S.attend(c["q"][rows], k, v, c["table"][r:r + 1], sub, c["length"][r:r + 1],
                                                scale=c["scale"], window=window, k_scale=c["ks"], v_scale=c["vs"])
        close(out[rows], want, tol)
        close(lse[rows], want_lse, tol_lse)


@pytest.mark.parametrize("window", [0, 4500])
@pytest.mark.parametrize("dim,dtype,cache", [(64, HF, E4), (64, BF, BF), (128, BF, BF), (128, BF, E4), (256, HF, HF), (256, BF, E4)])
@pytest.mark.parametrize("new,heads", [(1, 8), (4, 32), (3, 64), (8, 64)])
def test_long_requests_in_one_part(new, heads, dim, dtype, cache, window):
    """Many requests, so that the long ones among them are not cut and a wave goes through more than 32 tiles:
    its page numbers are read again, its ring comes round."""
    if dim == 256 and new == 8:
        new = 4                                           # 32 rows are its most
    length = [new + r % 9 for r in range(512)]
    long = {5: 9000, 100: 4097, 250: 4096 * 2 + 1, 511: 6111}
    for r, n in long.items():
        length[r] = n
    c = attend_case(new + dim, [new] * 512, length, heads, 8, dim, dtype, cache)
    assert B.pp_attention_workspace(c["q"], c["k"], c["table"], max_new=new, max_len=9000, window=window) == 0
    check_requests(c, [*long, 0, 8, 400], window)


@pytest.mark.parametrize("window", [0, 4500])
@pytest.mark.parametrize("dim,dtype,cache", [(64, HF, HF), (64, BF, E4), (128, BF, BF), (128, HF, E4), (256, BF, BF), (256, HF, E4)])
def test_long_prompts_in_one_part(dim, dtype, cache, window):
    """As many new tokens as leave no room for parts, so that a block goes through more than 64 tiles of keys."""
    filler = 8
    each = 2 ** 29 // (2 * 64 * dim * 4) // filler
    long = [64 * 64 - 1, 64 * 64 + 1, 64 * 130, 12_007]
    new, length = [37, 40, 9, 70] + [each] * filler, long + [each] * filler
    c = attend_case(dim, new, length, 64, 8, dim, dtype, cache)
    # two parts of the prompts' rows would take 2^29 bytes; what there is, is of single tokens, had there been any
    assert B.pp_attention_workspace(c["q"], c["k"], c["table"], max_new=each, max_len=12_007, window=window) < 2 ** 29
    check_requests(c, range(4), window)


@pytest.mark.parametrize("R", [65, 200])
@pytest.mark.parametrize("single", [False, True])
@pytest.mark.parametrize("dim,dtype,cache,top", [(128, BF, BF, 300), (64, HF, E4, 3000), (256, BF, BF, 3000)])
def test_many_prompts(R, single, dim, dtype, cache, top):
    """More requests than a wave has lanes, some of them empty, in one part and in several."""
    new = [0 if r % 11 == 3 else 1 if single and r % 3 else 5 + r * 7 % 40 for r in range(R)]
    length = [n + r * 37 % 130 for r, n in enumerate(new)]
    length[R // 2], length[-1] = top, top - 1
    c = attend_case(R, new, length, 16, 2, dim, dtype, cache)
    parts = B.pp_attention_workspace(c["q"], c["k"], c["table"], max_new=max(new), max_len=top)
    assert (parts > 0) == (top > 300)
    check_requests(c, range(R))


def test_expanded_tensors_that_are_read():
    """One row of queries, of pages and of the block table for all: the same as with copies of them."""
    c = attend_case(15, [1, 1, 1], [70, 70, 70], 8, 2, 128, BF, BF)
    c["table"][1:] = c["table"][:1]
    q = c["q"][:1, :1].expand(3, 8, 128)
    want = [x.clone() for x in attend(dict(c, q=q.contiguous()))]
    k, v = (c[x][:, :1].expand(-1, 2, -1, -1) for x in "kv")
    got = attend(dict(c, q=q, table=c["table"][:1].expand(3, -1)))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    want = [x.clone() for x in attend(dict(c, k=k.contiguous(), v=v.contiguous()))]
    got = attend(dict(c, k=k, v=v))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    pages = torch.zeros((2, 3, 2, 16, 128), dtype=BF, device="cuda")
    row = torch.randn((1, 1, 128), dtype=BF, device="cuda")
    B.pp_kv_write(row.expand(5, 2, 128), -row.expand(5, 2, 128), torch.arange(5, device="cuda"), pages[0], pages[1])
    assert torch.equal(pages[0, 0, :, :5], row.expand(2, 5, 128)) and torch.equal(pages[1, 0, :, :5], -row.expand(2, 5, 128))
    with pytest.raises(B.PPError):
        B.pp_kv_write(row.expand(1, 2, 128), row.expand(1, 2, 128), torch.arange(1, device="cuda"), pages[0, :1].expand(3, -1, -1, -1), pages[1, :1].expand(3, -1, -1, -1))
    with pytest.raises(B.PPError):
        attend(dict(c, out=c["out"][:, :1].expand(3, 8, 128)))

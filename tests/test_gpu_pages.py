"""Copies, forks and the free list of pages on the GPU against plain implementations."""

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


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


# ------------------------------------------------------------------ copies ---

def check_copy(pools, source, target, tokens, page, stream=None):
    want = [p.clone() for p in pools]
    for i, (a, b) in enumerate(zip(source, target)):
        n = page if tokens is None else min(max(int(tokens[i]), 0), page)
        if 0 <= a < pools[0].shape[0] and 0 <= b < pools[0].shape[0] and a != b:
            for p in want:
                p[b, :, :n] = p[a, :, :n]
    B.pp_page_copy(pools, dev(source), dev(target), None if tokens is None else dev(tokens), stream=stream)
    torch.cuda.synchronize()
    for p, w in zip(pools, want):
        assert torch.equal(p.view(torch.uint8) if p.dtype == E4 else p, w.view(torch.uint8) if p.dtype == E4 else w)


def pool_of(n, pages, heads, page, dim, dtype, order="heads", gap=0):
    shape = (n, pages, heads, page, dim + gap) if order == "heads" else (n, pages, page, heads, dim + gap)
    x = torch.randint(-2 ** 15, 2 ** 15, shape, dtype=torch.int16, device="cuda").remainder_(1000).to(torch.float32).to(dtype)[..., :dim]
    return list(x if order == "heads" else x.transpose(2, 3))


@pytest.mark.parametrize("order", ["heads", "tokens"])
@pytest.mark.parametrize("gap", [0, 16])
@pytest.mark.parametrize("heads,page,dim,dtype", [(1, 16, 64, E4), (2, 16, 128, BF), (8, 16, 128, HF), (3, 32, 72, BF), (1, 64, 576, BF), (1, 16, 576, E4),
                                                  (8, 1024, 16, BF), (5, 256, 256, BF)])
def test_copies(heads, page, dim, dtype, gap, order):
    rng = np.random.default_rng(heads)
    pools = pool_of(3, 19, heads, page, dim, dtype, order, gap)
    perm = rng.permutation(19)
    check_copy(pools, perm[:9], perm[9:18], None, page)
    tokens = rng.integers(-2, page + 3, 9)
    tokens[:4] = [0, 1, page, page - 1]
    check_copy(pools, perm[9:18], perm[:9], tokens, page)


def test_moves_that_do_nothing():
    pools = pool_of(2, 9, 2, 16, 64, BF)
    check_copy(pools, [-1, 0, 9, 1, 2 ** 31 - 1, 3, -2 ** 31, 4], [5, -1, 5, 9, 6, 3, 7, 8], None, 16)
    before = [p.clone() for p in pools]
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    B.pp_page_copy(pools, e, e)
    B.pp_page_copy([], dev([1]), dev([2]))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(pools, before))


@pytest.mark.parametrize("n", [127, 128, 129, 300])
def test_many_pools(n):
    """More layers than one launch takes."""
    pools = pool_of(n, 7, 1, 16, 64, BF)
    check_copy(pools, [0, 1], [5, 6], [16, 9], 16)


def test_pages_past_32_bits():
    """Pages whose offsets in bytes need more than 32 bits."""
    pages = 2 ** 31 // (16 * 512 * 2) + 40               # 4 GiB and some
    pool = torch.zeros((pages, 1, 16, 512), device="cuda", dtype=BF)
    last = pages - 1
    pool[last], pool[3] = 3.0, 4.0
    B.pp_page_copy([pool], dev([last, 3]), dev([7, last - 2]))
    torch.cuda.synchronize()
    assert bool((pool[7] == 3).all()) and bool((pool[last - 2] == 4).all()) and bool((pool[last] == 3).all())
    assert not bool(pool[8:last - 2].any()) and not bool(pool[:3].any())


# ------------------------------------------------------------------- forks ---

def check_fork(parent, length, table, free, page, rows=None, stream=None):
    rows = len(parent) if rows is None else rows
    out_table = np.full((rows, table.shape[1]), -7, np.int32)
    want = R.fork(parent, length, table, free, out_table, page)
    got = dict(out_table=dev(out_table), out_length=dev(np.full(rows, -7)), source=dev(np.full(rows, -7)), target=dev(np.full(rows, -7)),
               tokens=dev(np.full(rows, -7)), taken=dev([-7]))
    B.pp_fork_tables(dev(parent), dev(length), dev(table), dev(free), *got.values(), page_size=page, stream=stream)
    torch.cuda.synchronize()
    for k in got:
        assert np.array_equal(got[k].cpu().numpy(), want[k]), k


def fork_case(seed, rows, parents, blocks=9, page=16):
    rng = np.random.default_rng(seed)
    parent = rng.integers(0, max(parents, 1), rows)
    length = rng.integers(0, blocks * page + 1, parents)
    length[rng.random(parents) < 0.2] //= page
    table = rng.integers(0, 10 ** 6, (parents, blocks)).astype(np.int32)
    return parent, length, table, (2 * 10 ** 6 + rng.permutation(rows + 3)).astype(np.int32)


@pytest.mark.parametrize("rows,parents", [(1, 1), (2, 1), (15, 3), (16, 16), (17, 40), (64, 8), (65, 65), (1000, 7), (1000, 1000), (4097, 2000), (9000, 65536)])
def test_forks(rows, parents):
    parent, length, table, free = fork_case(rows, rows, parents)
    check_fork(parent, length, table, free, 16)


@pytest.mark.parametrize("page", [16, 64, 1024])
def test_fork_page_sizes(page):
    parent, length, table, free = fork_case(page, 40, 12, blocks=5, page=page)
    check_fork(parent, length, table, free, page)


def test_fork_long_rows():
    parent, length, table, free = fork_case(5, 20, 6, blocks=1337)
    check_fork(parent, length, table, free, 16)


def test_fork_numbers_out_of_range():
    parent, length, table, free = fork_case(6, 50, 10)
    parent[:8] = [-1, 10, 2 ** 31 - 1, -2 ** 31, 0, 0, 9, 9]
    length[:4] = [-5, 9 * 16 + 5, 2 ** 31 - 1, -2 ** 31]      # past the row: no last block, and nothing to copy
    table[5:8] = -1
    check_fork(parent, length, table, free, 16)


@pytest.mark.parametrize("n_free", [0, 1, 5])
def test_fork_short_of_pages(n_free):
    parent, length, table, free = fork_case(7, 60, 4)
    check_fork(parent, length, table, free[:n_free], 16)


def test_fork_of_nothing():
    parent, length, table, free = fork_case(8, 12, 3)
    check_fork(parent[:0], length, table, free, 16)
    check_fork(parent, length[:0], table[:0], free, 16)
    check_fork(parent, length, table[:, :0], free, 16)


def test_fork_most_rows():
    parent, length, table, free = fork_case(9, 65536, 65536, blocks=2)
    check_fork(parent, length, table, free, 16)


def test_fork_and_copy_captured():
    """A beam step as it is replayed: rows forked, pages copied; then the pages that no row names."""
    parent, length, table, free = fork_case(10, 24, 6, blocks=4)
    pages = 300
    rng = np.random.default_rng(0)
    table = rng.permutation(200)[:24].reshape(6, 4).astype(np.int32)
    free = (200 + rng.permutation(40)).astype(np.int32)
    pools = pool_of(4, pages, 2, 16, 64, BF)
    d = [dev(x) for x in (parent, length, table, free)]
    out = [dev(np.full((24, 4), -1))] + [dev(np.zeros(24)) for _ in range(4)] + [dev([0])]
    marks, left, count = torch.empty(pages, dtype=torch.uint8, device="cuda"), dev(np.full(pages, -1)), dev([0])

    def step():
        B.pp_fork_tables(*d, *out, page_size=16)
        B.pp_page_copy(pools, *out[2:5])
        B.pp_free_pages(out[0], out[1], left, count, marks, page_size=16, first=10)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        rng = np.random.default_rng(seed)
        parent, length = rng.integers(-1, 6, 24), rng.integers(0, 65, 6)
        d[0].copy_(dev(parent))
        d[1].copy_(dev(length))
        out[0].fill_(-1)
        left.fill_(-1)
        for p in pools:
            p.copy_(torch.randn(p.shape, device="cuda"))
        before = [p.clone() for p in pools]
        graph.replay()
        torch.cuda.synchronize()
        want = R.fork(parent, length, table, free, np.full((24, 4), -1, np.int32), 16)
        got = [x.cpu().numpy() for x in out]
        for k, x in zip(("out_table", "out_length", "source", "target", "tokens", "taken"), got):
            assert np.array_equal(x, want[k]), k
        for p, b in zip(pools, before):
            for s, t, n in zip(*got[2:5]):
                if s >= 0:
                    b[t, :, :n] = b[s, :, :n]
            assert torch.equal(p, b)
        free_now = R.free_pages(got[0], got[1], pages, 10, 16)
        assert int(count) == len(free_now)
        assert np.array_equal(left.cpu().numpy(), np.concatenate([free_now, np.full(pages - len(free_now), -1)]))


# -------------------------------------------------------------- free pages ---

def check_free(table, length, n_pages, first, page, room=None, stream=None):
    want = R.free_pages(table, length, n_pages, first, page)
    room = n_pages if room is None else room
    free, count = dev(np.full(room, -7)), dev([-7])
    marks = torch.full((n_pages,), 77, dtype=torch.uint8, device="cuda")
    B.pp_free_pages(dev(table), dev(length), free, count, marks, page_size=page, first=first, stream=stream)
    torch.cuda.synchronize()
    assert int(count) == len(want)
    n = min(len(want), room)
    assert np.array_equal(free.cpu().numpy(), np.concatenate([want[:n], np.full(room - n, -7)]))


def free_case(seed, requests, blocks, n_pages, page=16):
    rng = np.random.default_rng(seed)
    table = rng.integers(-3, n_pages + 3, (requests, blocks)).astype(np.int32)
    return table, rng.integers(-1, blocks * page + 20, requests)


@pytest.mark.parametrize("requests,blocks", [(0, 5), (1, 1), (3, 0), (5, 300), (64, 100), (700, 200), (3, 40_000)])
@pytest.mark.parametrize("n_pages,first", [(0, 0), (1, 0), (8, 8), (31, 3), (32, 0), (33, 1), (1000, 7), (70_001, 64), (262_147, 13)])
def test_free_pages(requests, blocks, n_pages, first):
    """Few rows, which one block takes, and many."""
    table, length = free_case(requests + n_pages, requests, blocks, n_pages)
    check_free(table, length, n_pages, first, 16)


@pytest.mark.parametrize("requests", [5, 900])
@pytest.mark.parametrize("page,room", [(16, 0), (64, 10), (1024, 999)])
def test_free_page_sizes_and_room(requests, page, room):
    table, length = free_case(page, requests, 100, 3000, page)
    check_free(table, length, 3000, 100, page, room)


@pytest.mark.parametrize("requests", [2, 1200])
def test_free_pages_of_a_large_pool(requests):
    """More pages than one block has bits for."""
    table, length = free_case(1, requests, 60, 1_100_003)
    check_free(table, length, 1_100_003, 5, 16)
    check_free(table, length, 1_100_003, 1_000_001, 16)


def test_on_another_stream():
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        pools = pool_of(2, 9, 2, 16, 64, BF)
        check_copy(pools, [1, 2], [5, 6], [16, 9], 16, stream=side)
        check_fork(*fork_case(3, 30, 9), 16, stream=side)
        check_free(*free_case(2, 30, 20, 500), 500, 3, 16, stream=side)


def test_refusals_of_the_binding():
    pools = pool_of(2, 9, 2, 16, 64, BF)
    i = dev([1, 2])
    for args in ((pools, i.long(), i), (pools, i, i[:1]), (pools, i, i, i.float()), ([pools[0], pools[1][:8]], i, i), ([pools[0], pools[1].to(HF)], i, i),
                 ([pools[0], pools[1].transpose(1, 2)], i, i), ([pools[0][0]], i, i), ([p.cpu() for p in pools], i, i), ([p.float() for p in pools], i, i)):
        with pytest.raises(ValueError):
            B.pp_page_copy(*args)
    with pytest.raises(B.PPError):
        B.pp_page_copy([pools[0][:, :, :, :4]], i, i)        # rows of 8 bytes
    with pytest.raises(B.PPError):
        B.pp_page_copy([pools[0][:1].expand(9, -1, -1, -1)], i, i)
    parent, length, table, free = (dev(x) for x in fork_case(3, 30, 9))
    out = [torch.zeros((30, 9), dtype=torch.int32, device="cuda")] + [dev(np.zeros(30)) for _ in range(4)] + [dev([0])]
    good = [parent, length, table, free, *out]
    for at, bad in ((0, parent.long()), (1, length[:8]), (2, table.long()), (3, free[None]), (4, out[0][:, :8]), (4, out[0][:29]), (5, out[1][:29]),
                    (9, out[1]), (6, out[2].float())):
        args = list(good)
        args[at] = bad
        with pytest.raises(ValueError):
            B.pp_fork_tables(*args, page_size=16)
    with pytest.raises(B.PPError):
        B.pp_fork_tables(*good, page_size=24)
    same = torch.zeros((39, 9), dtype=torch.int32, device="cuda")
    with pytest.raises(B.PPError):
        B.pp_fork_tables(parent, length, same[:9], free, same[8:38], *out[1:], page_size=16)
    marks, count = torch.zeros(100, dtype=torch.uint8, device="cuda"), dev([0])
    for args in ((table.long(), length, free, count, marks), (table, length[:3], free, count, marks), (table, length, free.long(), count, marks),
                 (table, length, free, free, marks), (table, length, free, count, marks.int())):
        with pytest.raises(ValueError):
            B.pp_free_pages(*args, page_size=16)
    for kw in (dict(page_size=8), dict(page_size=16, first=101), dict(page_size=16, first=-1)):
        with pytest.raises(B.PPError):
            B.pp_free_pages(table, length, free, count, marks, **kw)


@pytest.mark.parametrize("rows,parents", [(40, 40), (70, 40), (40, 70), (1, 1)])
def test_fork_tables_side_by_side(rows, parents):
    """Both tables in one tensor, a row of one beside the other's: no entry is in both."""
    parent, length, table, free = fork_case(rows, rows, parents)
    want = R.fork(parent, length, table, free, np.full((rows, 9), -5, np.int32), 16)
    most = max(rows, parents)
    for shape, pick in (((most, 2, 9), lambda x, i: x[:, i]), ((most, 23), lambda x, i: x[:, 14 * i:14 * i + 9])):
        for i in range(2):
            both = torch.full(shape, -5, dtype=torch.int32, device="cuda")
            t, out = pick(both, i)[:parents], pick(both, 1 - i)[:rows]
            t.copy_(dev(table))
            got = dict(out_table=out, **{k: dev(np.full(rows, -7)) for k in ("out_length", "source", "target", "tokens")}, taken=dev([-7]))
            B.pp_fork_tables(dev(parent), dev(length), t, dev(free), *got.values(), page_size=16)
            torch.cuda.synchronize()
            assert all(np.array_equal(got[k].cpu().numpy(), want[k]) for k in got)
            assert np.array_equal(t.cpu().numpy(), table)

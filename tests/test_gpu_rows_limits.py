"""The operators around the pages at sizes past what one launch takes (2^32 threads)."""

import pytest
import torch

from paper_2608_01655_amd import binding as B

pytestmark = pytest.mark.gpu
BF, E4 = torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(autouse=True)
def _say_case(request):
    print(f"\n[case] {request.node.name}", flush=True)
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("paged", [False, True])
def test_more_tokens_than_a_launch_takes(paged):
    """2^26 tokens and a few: the bits of a call a piece of them."""
    T, D = 2 ** 26 + 5, 16
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=BF)  # noqa: E731
    q, k, v = rand(T, 1, D), rand(T, 1, D), rand(T, 1, D)
    weight, turns = 1 + rand(D) / 8, torch.from_numpy(B.pp_rotary_turns(D)).cuda()
    position = torch.randint(0, 10 ** 6, (T,), generator=g, device="cuda", dtype=torch.int32)
    pages = -(-T // 16)
    place = pages * 16 - 1 - torch.arange(T, device="cuda")

    def call(pieces):
        out = torch.zeros_like(q)
        to = torch.zeros((2, pages, 1, 16, D), device="cuda", dtype=BF) if paged else torch.zeros_like(k)
        for i in range(pieces):
            s = slice(i * T // pieces, (i + 1) * T // pieces)
            kw = dict(v=v[s], slot_map=place[s], k_cache=to[0], v_cache=to[1]) if paged else dict(k_out=to[s])
            B.pp_rotary_write(position[s], turns, q=q[s], q_out=out[s], k=k[s], q_weight=weight, k_weight=weight, **kw)
        torch.cuda.synchronize()
        return out, to

    for a, b in zip(call(1), call(3)):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))
        assert bool((a[-1] != 0).any())


@pytest.mark.parametrize("pools,moves", [(129, 131_073), (1, 2 ** 24 + 3)])
def test_more_moves_than_a_launch_takes(pools, moves):
    """Past 2^24 pages in all pools, and in one."""
    n_pages = 2 * moves + 1
    g = torch.Generator(device="cuda").manual_seed(2)
    pool = torch.randint(0, 120, (pools, n_pages, 1, 16, 16), generator=g, device="cuda", dtype=torch.uint8)
    source = 2 * torch.arange(moves, device="cuda", dtype=torch.int32)
    want = pool.clone()
    want[:, 1:2 * moves:2] = pool[:, 0:2 * moves:2]
    B.pp_page_copy(list(pool.view(E4)), source, source + 1)
    torch.cuda.synchronize()
    assert torch.equal(pool, want)


@pytest.mark.parametrize("max_new,heads", [(1, 272), (100, 272)])
def test_attention_of_more_blocks_than_a_launch_takes(max_new, heads):
    """65,536 requests of 272 key heads are refused, not done in part."""
    R, D = 65_536, 64
    q = torch.zeros((R, heads, D), device="cuda", dtype=BF)
    out = torch.full_like(q, 7)
    pages = torch.zeros((1, heads, 16, D), device="cuda", dtype=BF)
    table, length = (torch.zeros(s, device="cuda", dtype=torch.int32) for s in ((R, 1), (R,)))
    with pytest.raises(B.PPError) as e:
        B.pp_paged_attention(q, pages, pages, table, torch.arange(R + 1, device="cuda", dtype=torch.int32), length + 1, out,
                             scale=0.1, max_new=max_new, max_len=16)
    assert e.value.code == B.PP_E_DEVICE
    torch.cuda.synchronize()
    assert bool((out == 7).all())

"""The operators around the pages: what their host side refuses and lays out (no GPU needed).
Refused calls never touch the pointers they are given."""

import ctypes

import numpy as np
import pytest

from paper_2608_01655_amd import binding as B
from tests import rows_ref as R
from tests.test_serve_host import AT, L, _attention  # noqa: F401


def code(name):
    return getattr(B, "PP_E_" + name)


# ------------------------------------------------------------------- turns ---

@pytest.mark.parametrize("dim", [0, 2, 16, 64, 128, 1024])
@pytest.mark.parametrize("base", [100.0, 10_000.0, 5e5])
def test_turns(L, dim, base):
    """Turns are the frequencies over 2 pi in units of 2^-64, to the precision of a double."""
    want = np.array([base ** (-2.0 * i / dim) for i in range(dim // 2)])
    got = B.pp_rotary_turns(dim, base).view(np.uint64).astype(np.float64) / 2.0 ** 64 * 2 * np.pi
    assert np.all(np.abs(got - want) <= 2.0 ** -50 * want + 2.0 ** -62)


@pytest.mark.parametrize("kw", [dict(factor=8.0, original=4096), dict(factor=3.0), dict(factor=40.0, original=4096, slow=1.0, fast=4.0),
                                dict(factor=2.0, original=10, slow=0.0, fast=1e-3)])
def test_scaled_turns(L, kw):
    want = R.frequencies(128, 10_000.0, **kw)
    got = B.pp_rotary_turns(128, 10_000.0, **kw).view(np.uint64).astype(np.float64) / 2.0 ** 64 * 2 * np.pi
    assert np.all(np.abs(got - want) <= 2.0 ** -48 * want + 2.0 ** -62)


def test_turns_of_any_frequency(L):
    """Whole turns fall out, negative frequencies turn back."""
    got = B.pp_turns([0.0, 2 * np.pi, -np.pi / 2, 1e-30, np.pi, -1e-30, 7.0]).view(np.uint64)
    unit = 2.0 ** 64
    want = [0, 0, 0.75 * unit, 1e-30 / (2 * np.pi) * unit, 0.5 * unit, 0, (7 / (2 * np.pi) - 1) * unit]
    for g, w in zip(got, want):
        off = abs(float(g) - w)
        assert min(off, unit - off) <= 2.0 ** 64 * 2.0 ** -50


def test_turns_refusals(L):
    ok = dict(dim=64, base=1e4, factor=2.0, original=4096.0, slow=1.0, fast=32.0)
    for kw, name in ((dict(dim=-2), "ARG"), (dict(dim=3), "ARG"), (dict(base=1.0), "RANGE"), (dict(base=float("nan")), "RANGE"),
                     (dict(base=float("inf")), "RANGE"), (dict(factor=0.5), "RANGE"), (dict(factor=float("inf")), "RANGE"),
                     (dict(original=-1.0), "RANGE"), (dict(slow=-1.0), "RANGE"), (dict(slow=32.0), "RANGE"), (dict(fast=float("nan")), "RANGE")):
        a = {**ok, **kw}
        assert L.pp_rotary_turns(*a.values(), None, None) == code(name) and B.pp_last_error()
    for bad in (float("nan"), float("inf")):
        with pytest.raises(B.PPError) as e:
            B.pp_turns([1.0, bad])
        assert e.value.code == B.PP_E_RANGE
    assert L.pp_turns(-1, None, None) == B.PP_E_ARG and L.pp_turns(2, None, None) == B.PP_E_ARG and L.pp_turns(0, None, None) == B.PP_OK


# ------------------------------------------------------------------ rotary ---

def _rotary(**kw):
    a = B.pp_rotary_args(tokens=3, dtype=B.PP_BF16, q_heads=4, q_dim=128, q_first=0, q_norm=128, k_heads=2, k_dim=128, k_first=0, k_norm=64,
                         rot_dim=64, interleaved=0, eps=1e-6, amplitude=1.0, q_token_stride=512, q_head_stride=128, q_out_token_stride=512,
                         q_out_head_stride=128, k_token_stride=256, k_head_stride=128, k_out_token_stride=256, k_out_head_stride=128,
                         v_token_stride=256, v_head_stride=128, q=AT, k=AT, v=AT, q_out=2 * AT, k_out=None, q_weight=AT, k_weight=AT,
                         position=AT, turns=AT, slot_map=AT)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _pages(**kw):
    p = B.pp_kv_pages(AT, AT, None, None, B.PP_BF16, 4, 16, 2, 128, 4096, 2048, 128)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("kw,name", [
    (dict(tokens=-1), "ARG"), (dict(q_heads=-1), "ARG"), (dict(k_heads=-1), "ARG"), (dict(dtype=B.PP_E4M3), "ARG"), (dict(dtype=B.PP_F16), "ARG"),
    (dict(rot_dim=8), "UNSUPPORTED"), (dict(rot_dim=-16), "UNSUPPORTED"), (dict(rot_dim=2048), "UNSUPPORTED"), (dict(rot_dim=144), "UNSUPPORTED"),
    (dict(q_dim=0), "UNSUPPORTED"), (dict(q_dim=132), "UNSUPPORTED"), (dict(q_dim=1032), "UNSUPPORTED"), (dict(q_first=4), "UNSUPPORTED"),
    (dict(q_first=-8), "UNSUPPORTED"), (dict(q_first=72), "UNSUPPORTED"), (dict(k_first=72), "UNSUPPORTED"), (dict(q_norm=4), "UNSUPPORTED"),
    (dict(q_norm=136), "UNSUPPORTED"), (dict(k_norm=-8), "UNSUPPORTED"), (dict(eps=-1e-9), "ARG"), (dict(eps=float("nan")), "ARG"),
    (dict(eps=float("inf")), "ARG"), (dict(amplitude=float("inf")), "ARG"), (dict(amplitude=float("nan")), "ARG"), (dict(k_heads=0), "ARG"),
    (dict(k_heads=3), "ARG"), (dict(k_dim=64, k_norm=0), "ARG"), (dict(v=None), "ARG"), (dict(q=AT + 8), "ARG"), (dict(q_out=AT + 2), "ARG"),
    (dict(k=AT + 8), "ARG"), (dict(v=AT + 8), "ARG"), (dict(q_weight=AT + 8), "ARG"), (dict(turns=AT + 8), "ARG"), (dict(q_token_stride=516), "ARG"),
    (dict(k_head_stride=-128), "ARG"), (dict(v_token_stride=1), "ARG"), (dict(q_out_head_stride=64), "ARG"), (dict(q_out_token_stride=0), "ARG"),
    (dict(q_out_token_stride=128), "ARG"), (dict(q_out=AT, q_out_token_stride=1024), "ARG"), (dict(tokens=2 ** 30), "UNSUPPORTED"),
    *[(dict([(f, None)]), "ARG") for f in ("q", "k", "q_out", "q_weight", "k_weight", "position", "turns", "slot_map")]])
def test_rotary_refusals(L, kw, name):
    assert L.pp_rotary_write(ctypes.byref(_rotary(**kw)), ctypes.byref(_pages()), None) == code(name)
    assert B.pp_last_error()


@pytest.mark.parametrize("kw,name", [
    (dict(k=None), "ARG"), (dict(v=None), "ARG"), (dict(dtype=B.PP_F16), "ARG"), (dict(k_scale=AT), "ARG"), (dict(n_pages=0), "ARG"),
    (dict(page_size=24), "UNSUPPORTED"), (dict(k=AT + 8), "ARG"), (dict(v=AT + 8), "ARG"), (dict(token_stride=132), "ARG"), (dict(page_stride=-4096), "ARG"),
    (dict(token_stride=64), "ARG"), (dict(head_stride=128), "ARG"), (dict(page_stride=2048), "ARG"), (dict(token_stride=2 ** 27), "UNSUPPORTED")])
def test_rotary_refuses_pages(L, kw, name):
    assert L.pp_rotary_write(ctypes.byref(_rotary()), ctypes.byref(_pages(**kw)), None) == code(name)


def test_rotary_without_pages(L):
    call = lambda **kw: L.pp_rotary_write(ctypes.byref(_rotary(**{**dict(v=None, k_out=2 * AT), **kw})), None, None)  # noqa: E731
    assert call(v=AT) == B.PP_E_ARG                       # values go to pages only
    assert call(k_out=None) == B.PP_E_ARG
    assert call(k_out_head_stride=120) == B.PP_E_ARG
    assert call(tokens=0) == B.PP_OK
    assert call(q_heads=0, k_heads=0) == B.PP_OK
    assert L.pp_rotary_write(None, None, None) == B.PP_E_ARG
    latent = dict(k_heads=1, k_dim=576, k_first=512, k_norm=512, k_token_stride=576, k_head_stride=576, v=None)
    pages = dict(v=None, heads=1, dim=576, page_stride=16 * 576, head_stride=0, token_stride=576)
    assert L.pp_rotary_write(ctypes.byref(_rotary(tokens=0, **latent)), ctypes.byref(_pages(**pages)), None) == B.PP_OK
    assert L.pp_rotary_write(ctypes.byref(_rotary(**latent)), ctypes.byref(_pages(**{**pages, "v_scale": AT, "dtype": B.PP_E4M3})), None) == B.PP_E_ARG


# ------------------------------------------------------------------ latent ---

def _latent_pages(**kw):
    return _pages(**{**dict(v=None, heads=1, dim=576, page_stride=16 * 576, head_stride=16 * 576, token_stride=576), **kw})


def _call(**kw):
    return _attention(**{**dict(q_heads=16, q_token_stride=16 * 576, q_head_stride=576, out_token_stride=16 * 512, out_head_stride=512), **kw})


@pytest.mark.parametrize("kw,value,name", [
    (dict(k=None), 512, "ARG"), (dict(v=AT), 512, "ARG"), (dict(v_scale=AT, dtype=B.PP_E4M3), 512, "ARG"), (dict(k_scale=AT), 512, "ARG"),
    (dict(heads=2), 512, "UNSUPPORTED"), (dict(), 448, "UNSUPPORTED"), (dict(), 256, "UNSUPPORTED"), (dict(dim=512), 448, "UNSUPPORTED"),
    (dict(dim=640), 576, "UNSUPPORTED"), (dict(dtype=B.PP_F16), 512, "ARG"), (dict(page_size=8), 512, "UNSUPPORTED"), (dict(k=AT + 8), 512, "ARG"),
    (dict(token_stride=580), 512, "ARG"), (dict(token_stride=2 ** 27), 512, "UNSUPPORTED"), (dict(dtype=B.PP_E4M3, token_stride=584), 512, "ARG")])
def test_latent_refuses_pages(L, kw, value, name):
    p, a = _latent_pages(**kw), _call()
    for rc in (L.pp_latent_workspace(ctypes.byref(p), value, ctypes.byref(a)), L.pp_latent_attention(ctypes.byref(p), value, ctypes.byref(a), None)):
        assert rc == code(name) and B.pp_last_error()


@pytest.mark.parametrize("kw,name", [
    (dict(requests=-1), "ARG"), (dict(requests=65537), "ARG"), (dict(tokens=-1), "ARG"), (dict(max_new=-1), "ARG"), (dict(max_len=-1), "ARG"),
    (dict(max_blocks=-1), "ARG"), (dict(window=-1), "ARG"), (dict(q_heads=0), "ARG"), (dict(dtype=B.PP_F16), "ARG"), (dict(scale=float("nan")), "ARG"),
    (dict(tokens=2 ** 28), "UNSUPPORTED"), (dict(max_blocks=2 ** 28), "UNSUPPORTED"), (dict(q=None), "ARG"), (dict(out=None), "ARG"),
    (dict(query_start=None), "ARG"), (dict(length=None), "ARG"), (dict(block_table=None), "ARG"), (dict(q=AT + 8), "ARG"), (dict(out=AT + 2), "ARG"),
    (dict(q_token_stride=4), "ARG"), (dict(out_head_stride=504), "ARG"), (dict(out_token_stride=512), "ARG"), (dict(out_token_stride=-8192), "ARG")])
def test_latent_refusals(L, kw, name):
    assert L.pp_latent_attention(ctypes.byref(_latent_pages()), 512, ctypes.byref(_call(**kw)), None) == code(name)
    assert B.pp_last_error()


def test_latent_attention_of_nothing(L):
    for kw in (dict(requests=0), dict(tokens=0), dict(max_new=0)):
        assert L.pp_latent_workspace(ctypes.byref(_latent_pages()), 512, ctypes.byref(_call(**kw))) == 0
        assert L.pp_latent_attention(ctypes.byref(_latent_pages()), 512, ctypes.byref(_call(**kw)), None) == B.PP_OK


@pytest.mark.parametrize("requests,tokens,q_heads,max_new,max_len", [
    (8, 8192, 16, 2048, 131_072), (33, 16_384, 128, 4096, 1_000_000), (1, 1, 16, 1, 2 ** 30), (256, 256, 128, 1, 100_000)])
def test_latent_workspace_stays_small(L, requests, tokens, q_heads, max_new, max_len):
    a = _call(requests=requests, tokens=tokens, q_heads=q_heads, max_new=max_new, max_len=max_len, max_blocks=10_000)
    need = L.pp_latent_workspace(ctypes.byref(_latent_pages()), 512, ctypes.byref(a))
    assert 0 <= need < 2 ** 29 + 2 * 4 * 512 * tokens * q_heads


@pytest.mark.parametrize("blocks", [1, 4, 300, 8192])
@pytest.mark.parametrize("requests,tokens,max_new,heads", [(1, 1, 1, 16), (512, 512, 1, 128), (64, 256, 4, 16), (1, 512, 512, 16)])
def test_latent_keys_end_with_the_block_table(L, requests, tokens, max_new, heads, blocks):
    kw = dict(requests=requests, tokens=tokens, max_new=max_new, q_heads=heads, max_blocks=blocks)
    size = lambda n: L.pp_latent_workspace(ctypes.byref(_latent_pages()), 512, ctypes.byref(_call(max_len=n, **kw)))  # noqa: E731
    want = size(blocks * 16)
    for n in (blocks * 16 + 1, 1 << 20, (1 << 31) - 1):
        if n > blocks * 16:
            assert size(n) == want >= 0


# ------------------------------------------------------- copies, forks, free ---

def _copy(**kw):
    pools = (ctypes.c_void_p * 2)(*kw.pop("at", (AT, 2 * AT)))
    a = B.pp_copy_args(moves=3, n_pools=2, dtype=B.PP_BF16, n_pages=9, page_size=16, heads=2, dim=64, page_stride=2048, head_stride=1024,
                       token_stride=64, pools=ctypes.cast(pools, ctypes.c_void_p), source=AT, target=AT, tokens=None)
    for k, v in kw.items():
        setattr(a, k, v)
    a.keep = pools
    return a


@pytest.mark.parametrize("kw,name", [
    (dict(moves=-1), "ARG"), (dict(n_pools=-1), "ARG"), (dict(dtype=0), "ARG"), (dict(dtype=4), "ARG"), (dict(n_pages=0), "ARG"), (dict(heads=0), "ARG"),
    (dict(dim=0), "ARG"), (dict(dim=60), "UNSUPPORTED"), (dict(dim=72, dtype=B.PP_E4M3), "UNSUPPORTED"), (dict(page_size=48), "UNSUPPORTED"),
    (dict(heads=2 ** 21, page_size=1024), "UNSUPPORTED"), (dict(pools=None), "ARG"), (dict(source=None), "ARG"), (dict(target=None), "ARG"),
    (dict(at=(AT, None)), "ARG"), (dict(at=(AT + 8, AT)), "ARG"), (dict(page_stride=-2048), "ARG"), (dict(token_stride=68), "ARG"),
    (dict(token_stride=32), "ARG"), (dict(head_stride=64), "ARG"), (dict(page_stride=1024), "ARG"), (dict(page_stride=0), "ARG")])
def test_copy_refusals(L, kw, name):
    assert L.pp_page_copy(ctypes.byref(_copy(**kw)), None) == code(name) and B.pp_last_error()


def test_copy_of_nothing(L):
    assert L.pp_page_copy(ctypes.byref(_copy(moves=0, source=None)), None) == B.PP_OK
    assert L.pp_page_copy(ctypes.byref(_copy(n_pools=0, pools=None)), None) == B.PP_OK
    assert L.pp_page_copy(None, None) == B.PP_E_ARG


def _fork(**kw):
    a = B.pp_fork_args(rows=6, parents=3, n_free=5, max_blocks=8, page_size=16, row_stride=8, out_row_stride=8, parent=AT, length=AT, block_table=AT,
                       free_pages=AT, out_table=2 * AT, out_length=AT, source=AT, target=AT, tokens=AT, taken=AT)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw,name", [
    (dict(rows=-1), "ARG"), (dict(rows=65537), "ARG"), (dict(parents=-1), "ARG"), (dict(parents=65537), "ARG"), (dict(n_free=-1), "ARG"),
    (dict(max_blocks=-1), "ARG"), (dict(row_stride=-1), "ARG"), (dict(out_row_stride=-1), "ARG"), (dict(out_row_stride=7), "ARG"),
    (dict(page_size=17), "UNSUPPORTED"), (dict(max_blocks=2 ** 28, out_row_stride=2 ** 28), "UNSUPPORTED"), (dict(out_table=AT), "ARG"),
    (dict(out_table=AT + 4 * 20), "ARG"), (dict(out_table=AT - 4 * 8), "ARG"),
    *[(dict([(f, None)]), "ARG") for f in ("parent", "length", "block_table", "free_pages", "out_table", "out_length", "source", "target", "tokens", "taken")]])
def test_fork_refusals(L, kw, name):
    assert L.pp_fork_tables(ctypes.byref(_fork(**kw)), None) == code(name) and B.pp_last_error()


def _free(**kw):
    a = B.pp_free_args(requests=3, max_blocks=8, page_size=16, n_pages=100, first=10, room=50, row_stride=8, length=AT, block_table=AT, free_pages=AT,
                       count=AT, marks=AT)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw,name", [
    (dict(requests=-1), "ARG"), (dict(requests=65537), "ARG"), (dict(max_blocks=-1), "ARG"), (dict(n_pages=-1), "ARG"), (dict(first=-1), "ARG"),
    (dict(first=101), "ARG"), (dict(room=-1), "ARG"), (dict(row_stride=-1), "ARG"), (dict(n_pages=2 ** 24 + 1), "UNSUPPORTED"),
    (dict(page_size=0), "UNSUPPORTED"), (dict(max_blocks=2 ** 28), "UNSUPPORTED"), (dict(marks=AT + 4), "ARG"),
    *[(dict([(f, None)]), "ARG") for f in ("length", "block_table", "free_pages", "count", "marks")]])
def test_free_refusals(L, kw, name):
    assert L.pp_free_pages(ctypes.byref(_free(**kw)), None) == code(name) and B.pp_last_error()


def test_null_arguments(L):
    assert L.pp_fork_tables(None, None) == L.pp_free_pages(None, None) == B.PP_E_ARG
    assert L.pp_latent_attention(ctypes.byref(_latent_pages()), 512, None, None) == B.PP_E_ARG


def test_layouts_agree():
    """The binding packs arguments by itself: as long as the structures of the C interface."""
    for packed, args in ((B._ROTARY_ARGS, B.pp_rotary_args), (B._COPY_ARGS, B.pp_copy_args), (B._FORK_ARGS, B.pp_fork_args), (B._FREE_ARGS, B.pp_free_args)):
        assert packed.size == ctypes.sizeof(args)


@pytest.mark.parametrize("row,out_row,at", [(16, 16, 7), (16, 16, -7), (16, 16, 9), (16, 24, 8), (24, 16, 8), (0, 16, 7), (16, 16, 16 + 9), (0, 8, -8), (20, 8, -8)])
def test_fork_refuses_tables_that_meet(L, row, out_row, at):
    """Rows of 8 entries of one table that lie among the other's and have entries in common with them."""
    a = _fork(row_stride=row, out_row_stride=out_row, out_table=AT + 4 * at)
    assert L.pp_fork_tables(ctypes.byref(a), None) == B.PP_E_ARG and B.pp_last_error()


# Bytes of the two regions of pp_latent_attention's workspace: 512 parts of 16 or of 128 rows with a log sum each,
# and 256 cuts of 20 bytes.
def _regions(value_dim):
    return tuple(512 * n * (value_dim + 1) * 4 + 5120 for n in (16, 128))


@pytest.mark.parametrize("value_dim", [256, 512])
@pytest.mark.parametrize("requests,tokens,q_heads,max_new,few,tiles", [
    (1, 1, 16, 1, True, False), (65_536, 65_536, 16, 1, True, False), (8, 16, 8, 2, True, False),       # 16 rows at most
    (1, 1, 17, 1, False, True), (1, 2, 16, 2, False, True), (33, 16_384, 7, 4096, True, True),
    (4, 4096, 16, 1024, False, True), (6, 4096, 16, 1024, True, True),                                   # apart unless all have max_new tokens
    (512, 512, 128, 1, False, True), (513, 513, 128, 1, False, False), (8, 8128, 16, 2048, True, True),  # up to 1,024 slots of 128 rows,
    (8, 8136, 16, 2048, True, False), (4, 8192, 16, 2048, False, False), (1, 131_073, 128, 131_073, False, False)])  # a request one more
def test_latent_workspace_sizes(L, requests, tokens, q_heads, max_new, few, tiles, value_dim):
    dim = value_dim + 64
    pages = _latent_pages(dim=dim, page_stride=16 * dim, head_stride=16 * dim, token_stride=dim)
    a = _call(requests=requests, tokens=tokens, q_heads=q_heads, max_new=max_new, max_len=100_000, max_blocks=100_000)
    row, slot = _regions(value_dim)
    assert L.pp_latent_workspace(ctypes.byref(pages), value_dim, ctypes.byref(a)) == few * row + tiles * slot


@pytest.mark.parametrize("blocks,apart", [(1, False), (132, False), (133, True), (10_000, True)])
def test_latent_keys_of_single_tokens_end_with_the_block_table(L, blocks, apart):
    """64 requests of 600 tokens, up to 512 each: two at least have more than one (536 beside one each), so 62 may be single
    tokens, which go apart where they may have more than 131,072 keys (2,114 each).  Keys end with the block
    table whatever the bound on the lengths."""
    row, slot = _regions(512)
    kw = dict(requests=64, tokens=600, max_new=512, q_heads=16, max_blocks=blocks)
    for n in (blocks * 16, blocks * 16 + 1, 1 << 20, (1 << 31) - 1):
        a = _call(max_len=n, **kw)
        assert L.pp_latent_workspace(ctypes.byref(_latent_pages()), 512, ctypes.byref(a)) == apart * row + slot

"""The prefix cache's host layouts, and what its device entries refuse before any device work
(no GPU needed: every call here ends at its checks)."""

import ctypes
import os

import numpy as np
import pytest

from paper_2608_01655_amd import binding as B
from paper_2608_01655_amd import workloads as W


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(B.LIB_PATH):
        from paper_2608_01655_amd import build

        build.build()
    return B.lib()


def _forest(n, rng, deep):
    """A random forest with shuffled ids; deep: mostly chains."""
    parent = np.full(n, -1, np.int32)
    for v in range(1, n):
        if rng.random() < 0.02:
            continue
        parent[v] = v - 1 if rng.random() < deep else rng.integers(0, v)
    perm = rng.permutation(n).astype(np.int32)
    out = np.full(n, -1, np.int32)
    for v in range(n):
        out[perm[v]] = -1 if parent[v] < 0 else perm[parent[v]]
    return out


@pytest.mark.parametrize("n,deep", [(1, 0.0), (2, 1.0), (15, 1.0), (16, 1.0), (300, 0.2), (700, 0.97)])
def test_prefix_table_lines(L, n, deep):
    parent = _forest(n, np.random.default_rng(n), deep)
    table = B.pp_prefix_table(parent)
    for v in range(n):
        path, u = [], v
        while u >= 0:
            path.append(u)
            u = parent[u]
        want = (path + [-1] * 15)[:15] + [len(path) - 1]
        assert table[v].tolist() == want


def test_prefix_table_refuses_what_is_no_tree(L):
    for bad in ([0], [1, 0], [-1, 5], [-2], [1, 2, 0, -1]):
        with pytest.raises(B.PPError) as e:
            B.pp_prefix_table(np.array(bad, np.int32))
        assert e.value.code == B.PP_E_TREE and B.pp_last_error()
    assert L.pp_prefix_table(0, None, None) == B.PP_E_ARG


@pytest.mark.parametrize("seed", range(5))
def test_cache_slots_keep_what_stays(L, seed):
    rng = np.random.default_rng(seed)
    n, n_slots = 400, 120
    first = (rng.random(n) < 0.25).astype(np.uint8)
    slot, fresh = B.pp_cache_slots(first, n_slots)
    assert fresh == first.sum()
    assert slot[first == 1].tolist() == list(range(int(first.sum())))
    second = np.where(rng.random(n) < 0.3, (rng.random(n) < 0.25), first).astype(np.uint8)
    if second.sum() > n_slots:
        second[np.flatnonzero(second)[n_slots:]] = 0
    again, fresh = B.pp_cache_slots(second, n_slots, held=slot)
    stays = (first & second) == 1
    assert np.array_equal(again[stays], slot[stays])
    assert np.all(again[second == 0] == -1)
    new = np.flatnonzero((second == 1) & ~stays)
    assert fresh == new.size
    free = sorted(set(range(n_slots)) - set(slot[stays].tolist()))
    assert again[new].tolist() == free[:new.size]


def test_cache_slots_refusals(L):
    t = np.ones(4, np.uint8)
    for kw in (dict(n_slots=3), dict(n_slots=4, held=[0, 0, -1, -1]), dict(n_slots=4, held=[4, -1, -1, -1])):
        with pytest.raises(B.PPError) as e:
            B.pp_cache_slots(t, **kw)
        assert e.value.code == B.PP_E_RANGE


# ------------------------------------------------- refusals of device calls ---

AT = 1 << 20   # an aligned address; no refused call reads it


def _block_args(**kw):
    a = B.pp_block_args(requests=2, n=4, n_slots=2, n_free=8, max_blocks=8, max_tokens=32,
                        page_size=16, chunk_tokens=32, max_new=0, row_stride=8)
    for f in ("leaf", "length", "cached", "prefix_table", "slot", "free_pages", "block_table",
              "query_start", "start", "end", "slot_map", "position", "taken"):
        setattr(a, f, AT)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw,code", [
    (dict(requests=-1), "ARG"), (dict(requests=65537), "ARG"), (dict(n=-1), "ARG"),
    (dict(n_slots=-1), "ARG"), (dict(n_free=-1), "ARG"), (dict(max_blocks=-1), "ARG"),
    (dict(max_tokens=-1), "ARG"), (dict(max_new=-1), "ARG"), (dict(row_stride=-1), "ARG"),
    (dict(page_size=8), "UNSUPPORTED"), (dict(page_size=48), "UNSUPPORTED"),
    (dict(page_size=2048, chunk_tokens=2048), "UNSUPPORTED"), (dict(chunk_tokens=40), "ARG"),
    (dict(chunk_tokens=0), "ARG"), (dict(n_slots=2 ** 31 - 1), "UNSUPPORTED"),
    (dict(max_blocks=2 ** 31 - 1), "UNSUPPORTED"), (dict(prefix_table=AT + 4), "ARG"),
    *[(dict([(f, None)]), "ARG") for f in ("leaf", "length", "cached", "prefix_table", "slot",
                                           "free_pages", "block_table", "query_start", "start",
                                           "end", "slot_map", "position", "taken")]])
def test_block_tables_refusals(L, kw, code):
    assert L.pp_block_tables(ctypes.byref(_block_args(**kw)), None) == getattr(B, "PP_E_" + code)
    assert B.pp_last_error()


def _kv_pages(**kw):
    p = B.pp_kv_pages(AT, AT, None, None, B.PP_BF16, 4, 16, 2, 128, 4096, 2048, 128)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


BAD_PAGES = [
    (dict(k=None), "ARG"), (dict(v=None), "ARG"), (dict(dtype=B.PP_F16), "ARG"), (dict(dtype=0), "ARG"),
    (dict(k_scale=AT), "ARG"), (dict(v_scale=AT), "ARG"), (dict(n_pages=0), "ARG"), (dict(heads=0), "ARG"),
    (dict(page_size=8), "UNSUPPORTED"), (dict(page_size=24), "UNSUPPORTED"),
    (dict(page_size=2048), "UNSUPPORTED"), (dict(dim=96), "UNSUPPORTED"), (dict(dim=0), "UNSUPPORTED"),
    (dict(k=AT + 8), "ARG"), (dict(v=AT + 2), "ARG"), (dict(token_stride=132), "ARG"),
    (dict(head_stride=-2048), "ARG"), (dict(page_stride=4097), "ARG"),
    (dict(token_stride=2 ** 27), "UNSUPPORTED"), (dict(dtype=B.PP_E4M3, token_stride=136), "ARG")]


@pytest.mark.parametrize("kw,code", BAD_PAGES)
def test_kv_write_refuses_pages(L, kw, code):
    rc = L.pp_kv_write(ctypes.byref(_kv_pages(**kw)), 3, B.PP_BF16, AT, 256, 128, AT, 256, 128, AT, None)
    assert rc == getattr(B, "PP_E_" + code) and B.pp_last_error()


def test_kv_write_refusals(L):
    p = ctypes.byref(_kv_pages())
    ok = [3, B.PP_BF16, AT, 256, 128, AT, 256, 128, AT, None]
    for i, bad in ((0, -1), (1, B.PP_E4M3), (1, B.PP_F16), (2, None), (2, AT + 4), (3, 252), (4, -128),
                   (5, None), (5, AT + 8), (6, 1), (7, 4), (8, None)):
        args = list(ok)
        args[i] = bad
        assert L.pp_kv_write(p, *args) == B.PP_E_ARG, (i, bad)
        assert B.pp_last_error()
    assert L.pp_kv_write(None, *ok) == B.PP_E_ARG
    assert L.pp_kv_write(p, 0, B.PP_BF16, None, 0, 0, None, 0, 0, None, None) == B.PP_OK   # nothing to write


def _attention(**kw):
    a = B.pp_attention_args(requests=2, tokens=3, q_heads=4, dtype=B.PP_BF16, max_new=2, max_len=64,
                            max_blocks=4, window=0, scale=0.1, q_token_stride=512, q_head_stride=128,
                            out_token_stride=512, out_head_stride=128, row_stride=4, q=AT, out=AT, lse=AT,
                            query_start=AT, length=AT, block_table=AT, workspace=None, workspace_bytes=0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw,code", BAD_PAGES)
def test_attention_refuses_pages(L, kw, code):
    p, a = _kv_pages(**kw), _attention()
    for rc in (L.pp_attention_workspace(ctypes.byref(p), ctypes.byref(a)),
               L.pp_paged_attention(ctypes.byref(p), ctypes.byref(a), None)):
        assert rc == getattr(B, "PP_E_" + code) and B.pp_last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(requests=-1), "ARG"), (dict(requests=65537), "ARG"), (dict(tokens=-1), "ARG"),
    (dict(max_new=-1), "ARG"), (dict(max_len=-1), "ARG"), (dict(max_blocks=-1), "ARG"),
    (dict(window=-1), "ARG"), (dict(row_stride=-1), "ARG"), (dict(q_heads=3), "ARG"), (dict(q_heads=0), "ARG"),
    (dict(dtype=B.PP_E4M3), "ARG"), (dict(dtype=B.PP_F16), "ARG"), (dict(scale=float("nan")), "ARG"),
    (dict(scale=float("inf")), "ARG"), (dict(tokens=2 ** 30), "UNSUPPORTED"),
    (dict(max_blocks=2 ** 28), "UNSUPPORTED"), (dict(q=None), "ARG"), (dict(out=None), "ARG"),
    (dict(query_start=None), "ARG"), (dict(length=None), "ARG"), (dict(block_table=None), "ARG"),
    (dict(q=AT + 8), "ARG"), (dict(out=AT + 2), "ARG"), (dict(q_token_stride=4), "ARG"),
    (dict(q_head_stride=-128), "ARG"), (dict(out_head_stride=127), "ARG"), (dict(out_token_stride=-512), "ARG")])
def test_attention_refusals(L, kw, code):
    a = _attention(**kw)
    assert L.pp_paged_attention(ctypes.byref(_kv_pages()), ctypes.byref(a), None) == getattr(B, "PP_E_" + code)
    assert B.pp_last_error()


def test_attention_of_nothing(L):
    for kw in (dict(requests=0), dict(tokens=0), dict(max_new=0)):
        a = _attention(**kw)
        assert L.pp_attention_workspace(ctypes.byref(_kv_pages()), ctypes.byref(a)) == 0
        assert L.pp_paged_attention(ctypes.byref(_kv_pages()), ctypes.byref(a), None) == B.PP_OK


def test_paths_of_a_workload(L):
    inst = W.make_workload("tree2k")
    table = B.pp_prefix_table(inst.parent)
    assert np.array_equal(table[:, 15], inst.depth)
    assert np.array_equal(table[:, 1], inst.parent)


@pytest.mark.parametrize("requests,tokens,q_heads,heads,max_new,max_len", [
    (8, 8192, 64, 8, 2048, 131_072), (33, 16_384, 128, 8, 4096, 1_000_000), (1, 1, 64, 1, 1, 2 ** 30)])
def test_attention_workspace_stays_small(L, requests, tokens, q_heads, heads, max_new, max_len):
    """Single tokens beside long prompts: parts of the few rows that are cut, not of every token."""
    a = _attention(requests=requests, tokens=tokens, q_heads=q_heads, max_new=max_new, max_len=max_len, max_blocks=1000)
    need = L.pp_attention_workspace(ctypes.byref(_kv_pages(heads=heads)), ctypes.byref(a))
    rows = 4 * 128 * tokens * q_heads
    assert 0 <= need < 2 ** 29 + 2 * rows


def test_refuses_a_page_whose_span_overflows(L):
    big = 1 << 47
    p = _kv_pages(heads=2 ** 30, head_stride=big, token_stride=big, page_stride=big)
    a = _attention(q_heads=2 ** 30, tokens=1)
    assert L.pp_attention_workspace(ctypes.byref(p), ctypes.byref(a)) == B.PP_E_UNSUPPORTED
    assert L.pp_attention_workspace(ctypes.byref(_kv_pages(page_stride=1 << 48)), ctypes.byref(a)) == B.PP_E_ARG

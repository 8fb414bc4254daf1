"""Bounds and sizes at their ends: what the prefix cache's host side makes of them (no GPU needed)."""

import ctypes

import pytest

from paper_2608_01655_amd import binding as B
from tests.test_serve_host import L, _attention, _kv_pages  # noqa: F401


def workspace(L, **kw):
    return L.pp_attention_workspace(ctypes.byref(_kv_pages(heads=8)), ctypes.byref(_attention(**kw)))


@pytest.mark.parametrize("blocks", [1, 4, 300, 8192])
@pytest.mark.parametrize("requests,tokens,max_new", [(1, 1, 1), (512, 512, 1), (64, 256, 4), (1, 512, 512), (33, 9000, 600)])
def test_keys_end_with_the_rows_of_the_block_table(L, requests, tokens, max_new, blocks):
    """A bound above what a row of the block table holds asks for no more memory than that."""
    kw = dict(requests=requests, tokens=tokens, max_new=max_new, q_heads=64, max_blocks=blocks)
    want = workspace(L, max_len=blocks * 16, **kw)
    for max_len in (blocks * 16 + 1, 1 << 20, (1 << 31) - 128, (1 << 31) - 1):
        if max_len > blocks * 16:
            assert workspace(L, max_len=max_len, **kw) == want >= 0

"""Bounds and sizes at their ends: what the prefix cache's host side makes of them (no GPU needed)."""

import ctypes
import os
import subprocess

import pytest

from paper_2608_01655_amd import binding as B
from paper_2608_01655_amd import build
from tests.test_serve_host import AT, L, _attention, _block_args, _kv_pages  # noqa: F401


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


ON_EACH_GPU = r"""
#include "pp_serve.h"
#include <cstdio>

int main() {
  pp::OnEachGpu once;
  int calls = 0;
  hipError_t answer = hipErrorUnknown;
  auto at = [&](int gpu) {
    return once(gpu, [&] {
      ++calls;
      return answer;
    });
  };
  if (at(0) != hipErrorUnknown || at(0) != hipErrorUnknown || calls != 2) return 1;   // a failure is not kept
  answer = hipSuccess;
  if (at(0) != hipSuccess || at(0) != hipSuccess || calls != 3) return 2;             // once where it succeeds
  if (at(1) != hipSuccess || calls != 4 || at(63) != hipSuccess || calls != 5) return 3;   // on each GPU
  answer = hipErrorUnknown;
  if (at(0) != hipSuccess || at(1) != hipSuccess || at(63) != hipSuccess || calls != 5) return 4;
  if (at(2) != hipErrorUnknown || at(64) != hipErrorUnknown || calls != 7) return 5;
  answer = hipSuccess;
  if (at(64) != hipSuccess || at(64) != hipSuccess || calls != 9) return 6;
  return 0;
}
"""


def test_what_is_set_up_on_each_gpu(tmp_path):
    """A kernel's LDS size is set on every GPU that it is launched on, and a failure is tried again."""
    src, exe = tmp_path / "once.cpp", tmp_path / "once"
    src.write_text(ON_EACH_GPU)
    include = os.path.join(os.path.dirname(os.path.dirname(build.hipcc())), "include")
    if not os.path.isdir(os.path.join(include, "hip")):
        include = "/opt/rocm/include"
    subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", include, "-I", build.INCLUDE, "-I", build.CSRC,
                    str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)]).returncode == 0


def test_block_tables_refuse_rows_that_overlap(L):
    """Rows of an expanded tensor, or closer than they are long, would be written over one another."""
    for kw in (dict(row_stride=0), dict(row_stride=7), dict(requests=65536, row_stride=7)):
        assert L.pp_block_tables(ctypes.byref(_block_args(**kw)), None) == B.PP_E_ARG
        assert "overlap" in B.pp_last_error()


@pytest.mark.parametrize("kw", [dict(max_len=30_000), dict(requests=1, tokens=600, max_new=600, max_len=30_000, max_blocks=2000)])
def test_attention_refuses_a_workspace_that_does_not_do(L, kw):
    """None, too little of it, and one that does not start at 256 bytes: refused before anything is enqueued."""
    kw = dict(dict(max_blocks=2000), **kw)
    p = _kv_pages()
    need = L.pp_attention_workspace(ctypes.byref(p), ctypes.byref(_attention(**kw)))
    assert need > 0
    for at, size in ((None, need), (AT, need - 1), (AT, 0), (AT, -1), (AT + 16, need + 1024), (AT + 128, need + 1024)):
        a = _attention(workspace=at, workspace_bytes=size, **kw)
        assert L.pp_paged_attention(ctypes.byref(p), ctypes.byref(a), None) == B.PP_E_ARG, (at, size)
        assert "workspace" in B.pp_last_error()


def test_writes_refuse_rows_that_overlap(L):
    """Pages of an expanded tensor, or rows closer than they are long; of one page or head its stride says nothing."""
    rows = (3, B.PP_BF16, AT, 256, 128, AT, 256, 128, AT, None)
    for kw in (dict(page_stride=0), dict(page_stride=64), dict(head_stride=0), dict(head_stride=120), dict(token_stride=0),
               dict(token_stride=64), dict(n_pages=1, token_stride=0), dict(heads=1, token_stride=0)):
        assert L.pp_kv_write(ctypes.byref(_kv_pages(**kw)), *rows) == B.PP_E_ARG
        assert "overlap" in B.pp_last_error()
    for kw in (dict(out_token_stride=0), dict(out_token_stride=120), dict(out_head_stride=0), dict(out_head_stride=64)):
        assert L.pp_paged_attention(ctypes.byref(_kv_pages()), ctypes.byref(_attention(**kw)), None) == B.PP_E_ARG
        assert "overlap" in B.pp_last_error()

// pp_serve.h -- shared declarations of the prefix cache's operators: host
// checks and dispatch (pp_serve.cpp), block tables and page writes
// (pp_cache.hip), attention (pp_attend.hip, pp_latent.hip), norms and rotary
// positions (pp_rotary.hip), copies, forks and the free list of pages
// (pp_pages.hip).  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

#include "prefixplace.h"

namespace pp {

// A line of the prefix table: 14 levels, the next line's node, the depth.
constexpr int kLine = 16;
constexpr int kHop = 14;

// Blocks that one launch takes: threads past 2^32 are left out, and no error says so.
constexpr int64_t most_blocks(int threads) { return 0xffffffff / threads; }

// What has to succeed once on each GPU.  A failure is tried again by the next call; two threads may
// both come through the first time.
class OnEachGpu {
  std::atomic<uint64_t> done_{0};      // one bit a GPU; those from 64 on are set up every time

 public:
  template <class F>
  hipError_t operator()(int gpu, F set) {
    const uint64_t bit = gpu >= 0 && gpu < 64 ? uint64_t{1} << gpu : 0;
    if (done_.load(std::memory_order_acquire) & bit) return hipSuccess;
    const hipError_t e = set();
    if (e == hipSuccess) done_.fetch_or(bit, std::memory_order_release);
    return e;
  }
};

hipError_t launch_block_tables(const pp_block_args& a, hipStream_t st);
hipError_t launch_kv_write(const pp_kv_pages& p, int32_t tokens, int32_t dtype, const void* k,
                           int64_t kt, int64_t kh, const void* v, int64_t vt, int64_t vh,
                           const int64_t* slot, hipStream_t st);

hipError_t launch_rotary(const pp_rotary_args& a, const pp_kv_pages* pages, hipStream_t st);
hipError_t launch_page_copy(const pp_copy_args& a, hipStream_t st);
hipError_t launch_fork_tables(const pp_fork_args& a, hipStream_t st);
hipError_t launch_free_pages(const pp_free_args& a, hipStream_t st);

int64_t latent_workspace(const pp_kv_pages& p, int32_t value_dim, const pp_attention_args& a);
hipError_t launch_latent(const pp_kv_pages& p, int32_t value_dim, const pp_attention_args& a, hipStream_t st);

int64_t attention_workspace(const pp_kv_pages& p, const pp_attention_args& a);
hipError_t launch_attention(const pp_kv_pages& p, const pp_attention_args& a, hipStream_t st);

}  // namespace pp

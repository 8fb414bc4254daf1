// pp_serve.h -- shared declarations of the prefix cache's operators: host
// checks and dispatch (pp_serve.cpp), block tables and page writes
// (pp_cache.hip), attention (pp_attend.hip).  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

#include "prefixplace.h"

namespace pp {

// A line of the prefix table: 14 levels, the next line's node, the depth.
constexpr int kLine = 16;
constexpr int kHop = 14;

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

int64_t attention_workspace(const pp_kv_pages& p, const pp_attention_args& a);
hipError_t launch_attention(const pp_kv_pages& p, const pp_attention_args& a, hipStream_t st);

}  // namespace pp

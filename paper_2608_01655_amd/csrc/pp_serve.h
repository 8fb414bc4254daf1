// pp_serve.h -- shared declarations of the prefix cache's operators: host
// checks and dispatch (pp_serve.cpp), block tables and page writes
// (pp_cache.hip), attention (pp_attend.hip).  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "prefixplace.h"

namespace pp {

// A line of the prefix table: 14 levels, the next line's node, the depth.
constexpr int kLine = 16;
constexpr int kHop = 14;

hipError_t launch_block_tables(const pp_block_args& a, hipStream_t st);
hipError_t launch_kv_write(const pp_kv_pages& p, int32_t tokens, int32_t dtype, const void* k,
                           int64_t kt, int64_t kh, const void* v, int64_t vt, int64_t vh,
                           const int64_t* slot, hipStream_t st);

int64_t attention_workspace(const pp_kv_pages& p, const pp_attention_args& a);
hipError_t launch_attention(const pp_kv_pages& p, const pp_attention_args& a, hipStream_t st);

}  // namespace pp

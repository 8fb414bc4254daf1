// pp_cache.hip -- block tables, slot maps and page writes of the prefix
// cache (gfx950).

#include "pp_serve.h"

namespace pp {

namespace {

constexpr int kWave = 64;
constexpr int kWalkWaves = 4;     // requests a block of k_walk looks up, one wave each
constexpr int kPathLds = 128;     // chunks of a path kept in LDS between its two uses
constexpr int kFillWaves = 16;    // waves of a block of k_fill
constexpr int kStepMost = 64;     // requests k_step takes

struct Span {
  int32_t start, end;
};

__device__ __forceinline__ int32_t ceil_div(int32_t a, int32_t shift) {
  return (int32_t)(((int64_t)a + (1 << shift) - 1) >> shift);
}

__device__ __forceinline__ int32_t clamp_end(const pp_block_args& a, int32_t len, int32_t start) {
  if (a.max_new == 0) return len;
  const int64_t e = (int64_t)start + a.max_new;
  return e < len ? (int32_t)e : len;
}

// Looks request r up and writes its row's found pages; one wave, all lanes
// active.  slots: kPathLds words of LDS of this wave's own.
//
// Found chunks are the run of resident ones from the root down, and the path
// is read from the leaf up: the run ends at the shallowest chunk without a
// slot, known only at the root.  So the slots wait in LDS (deeper paths are
// read twice) until then.
__device__ Span walk(const pp_block_args& a, int32_t r, int lane, int32_t* slots) {
  int32_t len = a.length[r];
  if (len < 0) len = 0;
  const int32_t cached = a.cached[r];
  if (cached >= 0) {
    const int32_t start = cached < len ? cached : len;
    return {start, clamp_end(a, len, start)};
  }
  const int32_t leaf = a.leaf[r];
  const int32_t most = len > 0 ? (len - 1) / a.chunk_tokens : 0;   // chunks before the last token
  int32_t depth = -1, hit = 0;
  if (leaf >= 0 && leaf < a.n && most > 0) {
    depth = a.prefix_table[(int64_t)leaf * kLine + kLine - 1];
    if (depth < 0 || depth >= a.n) depth = a.n - 1;
    hit = depth + 1;
  }
  // position of lane j of the current line: at - j
  int32_t v = leaf;
  for (int32_t at = depth; at >= 0; at -= kHop) {
    const int32_t id = lane < kLine ? a.prefix_table[(int64_t)v * kLine + lane] : -1;
    const bool mine = lane < kHop && at - lane >= 0;
    int32_t s = -1;
    if (mine && id >= 0 && id < a.n) {
      s = a.slot[id];
      if (s >= a.n_slots) s = -1;
    }
    if (mine && at - lane < kPathLds) slots[at - lane] = s;
    const uint64_t none = __ballot(mine && s < 0);
    if (none) hit = at - (63 - __builtin_clzll(none));
    v = __shfl(id, kHop);
    if (v < 0 || v >= a.n) {
      if (at >= kHop) hit = 0;   // the line does not reach its root
      break;
    }
  }
  const int32_t found = hit < most ? hit : most;
  const int32_t per = a.chunk_tokens / a.page_size;
  int32_t* row = a.block_table + (int64_t)r * a.row_stride;
  const int32_t in_lds = found < kPathLds ? found : kPathLds;
  const int64_t blocks = (int64_t)in_lds * per;
  for (int64_t b = lane; b < blocks && b < a.max_blocks; b += kWave)
    row[b] = slots[b / per] * per + (int32_t)(b % per);
  v = leaf;
  for (int32_t at = found > kPathLds ? depth : -1; at >= kPathLds; at -= kHop) {
    const int32_t id = lane < kLine ? a.prefix_table[(int64_t)v * kLine + lane] : -1;
    const bool mine = lane < kHop && at - lane >= kPathLds && at - lane < found;
    if (mine && id >= 0 && id < a.n) {
      const int32_t s = a.slot[id];
      for (int64_t j = 0, b = (int64_t)(at - lane) * per; j < per && b + j < a.max_blocks; ++j)
        row[b + j] = s * per + (int32_t)j;
    }
    v = __shfl(id, kHop);
    if (v < 0 || v >= a.n) break;
  }
  const int32_t start = found * a.chunk_tokens;
  return {start, clamp_end(a, len, start)};
}

// Bound by the chain of dependent reads: 257 new requests on paths of up to 8
// chunks 3.6 us; 4,096, 512 of them new on paths of up to 64, 11.4 us.
__global__ void __launch_bounds__(kWave* kWalkWaves) k_walk(pp_block_args a) {
  __shared__ int32_t slots[kWalkWaves][kPathLds];
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const int32_t r = blockIdx.x * kWalkWaves + wave;
  if (r >= a.requests) return;
  const Span s = walk(a, r, lane, slots[wave]);
  if (lane == 0) {
    a.start[r] = s.start;
    a.end[r] = s.end;
  }
}

__device__ __forceinline__ int32_t cap32(int64_t x) { return (int32_t)(x < INT32_MAX ? x : INT32_MAX); }

// Every block sums the tokens and pages of all requests and of those before its own (8 bytes a
// request out of L2), then EACH waves serve each request: 4 for up to 512 requests, where the chain
// of reads counts, else 1 (4,096 requests took 40 us with 4, 14 us with 1).
template <int EACH>
__global__ void __launch_bounds__(kWave* kFillWaves) k_fill(pp_block_args a, int shift) {
  constexpr int kOwn = kFillWaves / EACH;
  __shared__ int64_t part[kFillWaves][4];
  __shared__ int64_t mine[kOwn][2];
  const int wave = threadIdx.x / kWave, own = wave / EACH;
  const int at = threadIdx.x % (kWave * EACH);
  const int32_t first = blockIdx.x * kOwn, r = first + own;
  int32_t start = 0, end = 0;
  if (r < a.requests) {
    start = a.start[r];
    end = a.end[r];
  }
  int64_t sum[4] = {0, 0, 0, 0};     // tokens and pages: of the requests before, of all
#pragma unroll 2
  for (int32_t i = threadIdx.x; i < a.requests; i += kWave * kFillWaves) {
    const int32_t s = a.start[i], e = a.end[i];
    const int64_t t = e - s, p = ceil_div(e, shift) - ceil_div(s, shift);
    sum[0] += i < first ? t : 0;
    sum[1] += i < first ? p : 0;
    sum[2] += t;
    sum[3] += p;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    for (int o = kWave / 2; o; o >>= 1) sum[j] += __shfl_xor(sum[j], o);
  if (threadIdx.x % kWave == 0)
    for (int j = 0; j < 4; ++j) part[wave][j] = sum[j];
  const int32_t b0 = ceil_div(start, shift), b1 = ceil_div(end, shift);
  if (at == 0) {
    mine[own][0] = end - start;
    mine[own][1] = b1 - b0;
  }
  __syncthreads();
  int64_t t0 = 0, p0 = 0, t1 = 0, p1 = 0;
  for (int w = 0; w < kFillWaves; ++w) {
    t0 += part[w][0];
    p0 += part[w][1];
    t1 += part[w][2];
    p1 += part[w][3];
  }
  for (int w = 0; w < own; ++w) {
    t0 += mine[w][0];
    p0 += mine[w][1];
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.query_start[0] = 0;
    a.taken[0] = cap32(p1);
  }
  // numbers that no token has
  for (int64_t t = t1 + (int64_t)blockIdx.x * blockDim.x + threadIdx.x; t < a.max_tokens;
       t += (int64_t)gridDim.x * blockDim.x) {
    a.slot_map[t] = -1;
    a.position[t] = 0;
  }
  if (r >= a.requests) return;
  if (at == 0) a.query_start[r + 1] = cap32(t0 + end - start);
  int32_t* row = a.block_table + (int64_t)r * a.row_stride;
  // the page of block b >= b0
  auto fresh = [&](int32_t b) {
    const int64_t i = p0 + b - b0;
    return i < a.n_free ? a.free_pages[i] : -1;
  };
  constexpr int kThreads = kWave * EACH, kTurn = 4;
  for (int32_t b = b0 + at; b < b1 && b < a.max_blocks; b += kThreads) row[b] = fresh(b);
  const int32_t mask = a.page_size - 1;
  const int64_t last = t0 + (end - start) < a.max_tokens ? end - start : a.max_tokens - t0;
  for (int64_t i = at; i < last; i += kThreads * kTurn) {
    int32_t page[kTurn];
#pragma unroll
    for (int j = 0; j < kTurn; ++j) {      // the reads of a turn before its writes
      const int32_t b = (int32_t)((start + i + j * kThreads) >> shift);
      page[j] = i + j * kThreads < last && b < a.max_blocks ? (b < b0 ? row[b] : fresh(b)) : -1;
    }
#pragma unroll
    for (int j = 0; j < kTurn; ++j) {
      const int64_t n = i + j * kThreads;
      if (n >= last) break;
      const int32_t pos = (int32_t)(start + n);
      a.slot_map[t0 + n] = page[j] < 0 ? -1 : ((int64_t)page[j] << shift) + (pos & mask);
      a.position[t0 + n] = pos;
    }
  }
}

// The whole of it for few requests and tokens, in one launch and block: such a call is bound by its
// chain of reads, so what is needed from free_pages is read ahead of knowing how much.  64 requests
// that go on: 3.4 us, 8.2 us with the call (two launches took 14.7).
__global__ void __launch_bounds__(1024) k_step(pp_block_args a, int shift) {
  constexpr int kWaves = 16;
  __shared__ int32_t slots[kWaves][kPathLds], ahead[1024];
  __shared__ int32_t starts[kStepMost], ends[kStepMost], open[kStepMost];
  __shared__ int64_t tok[kStepMost + 1], page[kStepMost + 1];
  __shared__ uint64_t begins;
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, tid = threadIdx.x;
  const int32_t mask = a.page_size - 1, R = a.requests;
  const int32_t next = tid < a.n_free ? a.free_pages[tid] : -1;
  if (wave == 0) {
    const bool live = lane < R;
    int32_t len = live ? a.length[lane] : 0;
    const int32_t cached = live ? a.cached[lane] : 0;
    if (len < 0) len = 0;
    if (live && cached >= 0) {
      const int32_t s = cached < len ? cached : len;
      starts[lane] = s;
      ends[lane] = clamp_end(a, len, s);
      // the page its last token so far lies in
      open[lane] = (s & mask) && (s >> shift) < a.max_blocks ? a.block_table[lane * a.row_stride + (s >> shift)] : -1;
    }
    const uint64_t b = __ballot(live && cached < 0);
    if (lane == 0) begins = b;
  }
  ahead[tid] = next;
  __syncthreads();
  int k = 0;
  for (uint64_t left = begins; left; left &= left - 1, ++k) {
    if (k % kWaves != wave) continue;
    const int32_t r = __builtin_ctzll(left);
    const Span s = walk(a, r, lane, slots[wave]);
    if (lane == 0) {
      starts[r] = s.start;
      ends[r] = s.end;
    }
  }
  __syncthreads();
  if (wave == 0) {
    const int32_t s = lane < R ? starts[lane] : 0, e = lane < R ? ends[lane] : 0;
    int64_t t = e - s, p = ceil_div(e, shift) - ceil_div(s, shift);
    for (int o = 1; o < kWave; o <<= 1) {
      const int64_t x = __shfl_up(t, o), y = __shfl_up(p, o);
      if (lane >= o) {
        t += x;
        p += y;
      }
    }
    if (lane == 0) tok[0] = page[0] = 0;
    tok[lane + 1] = t;
    page[lane + 1] = p;
    if (lane < R) {
      a.start[lane] = s;
      a.end[lane] = e;
      a.query_start[lane + 1] = cap32(t);
    }
    if (lane == 0) a.query_start[0] = 0;
    if (lane == kWave - 1) a.taken[0] = cap32(p);
  }
  __syncthreads();
  auto fresh = [&](int64_t i) { return i >= a.n_free ? -1 : i < 1024 ? ahead[i] : a.free_pages[i]; };
  for (int32_t r = wave; r < R; r += kWaves) {
    const int32_t b0 = ceil_div(starts[r], shift), b1 = ceil_div(ends[r], shift);
    int32_t* row = a.block_table + (int64_t)r * a.row_stride;
    for (int32_t b = b0 + lane; b < b1 && b < a.max_blocks; b += kWave) row[b] = fresh(page[r] + b - b0);
  }
  for (int64_t t = tid; t < a.max_tokens; t += 1024) {
    int64_t slot = -1;
    int32_t pos = 0;
    if (t < tok[R]) {
      int32_t r = 0;              // the last request that starts at or before t
      for (int32_t o = kStepMost / 2; o; o >>= 1)
        if (r + o < R && tok[r + o] <= t) r += o;
      pos = (int32_t)(starts[r] + (t - tok[r]));
      const int32_t b = pos >> shift, b0 = ceil_div(starts[r], shift);
      int32_t pg = -1;
      if (b < a.max_blocks) pg = b < b0 ? open[r] : fresh(page[r] + b - b0);
      if (pg >= 0) slot = ((int64_t)pg << shift) + (pos & mask);
    }
    a.slot_map[t] = slot;
    a.position[t] = pos;
  }
}

// ------------------------------------------------------------ page writes ---

typedef __attribute__((__vector_size__(16))) int i32x4;
typedef __attribute__((__vector_size__(8))) int i32x2;

__device__ __forceinline__ float widen(uint16_t x, bool f16) {
  if (f16) return (float)__builtin_bit_cast(_Float16, x);
  return __builtin_bit_cast(float, (uint32_t)x << 16);
}

// value / scale, held to the type's range; NaN stays NaN.  The quotient is value * (1 / scale) with
// one correction by its residual, which rounds as the division does for the scales it is used for
// (2^-60 .. 2^60) wherever the result is not 0; the division itself took 11 instructions an element
// and bound the kernel.
struct Scale {
  float s, inv;
  bool plain;
};

__device__ __forceinline__ Scale scale_of(float s) { return {s, 1.f / s, s >= 0x1p-60f && s <= 0x1p60f}; }

__device__ __forceinline__ float shrink(float x, const Scale& c) {
  float y;
  if (c.plain) {
    const float q = x * c.inv;
    y = __builtin_fmaf(__builtin_fmaf(-q, c.s, x), c.inv, q);
    y = fabsf(q) > 512.f ? q : y;      // an infinity has no residual
  } else {
    y = x / c.s;
  }
  return y != y ? y : fminf(fmaxf(y, -448.f), 448.f);
}

// Eight elements of a row a thread, of k and of v.  Bound by what it moves:
// a row is read and written once, 16 bytes a lane.  65,536 tokens of 8 heads,
// dim 128 (537 MB) 104 us, 5.2 TB/s, a large copy's rate; 8,191 into 8 bits
// (50 MB) 12.1 us, 4.2 TB/s; 61 tokens of 2 heads 2.9 us.
template <bool kNarrow>
__global__ void __launch_bounds__(256) k_write(pp_kv_pages p, int32_t tokens, bool f16,
                                               const uint16_t* k, int64_t kt, int64_t kh,
                                               const uint16_t* v, int64_t vt, int64_t vh,
                                               const int64_t* slot, int shift, int dim8,
                                               int64_t total) {
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < total;
       i += (int64_t)gridDim.x * blockDim.x) {
    const int32_t d = (int32_t)(i % dim8) * 8;
    const int64_t th = i / dim8;
    const int32_t h = (int32_t)(th % p.heads);
    const int64_t t = th / p.heads;
    const int64_t at = slot[t];
    if (at < 0 || at >> shift >= p.n_pages) continue;
    const int64_t to = (at >> shift) * p.page_stride + h * p.head_stride +
                       (at & (p.page_size - 1)) * p.token_stride + d;
    const i32x4 x = *(const i32x4*)(k + t * kt + h * kh + d);
    const i32x4 y = *(const i32x4*)(v + t * vt + h * vh + d);
    if constexpr (!kNarrow) {
      *(i32x4*)((uint16_t*)p.k + to) = x;
      *(i32x4*)((uint16_t*)p.v + to) = y;
    } else {
      auto pack = [&](i32x4 w, const Scale& s) {
        float f[8];
        for (int j = 0; j < 8; ++j) f[j] = shrink(widen((uint16_t)(w[j / 2] >> (16 * (j % 2))), f16), s);
        i32x2 o;
        for (int j = 0; j < 2; ++j) {
          int q = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * j], f[4 * j + 1], 0, false);
          o[j] = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * j + 2], f[4 * j + 3], q, true);
        }
        return o;
      };
      *(i32x2*)((uint8_t*)p.k + to) = pack(x, scale_of(p.k_scale ? p.k_scale[h] : 1.f));
      *(i32x2*)((uint8_t*)p.v + to) = pack(y, scale_of(p.v_scale ? p.v_scale[h] : 1.f));
    }
  }
}

}  // namespace

hipError_t launch_block_tables(const pp_block_args& a, hipStream_t st) {
  const int shift = __builtin_ctz(a.page_size);
  // one block writes some 1,024 tokens a microsecond; two launches cost more than that up to here
  if (a.requests <= kStepMost && a.max_tokens <= 8192) {
    k_step<<<1, 1024, 0, st>>>(a, shift);
    return hipGetLastError();
  }
  if (a.requests)
    k_walk<<<(a.requests + kWalkWaves - 1) / kWalkWaves, kWave * kWalkWaves, 0, st>>>(a);
  const bool many = a.requests > 512;
  const int own = many ? kFillWaves : kFillWaves / 4;
  const int blocks = a.requests ? (a.requests + own - 1) / own : 1;
  (many ? k_fill<1> : k_fill<4>)<<<blocks, kWave * kFillWaves, 0, st>>>(a, shift);
  return hipGetLastError();
}

hipError_t launch_kv_write(const pp_kv_pages& p, int32_t tokens, int32_t dtype, const void* k,
                           int64_t kt, int64_t kh, const void* v, int64_t vt, int64_t vh,
                           const int64_t* slot, hipStream_t st) {
  const int shift = __builtin_ctz(p.page_size), dim8 = p.dim / 8;
  const int64_t total = (int64_t)tokens * p.heads * dim8;
  const int64_t blocks = (total + 255) / 256;
  const unsigned grid = (unsigned)(blocks < (1 << 20) ? blocks : (1 << 20));
  auto kern = p.dtype == PP_E4M3 ? k_write<true> : k_write<false>;
  kern<<<grid, 256, 0, st>>>(p, tokens, dtype == PP_F16, (const uint16_t*)k, kt, kh,
                             (const uint16_t*)v, vt, vh, slot, shift, dim8, total);
  return hipGetLastError();
}

}  // namespace pp

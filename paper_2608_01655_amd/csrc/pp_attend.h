// pp_attend.h -- what the attention kernels over pages share (pp_attend.hip, pp_latent.hip): matrix
// instructions, conversions, requests and their parts.
#pragma once

#include "pp_serve.h"

#include <cmath>
#include <type_traits>
#include <utility>

namespace pp {

// Functions here are of the file that includes them; not every one has a use in each.
namespace {

typedef __attribute__((__vector_size__(4))) short s16x2;
typedef __attribute__((__vector_size__(8))) short s16x4;
typedef __attribute__((__vector_size__(16))) short s16x8;
typedef __attribute__((__vector_size__(8))) int i32x2;
typedef __attribute__((__vector_size__(16))) int i32x4;
typedef __attribute__((__vector_size__(16))) uint32_t u32x4;
typedef __attribute__((__vector_size__(16))) float f32x4;
typedef __attribute__((__vector_size__(64))) float f32x16;
typedef __attribute__((__vector_size__(4))) __bf16 bf16x2;
typedef __attribute__((__vector_size__(16))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(4))) _Float16 f16x2;
typedef __attribute__((__vector_size__(16))) _Float16 f16x8;

#define LDS_PTR(T, a) ((__attribute__((address_space(3))) T*)(uintptr_t)(a))

constexpr int kWave = 64;
constexpr float kLog2e = 1.44269504088896340736f;

// Growth of the maximum, in the exponent, that is let pass, and what the weights are scaled up by for
// the second product.  f16 has a smallest normal value of 2^-14: without the scale a key 10 below the
// maximum is held in fewer bits and one 18 below not at all, although many such keys may be all that
// the output is made of.  With it weights lie below 2^14 (the type ends at 2^16, which leaves room for
// the rounding of c m), and a key is held whole down to 2^-24 of the largest, in units of 2^-34 below.
template <bool F16>
constexpr float kLag = F16 ? 4.f : 8.f;
template <bool F16>
constexpr float kLift = F16 ? 10.f : 0.f;

// f(0), f(1) .. f(N - 1), the numbers as constants.
template <int N, class F, int... I>
__device__ __forceinline__ void each_(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>()), ...);
}
template <int N, class F>
__device__ __forceinline__ void each(F&& f) {
  each_<N>(f, std::make_integer_sequence<int, N>());
}

extern __shared__ __attribute__((aligned(1024))) char g_lds[];

__device__ __forceinline__ uint32_t lds_base() {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)g_lds;
}

// 16 bytes a lane from base + off straight into LDS at `to` + 16 * lane; counted in vmcnt like any
// load, and the compiler is not told: wait_loads() before the reads.  (It keeps nothing in m0.)
__device__ __forceinline__ void load_lds(uint32_t to, uint32_t off, const char* base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :: "s"(__builtin_amdgcn_readfirstlane(to)), "v"(off), "s"(base) : "memory");
}

// The same into LDS at to + N.
template <int N>
__device__ __forceinline__ void load_lds_at(uint32_t to, uint32_t off, const char* base) {
  asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :: "s"(to), "v"(off), "s"(base), "n"(N) : "memory", "scc");
}

template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

__device__ __forceinline__ void barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// What is taken off a score's exponent under the maximum m.
template <bool F16>
__device__ __forceinline__ float top_of(float m, float c) {
  return m == -INFINITY ? 0.f : F16 ? __builtin_fmaf(m, c, -kLift<F16>) : m * c;
}

template <bool F16>
__device__ __forceinline__ f32x4 mfma16(s16x8 a, s16x8 b, f32x4 c) {
  if constexpr (F16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

template <bool F16>
__device__ __forceinline__ f32x16 mfma32(s16x8 a, s16x8 b, f32x16 c) {
  if constexpr (F16)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Two floats rounded to nearest into the rows' type.
template <bool F16>
__device__ __forceinline__ int pack2(float x, float y) {
  if constexpr (F16) {
    f16x2 v = {(_Float16)x, (_Float16)y};
    return __builtin_bit_cast(int, v);
  } else {
    bf16x2 v = {(__bf16)x, (__bf16)y};
    return __builtin_bit_cast(int, v);
  }
}

template <bool F16>
__device__ __forceinline__ s16x8 pack8(const float* x) {
  i32x4 v;
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = pack2<F16>(x[2 * j], x[2 * j + 1]);
  return __builtin_bit_cast(s16x8, v);
}

// Eight e4m3 values widened to the rows' type (exact).
template <bool F16>
__device__ __forceinline__ s16x8 widen8(i32x2 x) {
  i32x4 v;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    if constexpr (F16) {
      v[2 * j] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x[j], 1.f, false));
      v[2 * j + 1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x[j], 1.f, true));
    } else {
      v[2 * j] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[j], 1.f, false));
      v[2 * j + 1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[j], 1.f, true));
    }
  }
  return __builtin_bit_cast(s16x8, v);
}

// A tile that some row does not see whole gives those keys a weight of 0, and 0 times an infinity
// or NaN would still be NaN.  There V goes into the product with such values as 0, and where one
// turned up, a second product counts them for the rows that do see them: +infinities as 1,
// -infinities as 128, NaN as 16,384 (a tile has at most 64 keys, so the counts stay apart).
template <bool F16>
__device__ __forceinline__ uint32_t not_finite(uint32_t x) {   // bit 15 and bit 31 for the two halves
  if constexpr (F16) return ((x & 0x7c007c00u) + 0x04000400u) & 0x80008000u;
  return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
}

template <bool F16>
__device__ __forceinline__ s16x8 only_finite(s16x8 v, uint32_t& odd) {
  u32x4 x = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t n = not_finite<F16>(x[j]);
    odd |= n;
    x[j] &= ~((n >> 15) * 0xffffu);
  }
  return __builtin_bit_cast(s16x8, x);
}

template <bool F16>
__device__ __forceinline__ s16x8 marks(s16x8 v) {
  s16x8 o;
  const uint16_t top = F16 ? 0x7c00 : 0x7f80;
  const short one = F16 ? 0x3c00 : 0x3f80, b = F16 ? 0x5800 : 0x4300, c = F16 ? 0x7400 : 0x4680;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint16_t u = (uint16_t)v[j];
    o[j] = (u & top) != top ? 0 : (u & 0x7fff) != top ? c : (u >> 15) ? b : one;
  }
  return o;
}

// 1 where the low bits say so.
template <bool F16>
__device__ __forceinline__ s16x8 ones8(uint32_t bits) {
  s16x8 o;
#pragma unroll
  for (int j = 0; j < 8; ++j) o[j] = (bits >> j & 1) ? (short)(F16 ? 0x3c00 : 0x3f80) : (short)0;
  return o;
}

__device__ __forceinline__ float counted(float acc, float n) {
  const int k = (int)n;
  if (k & 127) acc += INFINITY;
  if ((k >> 7) & 127) acc -= INFINITY;
  if (k >> 14) acc += __builtin_nanf("");
  return acc;
}

// Over the two halves of the wave, and over the two 16-lane rows of each half.
template <class F>
__device__ __forceinline__ float over_halves(float x, F f) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto v = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return f(__builtin_bit_cast(float, (uint32_t)v[0]), __builtin_bit_cast(float, (uint32_t)v[1]));
}

template <class F>
__device__ __forceinline__ float over_rows(float x, F f) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto v = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return f(__builtin_bit_cast(float, (uint32_t)v[0]), __builtin_bit_cast(float, (uint32_t)v[1]));
}

struct Max {
  __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct Sum {
  __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};

// ------------------------------------------------------------- requests ---

// How a call is split: requests of at most `few` rows go to k_rows, the others to k_tiles; a
// request's keys are cut every `cut` keys, into at most `parts` parts of which the last is open.
struct Plan {
  int32_t few, group;
  int32_t cut_rows, parts_rows, cut_tiles, parts_tiles;
  int32_t slots;                 // tiles of rows at most, for k_tiles' grid
  float c;                       // |scale| log2(e)
  int32_t negative, shift;
  // normalised parts [parts_tiles][tokens][q_heads][dim] of k_tiles, [parts_rows][requests][heads][few][dim]
  // of k_rows (which may have many parts, but of few rows), and their log sums
  float *part, *part_lse, *row_part, *row_lse;
};

struct Request {
  int32_t first, count;          // its tokens
  int32_t start;                 // position of the first one
  int32_t lo, hi;                // keys any of its rows sees, lo a multiple of 64
};

__device__ __forceinline__ Request request(const pp_attention_args& a, const Plan& pl, int32_t r) {
  Request q;
  int32_t b = a.query_start[r], e = a.query_start[r + 1];
  b = b < 0 ? 0 : b < a.tokens ? b : a.tokens;
  e = e < b ? b : e < a.tokens ? e : a.tokens;
  const int32_t len = a.length[r] > 0 ? a.length[r] : 0;
  const int64_t room = (int64_t)a.max_blocks << pl.shift;
  q.first = b;
  q.count = e - b;
  q.start = len - q.count;
  q.hi = len < room ? len : (int32_t)room;
  q.lo = a.window && q.start >= a.window ? (q.start - a.window + 1) & ~63 : 0;
  return q;
}

__device__ __forceinline__ int32_t parts_of(const Request& q, int32_t cut, int32_t most) {
  if (q.hi <= q.lo) return 1;
  const int32_t n = (int32_t)(((int64_t)q.hi - q.lo + cut - 1) / cut);
  return n < most ? n : most;
}

__device__ __forceinline__ bool sees(int32_t pos, int32_t key, int32_t window) {
  return key <= pos && (window == 0 || (uint32_t)(pos - key) < (uint32_t)window);
}

// Of nt tiles of N keys from `key` on: tiles whole .. tail - 1 are seen whole by every row.
struct Span3 {
  int32_t whole, tail;
};

template <int N>
__device__ __forceinline__ Span3 spans(int32_t key, int32_t nt, int32_t pos_lo, int32_t pos_hi, int32_t k1,
                                       int32_t window) {
  int64_t w = 0;
  if (window) {                                       // tiles with a key <= pos_hi - window
    w = (int64_t)pos_hi - window - key;
    w = w < 0 ? 0 : w / N + 1;
  }
  int64_t e = pos_lo + 1 < k1 ? pos_lo + 1 : k1;      // keys before e are seen, but for the window
  e = e <= key ? 0 : (e - key) / N;
  Span3 s;
  s.whole = __builtin_amdgcn_readfirstlane((int32_t)(w < nt ? w : nt));
  s.tail = __builtin_amdgcn_readfirstlane((int32_t)(e < nt ? e : nt));
  return s;
}

// The last r with f(r) <= x, f increasing, f(0) <= x; all lanes active.
template <class F>
__device__ __forceinline__ int32_t find_last(int32_t count, int32_t x, F f) {
  int32_t n = 0;
  for (int32_t base = 0; base < count; base += kWave) {
    const int32_t r = base + (int32_t)(threadIdx.x % kWave);
    const int32_t k = __popcll(__ballot(r < count && f(r) <= x));
    n += k;
    if (k < kWave) break;
  }
  return __builtin_amdgcn_readfirstlane(n - 1);
}

// The request that a slot of 128 rows is of, and its first slot; r < 0: of none.
struct Slot {
  int32_t r, first;
};

__device__ __forceinline__ Slot slot_of(const pp_attention_args& a, const Plan& pl, int32_t slot) {
  const int lane = threadIdx.x % kWave, G = pl.group;
  if (a.requests <= kWave) {
    // longest request first, so that no long block starts late: on 4 requests of 8,192 to 16,384 tokens the
    // last blocks end 4% after the average and not 18%
    const Request mine = request(a, pl, lane < a.requests ? lane : 0);
    const int64_t mine_rows = lane < a.requests ? (int64_t)mine.count * G : 0;
    const int32_t tiles = mine_rows > pl.few ? (int32_t)((mine_rows + 127) / 128) : 0, keys = mine.hi - mine.lo;
    int32_t base = 0;
    for (int j = 0; j < a.requests; ++j) {
      const int32_t kj = __builtin_amdgcn_readlane(keys, j), tj = __builtin_amdgcn_readlane(tiles, j);
      if (kj > keys || (kj == keys && j < lane)) base += tj;
    }
    const uint64_t at = __ballot(slot >= base && slot < base + tiles);
    if (!at) return {-1, 0};
    const int32_t r = __builtin_ctzll(at);
    return {r, __builtin_amdgcn_readlane(base, r)};
  }
  // request r's tiles start at slot floor(first token * G / 128) + r, which leaves it enough of them
  auto base_of = [&](int32_t i) {
    const int32_t t = a.query_start[i];
    return (int32_t)((int64_t)(t < 0 ? 0 : t < a.tokens ? t : a.tokens) * G / 128) + i;
  };
  const int32_t r = find_last(a.requests, slot, base_of);
  if (r < 0) return {-1, 0};
  const int32_t first = base_of(r);
  return {first > slot ? -1 : r, first};
}

// Page numbers of 64 consecutive tiles of keys, one a lane.
__device__ __forceinline__ int32_t page_of(const pp_kv_pages& p, const pp_attention_args& a,
                                           const Plan& pl, const int32_t* blocks, int64_t key) {
  const int64_t b = key >> pl.shift;
  int32_t page = b < a.max_blocks ? blocks[b] : 0;
  return page < 0 ? 0 : page < p.n_pages ? page : p.n_pages - 1;
}

// Four neighbouring values of a row of out.
template <bool F16>
__device__ __forceinline__ void store4(const pp_attention_args& a, int32_t t, int32_t g, int32_t d, f32x4 x) {
  const i32x2 v = {pack2<F16>(x[0], x[1]), pack2<F16>(x[2], x[3])};
  *(i32x2*)((uint16_t*)a.out + t * a.out_token_stride + g * a.out_head_stride + d) = v;
}

template <class K>
hipError_t allow_lds(OnEachGpu& once, K kern, int bytes) {
  int gpu;
  const hipError_t e = hipGetDevice(&gpu);
  if (e != hipSuccess) return e;
  return once(gpu, [&] { return hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes); });
}

}  // namespace

}  // namespace pp

// pp_attend.hip -- attention of new tokens over paged keys and values (gfx950).
//
// out = sum_j w_j V_j / sum_j w_j, w_j = 2^(c s_j - c m), c = scale log2(e) k_scale, s = <q, K_j>,
// in one pass over the keys with a running maximum m: where it grows by more than kLag in the exponent
// (weights stay below 2^(kLag + kLift)), sums and accumulators are scaled down by 2^(c (m_old - m_new)).
//
// The query heads of a key head and the new tokens of a request are packed into rows (row =
// token * G + head), so that a tile of keys is read once for all of them.  Both products are taken
// transposed: S^T = K Q^T leaves a query in a lane's column and its keys in that lane's registers,
// which is what the second product O^T = V^T P^T takes as its right operand, with the keys in the
// registers' own order.  So weights never leave registers; the keys of V^T are put in the same
// order by transposing LDS reads.
//
// Two kernels share this.  k_rows takes requests of few rows, which the reading of the pages
// bounds: its waves split the keys and each streams its own through LDS with nothing but its own
// counters to wait for.  k_tiles takes the others, which the matrix cores bound: four waves of 32 rows
// share each tile of 64 keys.  Both split long requests over blocks, which leave normalised parts
// and their log sums in the workspace for k_join.
//
// Weights are rounded to the queries' type for the second product (the matrix cores take 32-bit ones
// at a sixteenth of the rate); scores, sums and accumulators are 32 bits.  What it costs: half a unit
// of each weight, in all about as much as rounding the output does (error against 64 bits 2.3e-3 in
// bf16 and 2.9e-4 in f16, where rounding the output alone gives 1.7e-3 and 2.1e-4).
// 8-bit pages are widened to the queries' type after LDS, which is exact.

#include "pp_serve.h"

#include <cmath>
#include <type_traits>
#include <utility>

namespace pp {

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

// ---------------------------------------------------------------- k_rows ---

// Swizzles: the 16-byte unit u of a row lies at u ^ f(row), so that the rows a read takes together
// fall into different banks.
template <int RB>
struct RowsSwizzle {
  static constexpr int kUnits = RB / 16;
  static __device__ __forceinline__ int k(int row) { return row & (kUnits < 16 ? kUnits - 1 : 15); }
  static __device__ __forceinline__ int v(int row, bool narrow) {
    if (narrow) return kUnits >= 8 ? (row & 3) | ((row >> 2) & 4) : row & 3;
    return kUnits >= 16 ? (row & 7) * 2 : (row & 3) * 2;
  }
};

template <bool NARROW, int D, int RT>
struct RowsShape {
  static constexpr int kRB = D * (NARROW ? 1 : 2);          // bytes of a row
  static constexpr int kStage = 2 * 32 * kRB;               // K and V of 32 keys
  static constexpr int kNW = kStage > 8192 ? 2 : 4;         // waves
  static constexpr int kNS = kStage > 4096 ? 2 : 4;         // stages of a wave's ring
  static constexpr int kRing = kNW * kNS * kStage;
  static constexpr int kRow = D + 4;                        // floats of a joined row
  static constexpr int kJoin = kNW * 16 * RT * (kRow + 2) * 4;
  static constexpr int kLds = kRing > kJoin ? kRing : kJoin;
};

// One request, key head and part a block: up to 16 RT rows, in tiles of 16.  Bound by reading the
// pages: 256 requests of 1,024 to 16,384 tokens in 8 bits (2.9 GB) 552 us, 5.3 TB/s; 64 of 500 to
// 8,190 in bf16 75 us, 4.9 TB/s.  Each wave has a ring of its own and keeps NS - 1 tiles of 32 keys
// in flight without a barrier; with four rows in 16 used the matrix cores are 5 to 13% busy.
template <bool F16, bool NARROW, int D, int RT>
__global__ void __launch_bounds__((kWave * RowsShape<NARROW, D, RT>::kNW))
k_rows(pp_kv_pages p, pp_attention_args a, Plan pl) {
  using Sh = RowsShape<NARROW, D, RT>;
  using Sw = RowsSwizzle<Sh::kRB>;
  constexpr int RB = Sh::kRB, UPR = RB / 16, NW = Sh::kNW, NS = Sh::kNS;
  constexpr int kLoads = 32 * RB / 1024;                    // loads a matrix and tile
  constexpr int kRowsPerLoad = 1024 / RB;
  constexpr int DB = D / 16, KS = D / 32;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int h = blockIdx.x % p.heads;
  const int part = (blockIdx.x / p.heads) % pl.parts_rows;
  const int32_t r = blockIdx.x / p.heads / pl.parts_rows;
  const Request q = request(a, pl, r);
  const int G = pl.group;
  const int64_t rows64 = (int64_t)q.count * G;
  if (rows64 == 0 || rows64 > pl.few) return;
  const int32_t rows = (int32_t)rows64;
  const int32_t parts = parts_of(q, pl.cut_rows, pl.parts_rows);
  if (part >= parts) return;
  int64_t k0 = q.lo + (int64_t)part * pl.cut_rows;
  int64_t k1 = part + 1 < parts ? k0 + pl.cut_rows : q.hi;
  if (k1 > q.hi) k1 = q.hi;
  const int32_t tiles = k1 > k0 ? (int32_t)((k1 - k0 + 31) / 32) : 0;
  const int32_t each = (tiles + NW - 1) / NW;
  const int32_t t0 = wave * each < tiles ? wave * each : tiles;
  const int32_t nt = t0 + each < tiles ? each : tiles - t0;
  const int32_t kbase = (int32_t)k0 + t0 * 32;

  // this lane's row of each tile of rows: its token's position, or -1
  int32_t pos[RT];
  s16x8 qf[RT][KS];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int32_t row = rt * 16 + lane % 16;
    const int32_t tok = row / G, g = h * G + row % G;
    pos[rt] = row < rows ? q.start + tok : -1;
    const uint16_t* src = (const uint16_t*)a.q + (q.first + (row < rows ? tok : 0)) * a.q_token_stride +
                          (row < rows ? g : h * G) * a.q_head_stride + (lane / 16) * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      i32x4 x = *(const i32x4*)(src + ks * 32);
      if (pl.negative) x ^= (int)0x80008000;
      qf[rt][ks] = __builtin_bit_cast(s16x8, x);
    }
  }
  const float c = pl.c * (NARROW && p.k_scale ? p.k_scale[h] : 1.f);

  const int64_t es = NARROW ? 1 : 2;
  const int64_t page_b = p.page_stride * es, tok_b = p.token_stride * es;
  const char* kh = (const char*)p.k + h * p.head_stride * es;
  const char* vh = (const char*)p.v + h * p.head_stride * es;
  const uint32_t ring = lds_base() + wave * (NS * Sh::kStage);
  // this lane's source in a group of 16 keys, load by load
  constexpr int kPer16 = kLoads / 2;
  uint32_t koff[kPer16], voff[2][kPer16];
#pragma unroll
  for (int i = 0; i < kPer16; ++i) {
    const int row = i * kRowsPerLoad + lane / UPR;
    koff[i] = (uint32_t)(row * tok_b) + ((lane % UPR) ^ Sw::k(row)) * 16;
    voff[0][i] = (uint32_t)(row * tok_b) + ((lane % UPR) ^ Sw::v(row, NARROW)) * 16;
    voff[1][i] = (uint32_t)(row * tok_b) + ((lane % UPR) ^ Sw::v(row + 16, NARROW)) * 16;
  }
  const int32_t* blocks = a.block_table + r * a.row_stride;
  int32_t held = 0;
  auto issue = [&](int32_t t) {
    const uint32_t to = ring + (t % NS) * Sh::kStage;
    if ((t & 31) == 0) held = page_of(p, a, pl, blocks, (int64_t)kbase + (t + lane / 2) * 32 + (lane & 1) * 16);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int64_t page = __builtin_amdgcn_readlane(held, (t & 31) * 2 + half);
      const int64_t at = page * page_b + ((kbase + t * 32 + half * 16) & (p.page_size - 1)) * tok_b;
#pragma unroll
      for (int i = 0; i < kPer16; ++i)
        load_lds(to + half * 16 * RB + i * 1024, koff[i], kh + at);
#pragma unroll
      for (int i = 0; i < kPer16; ++i)
        load_lds(to + 32 * RB + half * 16 * RB + i * 1024, voff[half][i], vh + at);
    }
  };

  f32x4 acc[RT][DB];
  float m[RT], l[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m[rt] = -INFINITY;
    l[rt] = 0;
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[rt][d] = f32x4{0, 0, 0, 0};
  }
  // reads: K row lane % 16, its units lane / 16 + 4 ks; V four keys a 16-lane group, transposed
  const int grp = lane / 16, i16 = lane % 16;
  const uint32_t krow = i16 * RB;
  const uint32_t kx = NARROW ? ((grp / 2) ^ Sw::k(i16)) * 16 + (grp % 2) * 8 : (grp ^ Sw::k(i16)) * 16;
  const int vrow = NARROW ? ((i16 / 2) / 4) * 16 + 4 * grp + (i16 / 2) % 4 : 4 * grp + i16 / 4;
  const uint32_t vat = vrow * RB;
  const uint32_t vx = NARROW ? Sw::v(vrow, true) * 16 + (i16 % 2) * 8
                             : (((i16 % 4) / 2) ^ Sw::v(vrow, false)) * 16 + (i16 % 2) * 8;
  const int32_t pos_lo = q.start;   // the first row's; rows of -1 see nothing in any case
  const int32_t pos_hi = q.start + q.count - 1;

  auto tile = [&](int32_t t, auto masked) {
    constexpr bool kMasked = decltype(masked)::value;   // some row does not see all of it
    if (t + NS - 1 < nt) {
      issue(t + NS - 1);
      wait_loads<(NS - 1) * 2 * kLoads>();
    } else if (NS > 3 && t + NS - 2 < nt) {
      wait_loads<(NS > 2 ? NS - 2 : 0) * 2 * kLoads>();
    } else if (NS > 2 && t + NS - 3 < nt) {
      wait_loads<(NS > 3 ? NS - 3 : 0) * 2 * kLoads>();
    } else {
      wait_loads<0>();
    }
    const uint32_t kt = ring + (t % NS) * Sh::kStage, vt = kt + 32 * RB;
    f32x4 s[RT][2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) s[rt][kb] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        s16x8 f;
        if constexpr (NARROW)
          f = widen8<F16>(*LDS_PTR(i32x2, kt + kb * 16 * RB + krow + (kx ^ (ks * 32))));
        else
          f = *LDS_PTR(s16x8, kt + kb * 16 * RB + krow + (kx ^ (ks * 64)));
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) s[rt][kb] = mfma16<F16>(f, qf[rt][ks], s[rt][kb]);
      }
    }
    const int32_t key0 = kbase + t * 32 + 4 * grp;   // of s[.][0][0]; + 16 kb + i
    s16x8 pf[RT];
    uint32_t seen[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float x[8], w[8];
      seen[rt] = 0xff;
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = s[rt][j / 4][j % 4];
      if constexpr (kMasked) {
        seen[rt] = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int32_t key = key0 + (j / 4) * 16 + j % 4;
          const bool ok = sees(pos[rt], key, a.window) && key < k1;
          seen[rt] |= ok ? 1u << j : 0;
          if (!ok) x[j] = -INFINITY;
        }
      }
      float mx = x[0];
#pragma unroll
      for (int j = 1; j < 8; ++j) mx = fmaxf(mx, x[j]);
      mx = over_halves(over_rows(mx, Max()), Max());
      const bool grow = mx > m[rt] && (m[rt] == -INFINITY || (mx - m[rt]) * c > kLag<F16>);
      if (__any(grow)) {
        const float n = fmaxf(m[rt], mx);
        const float al = m[rt] == -INFINITY ? 0.f : exp2_((m[rt] - n) * c);
        l[rt] *= al;
#pragma unroll
        for (int d = 0; d < DB; ++d) acc[rt][d] *= al;
        m[rt] = n;
      }
      const float mc = top_of<F16>(m[rt], c);
      float sum = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        w[j] = exp2_(__builtin_fmaf(x[j], c, -mc));
        if (kMasked && !(seen[rt] >> j & 1)) w[j] = 0;
        sum += w[j];
      }
      l[rt] += sum;
      pf[rt] = pack8<F16>(w);
    }
    auto v_frag = [&](int db) -> s16x8 {
      if constexpr (NARROW) {
        return widen8<F16>(__builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(
            LDS_PTR(i32x2, vt + vat + (vx ^ (db * 16))))));
      } else {
        const uint32_t at = vt + vat + (vx ^ (db * 32));
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, at));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, at + 16 * RB));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      }
    };
    if constexpr (!kMasked) {
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const s16x8 f = v_frag(db);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) acc[rt][db] = mfma16<F16>(f, pf[rt], acc[rt][db]);
      }
    } else {
      uint32_t odd = 0;
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const s16x8 f = only_finite<F16>(v_frag(db), odd);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) acc[rt][db] = mfma16<F16>(f, pf[rt], acc[rt][db]);
      }
      if (__any(odd != 0)) {
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const s16x8 f = marks<F16>(v_frag(db));
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            const f32x4 n = mfma16<F16>(f, ones8<F16>(seen[rt]), f32x4{0, 0, 0, 0});
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[rt][db][i] = counted(acc[rt][db][i], n[i]);
          }
        }
      }
    }
    wait_lds();   // this stage's reads are done before its next load is issued
  };
  // tiles before `whole` start before the last row's window, those from `tail` on end past what the
  // first row sees or past the keys
  const Span3 sp = spans<32>(kbase, nt, pos_lo, pos_hi, (int32_t)k1, a.window);
  for (int32_t t = 0; t < NS - 1 && t < nt; ++t) issue(t);
  int32_t t = 0;
  for (int pass = 0; pass < 2; ++pass) {
    for (const int32_t e = pass ? nt : sp.whole; t < e; ++t) tile(t, std::true_type());
    if (pass == 0)
      for (; t < sp.tail; ++t) tile(t, std::false_type());
  }

  // the waves' parts of the rows are joined in LDS
  barrier();
  constexpr int R16 = 16 * RT;
  float* js = (float*)g_lds;                       // [NW][R16][kRow]
  float* jm = js + NW * R16 * Sh::kRow;            // [NW][R16]
  float* jl = jm + NW * R16;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float ls = over_halves(over_rows(l[rt], Sum()), Sum());
    const int row = rt * 16 + i16;
    if (grp == 0) {
      jm[wave * R16 + row] = m[rt];
      jl[wave * R16 + row] = ls;
    }
#pragma unroll
    for (int db = 0; db < DB; ++db)
      *(f32x4*)&js[(wave * R16 + row) * Sh::kRow + db * 16 + grp * 4] = acc[rt][db];
  }
  __syncthreads();
  const float vs = NARROW && p.v_scale ? p.v_scale[h] : 1.f;
  for (int i = threadIdx.x; i < rows * (D / 4); i += NW * kWave) {
    const int row = i / (D / 4), d = i % (D / 4) * 4;
    float mm = -INFINITY, ll = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) mm = fmaxf(mm, jm[w * R16 + row]);
    f32x4 o = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float mw = jm[w * R16 + row], lw = jl[w * R16 + row];
      if (lw == 0) continue;      // it saw nothing
      const float f = mw == mm ? 1.f : exp2_((mw - mm) * c);
      ll += f * lw;
      o += f * *(const f32x4*)&js[(w * R16 + row) * Sh::kRow + d];
    }
    const float inv = ll == 0 ? 0.f : vs / ll;
    o *= inv;
    const float lse = ll == 0 ? -INFINITY : mm * c + (__log2f(ll) - kLift<F16>);
    const int32_t tk = q.first + row / G, g = h * G + row % G;
    if (parts == 1) {
      store4<F16>(a, tk, g, d, o);
      if (a.lse && d == 0) a.lse[(int64_t)tk * a.q_heads + g] = lse / kLog2e;
    } else {
      const int64_t at = (((int64_t)part * a.requests + r) * p.heads + h) * pl.few + row;
      *(f32x4*)&pl.row_part[at * D + d] = o;
      if (d == 0) pl.row_lse[at] = lse;
    }
  }
}

// --------------------------------------------------------------- k_tiles ---

template <int RB>
struct TilesSwizzle {
  static constexpr int kUnits = RB / 16;
  static __device__ __forceinline__ int k(int row) { return row & (kUnits < 16 ? kUnits - 1 : 15); }
  static __device__ __forceinline__ int v(int row, bool narrow) {
    if (narrow) return kUnits >= 8 ? (row & 3) | ((row >> 1) & 4) : row & 3;
    return kUnits >= 16 ? (row & 3) * 4 + (row & 2) : (row & 3) * 2;
  }
};

template <bool NARROW, int D>
constexpr int kTilesLds = 2 * 2 * 64 * D * (NARROW ? 1 : 2);

// 128 rows of one request and key head, and one part of its keys, a block.  Bound by the matrix
// cores, the exponentials beside them and LDS, which at the matrix cores' full rate would give all it
// has, 128 bytes a clock: every wave reads the whole tile for its 32 rows.  4 x 2,048 new tokens behind
// 6,144 to 14,336 (32 heads, dim 128) take 1.04 to 1.12 ms from card to card, 0.95 to 1.03 PFLOP/s,
// matrix cores 58% busy (6% longer in f16); a product of 8,192 squared reaches 1.2 to 1.3.  Two blocks
// of four waves share a CU, so that one's loads and joins hide behind the other's products.
template <bool F16, bool NARROW, int D>
__global__ void __launch_bounds__(256, D == 256 ? 1 : 2)
k_tiles(pp_kv_pages p, pp_attention_args a, Plan pl) {
  constexpr int RB = D * (NARROW ? 1 : 2), UPR = RB / 16;
  using Sw = TilesSwizzle<RB>;
  constexpr int kLoads = 16 * RB / 1024, kRowsPerLoad = 1024 / RB;
  constexpr int DB = D / 32, KS = D / 16;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int h = blockIdx.x % p.heads;
  const int part = (blockIdx.x / p.heads) % pl.parts_tiles;
  const int32_t slot = blockIdx.x / p.heads / pl.parts_tiles;
  const int G = pl.group;
  int32_t r, first_slot;
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
    if (!at) return;
    r = __builtin_ctzll(at);
    first_slot = __builtin_amdgcn_readlane(base, r);
  } else {
    // request r's tiles start at slot floor(first token * G / 128) + r, which leaves it enough of them
    auto base_of = [&](int32_t i) {
      const int32_t t = a.query_start[i];
      return (int32_t)((int64_t)(t < 0 ? 0 : t < a.tokens ? t : a.tokens) * G / 128) + i;
    };
    r = find_last(a.requests, slot, base_of);
    if (r < 0) return;
    first_slot = base_of(r);
    if (first_slot > slot) return;
  }
  const Request q = request(a, pl, r);
  const int64_t rows = (int64_t)q.count * G;
  const int64_t row0 = (int64_t)(slot - first_slot) * 128;
  if (rows <= pl.few || row0 >= rows) return;
  const int32_t parts = parts_of(q, pl.cut_tiles, pl.parts_tiles);
  if (part >= parts) return;

  const int64_t row = row0 + wave * 32 + lane % 32;
  const bool live = row < rows;
  const int32_t tok = (int32_t)((live ? row : 0) / G), g = h * G + (int32_t)((live ? row : 0) % G);
  const int32_t pos = live ? q.start + tok : -1;
  const int half = lane / 32;

  // keys of this part that the tile's rows see
  const int32_t tok_lo = (int32_t)(row0 / G);
  const int64_t last = row0 + 127 < rows ? row0 + 127 : rows - 1;
  const int32_t pos_lo = q.start + tok_lo, pos_hi = q.start + (int32_t)(last / G);
  int64_t k0 = q.lo + (int64_t)part * pl.cut_tiles;
  int64_t k1 = part + 1 < parts ? k0 + pl.cut_tiles : q.hi;
  if (k1 > (int64_t)pos_hi + 1) k1 = (int64_t)pos_hi + 1;
  if (k1 > q.hi) k1 = q.hi;
  if (a.window && (int64_t)pos_lo - a.window + 1 > k0) k0 = (pos_lo - a.window + 1) & ~63;
  const int32_t nt = k1 > k0 ? (int32_t)((k1 - k0 + 63) / 64) : 0;
  const int32_t kbase = (int32_t)k0;

  s16x8 qf[KS];
  {
    const uint16_t* src = (const uint16_t*)a.q + (q.first + tok) * a.q_token_stride + g * a.q_head_stride + half * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      i32x4 x = *(const i32x4*)(src + ks * 16);
      if (pl.negative) x ^= (int)0x80008000;
      qf[ks] = __builtin_bit_cast(s16x8, x);
    }
  }
  const float c = pl.c * (NARROW && p.k_scale ? p.k_scale[h] : 1.f);

  const int64_t es = NARROW ? 1 : 2;
  const int64_t page_b = p.page_stride * es, tok_b = p.token_stride * es;
  const char* kh = (const char*)p.k + h * p.head_stride * es;
  const char* vh = (const char*)p.v + h * p.head_stride * es;
  constexpr uint32_t kTile = 64 * RB;
  const uint32_t lds = lds_base();
  // this lane's source in a group of 16 keys: row i * kRowsPerLoad + lane / UPR of load i, whose
  // swizzle is that of the two summands' together (both are linear over xor, and read no higher bit)
  const uint32_t off_row = (uint32_t)(lane / UPR * tok_b);
  const uint32_t off_k = ((lane % UPR) ^ Sw::k(lane / UPR)) * 16;
  const uint32_t off_v = ((lane % UPR) ^ Sw::v(lane / UPR, NARROW)) * 16;
  // wave w brings keys 16 w .. 16 w + 15 of a tile.  K and V have two buffers each and go their own
  // pace: V of a tile is brought with K of the same tile or of the next, from the same place in its pages.
  const int32_t* blocks = a.block_table + r * a.row_stride;
  const uint32_t tok32 = (uint32_t)tok_b;
  const Span3 sp = spans<64>(kbase, nt, pos_lo, pos_hi, (int32_t)k1, a.window);
  const int32_t flip = sp.whole & 1;                 // the pipeline below starts in buffer 0
  auto buffer = [&](int32_t t) { return (uint32_t)((t ^ flip) & 1) * kTile; };
  int32_t held = 0, next_k = 0, next_v = 0;
  int64_t place = 0;              // of tile next_v
  auto bring_k = [&](auto i, const char* from, uint32_t to) {
    load_lds_at<i * 1024>(to, off_row + (off_k ^ (Sw::k(i * kRowsPerLoad) * 16)), from + i * kRowsPerLoad * tok32);
  };
  auto bring_v = [&](auto i, const char* from, uint32_t to) {
    load_lds_at<i * 1024>(to, off_row + (off_v ^ (Sw::v(i * kRowsPerLoad, NARROW) * 16)), from + i * kRowsPerLoad * tok32);
  };
  const uint32_t own = __builtin_amdgcn_readfirstlane(lds + wave * 16 * RB);
  auto place_of = [&](int32_t t) {
    if ((t & 63) == 0) held = page_of(p, a, pl, blocks, (int64_t)kbase + (t + lane) * 64 + wave * 16);
    const uint32_t page = __builtin_amdgcn_readlane(held, t & 63);
    place = (int64_t)page * page_b + ((kbase + t * 64 + wave * 16) & (p.page_size - 1)) * tok32;
  };
  auto issue_k = [&] {
    const int32_t t = next_k++;
    if (t >= nt) return;
    place_of(t);
    each<kLoads>([&](auto i) { bring_k(i, kh + place, own + buffer(t)); });
  };
  auto issue_v = [&] {            // before issue_k moves on
    const int32_t t = next_v++;
    if (t >= nt) return;
    each<kLoads>([&](auto i) { bring_v(i, vh + place, own + 2 * kTile + buffer(t)); });
  };

  f32x16 acc[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[d][i] = 0;
  float m = -INFINITY, l = 0;

  const int l32 = lane % 32, i16 = lane % 16, dh = (lane / 16) % 2;
  const uint32_t krow = l32 * RB;
  const uint32_t kx = NARROW ? Sw::k(l32) * 16 + half * 8 : (half ^ Sw::k(l32)) * 16;
  const int vrow = NARROW ? ((i16 / 2) / 4) * 8 + 4 * half + (i16 / 2) % 4 : 4 * half + i16 / 4;
  const uint32_t vat = vrow * RB;
  const uint32_t vx = NARROW ? (dh ^ Sw::v(vrow, true)) * 16 + (i16 % 2) * 8
                             : ((dh * 2 + (i16 % 4) / 2) ^ Sw::v(vrow, false)) * 16 + (i16 % 2) * 8;

  // addresses of the fragments in the first tile; opaque, so that the pipeline's constant offsets go
  // into the instructions
  uint32_t k_lds[KS], v_lds[DB];
  each<KS>([&](auto i) {
    k_lds[i] = lds + krow + (kx ^ (i * (NARROW ? 16 : 32)));
    asm volatile("" : "+v"(k_lds[i]));
  });
  each<DB>([&](auto i) {
    v_lds[i] = lds + 2 * kTile + vat + (vx ^ (i * (NARROW ? 32 : 64)));
    asm volatile("" : "+v"(v_lds[i]));
  });
  auto k_frag = [&](uint32_t at, int ks) -> s16x8 {
    const auto* f = LDS_PTR(char, k_lds[ks]) + at;
    if constexpr (NARROW) return widen8<F16>(*(__attribute__((address_space(3))) i32x2*)f);
    else return *(__attribute__((address_space(3))) s16x8*)f;
  };
  // keys 8 (j / 4) + 4 half + j % 4 of 16, as the weights' registers have them
  auto v_frag = [&](uint32_t at, int db) -> s16x8 {
    auto* f = LDS_PTR(char, v_lds[db]) + at;
    if constexpr (NARROW) {
      return widen8<F16>(__builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(
          (__attribute__((address_space(3))) i32x2*)f)));
    } else {
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)f);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(f + 8 * RB));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  };
  auto scores = [&](uint32_t at) -> f32x16 {       // of 32 keys
    f32x16 x;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 0;
    each<KS>([&](auto ks) { x = mfma32<F16>(k_frag(at, ks), qf[ks], x); });
    return x;
  };
  auto largest = [&](const f32x16& x) {
    float mx = x[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, x[i]);
    return mx;
  };
  auto rescale = [&](float from, float to) {
    const float al = from == -INFINITY ? 0.f : exp2_((from - to) * c);
    l *= al;
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[d] *= al;
  };
  auto grows = [&](float mx) { return __any(mx > m && (m == -INFINITY || (mx - m) * c > kLag<F16>)); };

  // Half a tile that some row does not see whole.
  auto masked_half = [&](uint32_t at, int32_t key0) {
    f32x16 s = scores(at);
    uint32_t seen = 0;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const int32_t key = key0 + (j / 4) * 8 + j % 4;
      const bool ok = sees(pos, key, a.window) && key < k1;
      seen |= ok ? 1u << j : 0;
      if (!ok) s[j] = -INFINITY;
    }
    const float mx = over_halves(largest(s), Max());
    if (grows(mx)) {
      const float to = fmaxf(m, mx);
      rescale(m, to);
      m = to;
    }
    const float mc = top_of<F16>(m, c);
    float w[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      w[j] = (seen >> j & 1) ? exp2_(__builtin_fmaf(s[j], c, -mc)) : 0.f;
      l += w[j];
    }
    const s16x8 x[2] = {pack8<F16>(w), pack8<F16>(w + 8)};
    uint32_t odd = 0;
    each<2 * DB>([&](auto i) {
      acc[i / 2] = mfma32<F16>(only_finite<F16>(v_frag(at + i % 2 * 16 * RB, i / 2), odd), x[i % 2], acc[i / 2]);
    });
    if (__any(odd != 0)) {
      each<DB>([&](auto db) {
        f32x16 n;
#pragma unroll
        for (int i = 0; i < 16; ++i) n[i] = 0;
#pragma unroll 1
        for (int k = 0; k < 2; ++k)
          n = mfma32<F16>(marks<F16>(v_frag(at + k * 16 * RB, db)), ones8<F16>(seen >> (k * 8)), n);
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[db][i] = counted(acc[db][i], n[i]);
      });
    }
  };
  auto masked_tile = [&](int32_t t) {
    wait_loads<0>();
    barrier();                    // every wave's keys are there, and the other buffers are read
    if (next_k == t + 1) issue_k();
    issue_v();
#pragma unroll 1
    for (int b = 0; b < 2; ++b) masked_half(buffer(t) + b * 32 * RB, kbase + t * 64 + b * 32 + 4 * half);
  };

  // At dim 256 the pipeline below does not fit the registers, and a tile that every row sees whole goes
  // through in order: scores, weights, values.  4 x 2,048 new tokens behind up to 6,144: 1.47 ms (675
  // TFLOP/s), 6.18 ms with the pipeline and its spills; 512 behind 31,744 221 us and 1,010 us.
  // (Half a tile's scores beside the other half's weights, in that order: 1.57 ms.)
  [[maybe_unused]] auto whole_tile = [&](int32_t t) {
    wait_loads<0>();
    barrier();
    if (next_k == t + 1) issue_k();
    issue_v();
    const uint32_t at = buffer(t);
    const f32x16 s[2] = {scores(at), scores(at + 32 * RB)};
    const float mx = over_halves(fmaxf(largest(s[0]), largest(s[1])), Max());
    if (grows(mx)) {
      const float to = fmaxf(m, mx);
      rescale(m, to);
      m = to;
    }
    const float top = top_of<F16>(m, c);
    each<2>([&](auto b) {
      float w[16], sum = 0;
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        w[j] = exp2_(__builtin_fmaf(s[b][j], c, -top));
        sum += w[j];
      }
      l += sum;
      const s16x8 x[2] = {pack8<F16>(w), pack8<F16>(w + 8)};
      each<2 * DB>([&](auto i) {
        acc[i / 2] = mfma32<F16>(v_frag(at + b * 32 * RB + i % 2 * 16 * RB, i / 2), x[i % 2], acc[i / 2]);
      });
    });
  };

  // Tiles that every row sees whole go through a pipeline of 32 keys: while the weights of one half
  // tile are worked out, the matrix cores have the scores of the next and the values of the one
  // before.  (Without it the two took turns, although two waves share a SIMD.)
  // Its order is laid down by hand, one matrix instruction at a time with a sixteenth of the rest
  // beside it: left alone the compiler reads each fragment right before its use.
  f32x16 even, odds;              // scores of a tile's first and second half
  s16x8 pf[2];
  float mc = 0, old = 0;
  bool grow = false;              // of the scores that a step starts with
  auto peak = [&](float mx) {
    mx = over_halves(mx, Max());
    grow = grows(mx);
    old = m;
    m = grow ? fmaxf(m, mx) : m;
    mc = top_of<F16>(m, c);
  };
  constexpr int kAhead = 3;       // fragments read ahead of their use
  s16x8 pre[kAhead];              // the first ones of the next step, where no barrier comes before it
  constexpr std::integral_constant<int, 0> kFirst{};     // nothing before it yet
  constexpr std::integral_constant<int, 1> kTurn{};      // behind a barrier, with loads to issue
  constexpr std::integral_constant<int, 2> kSecond{};    // `pre` is there
  auto step = [&](const f32x16& cur, f32x16& next, uint32_t k_next, uint32_t v_last, auto kind, auto beside) {
    constexpr int kKind = decltype(kind)::value;
    constexpr int NV = kKind == 0 ? 0 : 2 * DB, NM = KS + NV;
    s16x8 f[NM], x[2];
    auto read = [&](auto at) {
      constexpr int i = decltype(at)::value;
      if constexpr (i < KS) f[i] = k_frag(k_next, i);
      else f[i] = v_frag(v_last + (i - KS) % 2 * 16 * RB, (i - KS) / 2);
    };
    float w[16], sum = 0, mx = -INFINITY;
    const float mc_now = mc, m_now = m, old_now = old;
    const bool grow_now = grow;
    f32x16 y;
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = 0;
    each<kAhead>([&](auto i) {
      if constexpr (kKind == 2) f[i] = pre[i];
      else read(i);
    });
    each<NM>([&](auto at) {
      constexpr int i = decltype(at)::value;
      if constexpr (i + kAhead < NM) read(std::integral_constant<int, i + kAhead>());
      else if constexpr (kKind == 1) pre[i + kAhead - NM] = k_frag(k_next + 32 * RB, i + kAhead - NM);
      if constexpr (i < KS) y = mfma32<F16>(f[i], qf[i], y);
      else acc[(i - KS) / 2] = mfma32<F16>(f[i], pf[(i - KS) % 2], acc[(i - KS) / 2]);
      beside(at);
#pragma unroll
      for (int j = i * 16 / NM; j < (i + 1) * 16 / NM; ++j) {
        w[j] = exp2_(__builtin_fmaf(cur[j], c, -mc_now));
        asm volatile("" : "+v"(w[j]));   // here, and not behind the branch at the end: so for the others
        sum += w[j];
      }
      asm volatile("" : "+v"(sum));
      if constexpr (i == NM / 2) {
        x[0] = pack8<F16>(w);
        asm volatile("" : "+v"(x[0]));
      }
      if constexpr (i >= KS && i < NM - 1) {
        constexpr int q = i - KS;     // the scores are there a little after their last instruction
#pragma unroll
        for (int j = q > 0 ? (q - 1) * 16 / (NV - 2) : 0; j < q * 16 / (NV - 2); ++j) mx = fmaxf(mx, y[j]);
        asm volatile("" : "+v"(mx));
        if constexpr (i == NM - 2) {
          peak(mx);
          asm volatile("" : "+v"(m), "+v"(mc));
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    });
    x[1] = pack8<F16>(w + 8);
    asm volatile("" : "+v"(x[1]));
    next = y;
    pf[0] = x[0];
    pf[1] = x[1];
    if (grow_now) rescale(old_now, m_now);
    l += sum;
    if constexpr (NV == 0) peak(largest(y));
  };

  issue_k();
  issue_v();
  int32_t t = 0;
  for (; t < sp.whole; ++t) masked_tile(t);
  const int32_t tail = t + ((sp.tail - t) & ~1);   // the loop takes two at a time
  if constexpr (D == 256) {
    for (; t < sp.tail; ++t) whole_tile(t);
  } else if (t < tail) {
    constexpr uint32_t kHalf = 32 * RB;
    wait_loads<0>();
    barrier();
    issue_k();
    even = scores(0);
    peak(largest(even));
    const auto nothing = [](auto) {};
    step(even, odds, kHalf, 0, kFirst, nothing);
    auto turn = [&](auto buf) {   // K of t + 1 and V of t are there; K of t and V of t - 1 are read
      constexpr uint32_t other = (1 - decltype(buf)::value) * kTile, same = decltype(buf)::value * kTile;
      wait_loads<0>();
      barrier();
      // V of t + 1 and K of t + 2, or some tile again where there are no more
      const char* vp = vh + place;
      place_of(next_k < nt ? next_k : nt - 1);
      const char* kp = kh + place;
      ++next_k;
      ++next_v;
      __builtin_amdgcn_s_setprio(1);   // over the other block's wave, until this one is ahead: 1.08 to 1.06 ms
      step(odds, even, other, same, kTurn, [&](auto i) {
        if constexpr (i < kLoads) bring_v(i, vp, own + 2 * kTile + other);
        else if constexpr (i < 2 * kLoads) bring_k(std::integral_constant<int, i - kLoads>(), kp, own + same);
      });
      __builtin_amdgcn_s_setprio(0);
      ++t;
    };
    for (;;) {
      turn(std::integral_constant<int, 0>());
      step(even, odds, kTile + kHalf, kHalf, kSecond, nothing);
      turn(std::integral_constant<int, 1>());
      if (t == tail) break;
      step(even, odds, kHalf, kTile + kHalf, kSecond, nothing);
    }
    m = old;                      // the scores past the last tile are nobody's
    each<2 * DB>([&](auto i) {
      acc[i / 2] = mfma32<F16>(v_frag(kTile + kHalf + i % 2 * 16 * RB, i / 2), pf[i % 2], acc[i / 2]);
    });
  }
  for (; t < nt; ++t) masked_tile(t);
  wait_loads<0>();                // the last loads of a tile that was there already

  l = over_halves(l, Sum());
  if (!live) return;
  const float vs = NARROW && p.v_scale ? p.v_scale[h] : 1.f;
  const float inv = vs / l;
  const float lse = l == 0 ? -INFINITY : m * c + (__log2f(l) - kLift<F16>);
  const int32_t tk = q.first + tok;
  const int64_t at = ((int64_t)part * a.tokens + tk) * a.q_heads + g;
  auto each4 = [&](auto put) {
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        f32x4 o = {acc[db][4 * b], acc[db][4 * b + 1], acc[db][4 * b + 2], acc[db][4 * b + 3]};
        // where l is 0 the products may still hold 0 times an infinity
        put(db * 32 + b * 8 + half * 4, l == 0 ? f32x4{0, 0, 0, 0} : o * inv);
      }
  };
  if (parts == 1) each4([&](int d, f32x4 o) { store4<F16>(a, tk, g, d, o); });
  else each4([&](int d, f32x4 o) { *(f32x4*)&pl.part[at * D + d] = o; });
  if (half == 0) {
    if (parts > 1) pl.part_lse[at] = lse;
    else if (a.lse) a.lse[(int64_t)tk * a.q_heads + g] = lse / kLog2e;
  }
}

// ---------------------------------------------------------------- k_join ---

// Rows of requests in several parts: a wave takes 256 / D of them, four values a lane.  Bound by the
// chain of its loads, so eight parts are read at a time, their log sums with them.
// few_rows: a wave's rows are some of few_rows rows of one of the key heads of a request of k_rows
// (where no request of k_tiles is in parts); 0: they are heads of one of the call's tokens.
template <bool F16, int D>
__global__ void __launch_bounds__(256) k_join(pp_attention_args a, Plan pl, int32_t few_rows, int32_t heads) {
  constexpr int kRows = 256 / D, kTurn = 8;
  const int lane = threadIdx.x % kWave, sub = lane / (D / 4), d = lane % (D / 4) * 4;
  const int64_t id = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  int32_t t, g, r, row, h;
  Request q;
  bool live, few;
  if (few_rows) {
    const int32_t each = (few_rows + kRows - 1) / kRows;
    if (id / each / heads >= a.requests) return;
    r = (int32_t)(id / each / heads);
    row = (int32_t)(id % each) * kRows + sub;
    h = (int32_t)(id / each % heads);
    q = request(a, pl, r);
    const int64_t rows = (int64_t)q.count * pl.group;
    if (rows > pl.few) return;
    few = true;
    live = row < few_rows && row < rows;
    t = q.first + row / pl.group;
    g = h * pl.group + row % pl.group;
  } else {
    const int32_t each = (a.q_heads + kRows - 1) / kRows;
    if (id / each >= a.tokens) return;
    t = (int32_t)(id / each);
    g = (int32_t)(id % each) * kRows + sub;
    live = g < a.q_heads;
    r = find_last(a.requests, t, [&](int32_t i) { return a.query_start[i]; });
    if (r < 0) return;
    q = request(a, pl, r);
    if (t < q.first || t >= q.first + q.count) return;
    few = (int64_t)q.count * pl.group <= pl.few;
    row = few ? (t - q.first) * pl.group + g % pl.group : 0;
    h = g / pl.group;
  }
  const int32_t parts = few ? parts_of(q, pl.cut_rows, pl.parts_rows) : parts_of(q, pl.cut_tiles, pl.parts_tiles);
  if (parts == 1 || !live) return;
  const int64_t at = (int64_t)t * a.q_heads + g;
  const int64_t own = few ? ((int64_t)r * heads + h) * pl.few + row : at;
  const int64_t step = few ? (int64_t)a.requests * heads * pl.few : (int64_t)a.tokens * a.q_heads;
  const float* from = (few ? pl.row_part : pl.part) + own * D + d;
  const float* sums = (few ? pl.row_lse : pl.part_lse) + own;
  float m = -INFINITY, sum = 0;
  f32x4 o = {0, 0, 0, 0};
  for (int32_t base = 0; base < parts; base += kTurn) {
    float x[kTurn];
    f32x4 y[kTurn];
#pragma unroll
    for (int j = 0; j < kTurn; ++j) {
      const int32_t i = base + j < parts ? base + j : parts - 1;
      x[j] = sums[i * step];
      y[j] = *(const f32x4*)(from + i * step * D);
    }
    float n = m;
#pragma unroll
    for (int j = 0; j < kTurn; ++j) n = fmaxf(n, x[j]);
    const float al = m == -INFINITY ? 0.f : exp2_(m - n);
    o *= al;
    sum *= al;
    m = n;
#pragma unroll
    for (int j = 0; j < kTurn; ++j) {
      if (base + j >= parts || x[j] == -INFINITY) continue;   // a part that saw nothing may hold anything
      const float w = x[j] == n ? 1.f : exp2_(x[j] - n);
      sum += w;
      o += w * y[j];
    }
  }
  o *= sum == 0 ? 0.f : 1.f / sum;
  store4<F16>(a, t, g, d, o);
  if (a.lse && d == 0) a.lse[at] = sum == 0 ? -INFINITY : (m + __log2f(sum)) / kLog2e;
}

// -------------------------------------------------------------- dispatch ---

// Blocks of k_tiles that the rule below counts on at a time.  At dim 256 its registers leave room for
// one a CU (100 new tokens behind 15,900 in 18 parts 61 us, counted as two a CU in 25 parts 90 us; 8 x 200
// behind up to 8,800 403 and 507 us; 3 x 700 the other way, 399 and 383).  At dim 64 three fit, but
// counted as three the calls are not faster: 512 behind 7,680 39 and 38 us, 4 x 700 behind up to 8,300 87
// and 103 us.
int tile_blocks(int32_t dim) { return dim == 256 ? 256 : 512; }

int64_t round_up(int64_t x, int32_t m) { return (x + m - 1) / m * m; }

struct Choice {
  int rt;                       // tiles of 16 rows in k_rows, 0 = not launched
  bool tiles, join;
};

// Every rule here goes by sizes the host knows, so the workspace is known before the call.
Choice choose(const pp_kv_pages& p, const pp_attention_args& a, Plan& pl) {
  Choice ch{};
  pl.group = a.q_heads / p.heads;
  pl.shift = __builtin_ctz(p.page_size);
  const int most = p.dim == 256 ? 32 : 64;      // rows k_rows has registers for
  const int64_t rows = (int64_t)a.max_new * pl.group;
  auto tiles16 = [](int64_t n) { return n <= 16 ? 1 : n <= 32 ? 2 : 4; };
  if (rows <= most) {
    ch.rt = tiles16(rows);
  } else {
    ch.tiles = true;
    // single tokens apart, unless every request has max_new tokens
    if (pl.group <= most && (int64_t)a.requests * a.max_new != a.tokens) ch.rt = tiles16(pl.group);
  }
  pl.few = ch.rt * 16;
  // keys that a request's rows see, at most; tokens past a row of the block table do not exist
  int64_t keys = (int64_t)a.max_blocks * p.page_size;
  if (a.max_len < keys) keys = a.max_len;
  if (keys < 1) keys = 1;
  if (a.window && (int64_t)a.window + a.max_new + 64 < keys) keys = (int64_t)a.window + a.max_new + 64;
  // n parts at most; the last one is open, so a size held to 31 bits loses no key
  auto cut = [&](int32_t n, int32_t unit, int32_t& size, int32_t& parts) {
    const int64_t x = round_up((keys + n - 1) / n, unit), most = INT32_MAX / 128 * 128;
    size = (int32_t)(x < most ? x : most);
    const int64_t count = (keys + size - 1) / size;
    parts = (int32_t)(count < n ? count : n);
  };
  cut(1, 128, pl.cut_rows, pl.parts_rows);
  cut(1, 128, pl.cut_tiles, pl.parts_tiles);
  if (ch.rt) {
    // As many parts as make 8,192 blocks (4,096 where requests times heads is 512 or more), but of 256 keys at
    // least, rounded up to a multiple of 128: where that decides, parts of 384 keys, or of 256 where keys
    // is a multiple of 256.  Lengths differ, so the fewer requests there are the smaller their parts have to be,
    // and in small parts a block's start and end and the join are most of it.  In parts of 128, 256, 384,
    // 512 and 1,024 keys 64 requests of up to 8,190 and 4 heads take 106, 90, 85, 90 and 104 us; one of
    // 16,000 and 2 heads in the first four 25, 18, 17 and 17 us, one of 4,097 13, 13, 13 and 15.  256
    // requests of up to 16,384 and 8 heads take 552 us whole, 555 in two parts (which the rule takes) and
    // 652 in four: a block that finds no keys still waits for its turn.
    const int64_t base = (int64_t)a.requests * p.heads;
    int64_t n = ((base < 512 ? 8192 : 4096) + base - 1) / base;
    if (n > keys / 256) n = keys / 256;
    cut((int32_t)(n > 1 ? n : 1), 128, pl.cut_rows, pl.parts_rows);
  }
  pl.slots = (int32_t)((int64_t)a.tokens * pl.group / 128) + a.requests;
  if (ch.tiles) {
    // as many parts as end soonest: rounds of resident blocks, each of its share of the tiles and some
    // four tiles' time to start and end, and the join's reading and writing of every part
    const double blocks = (double)a.tokens * pl.group / 128 * p.heads + 1, tiles = keys / 64.0;
    const double tile_us = 0.8 + 0.8 * p.dim / 128;
    const double part_us = (double)a.tokens * a.q_heads * p.dim * 8 / 4e6;
    double best = 0;
    int32_t n = 1;
    const double part_bytes = (double)a.tokens * a.q_heads * p.dim * 4;
    // 512 MiB of parts at most: calls beyond have so many blocks that cutting gains a percent or two
    for (int32_t i = 1; i <= 64 && (i == 1 || (tiles / i >= 8 && i * part_bytes <= 0x1p29)); ++i) {
      const double t = std::ceil(blocks * i / tile_blocks(p.dim)) * (tiles / i + 4) * tile_us + (i > 1 ? 4 + i * part_us : 0);
      if (i == 1 || t < best) {
        best = t;
        n = i;
      }
    }
    cut(n, 64, pl.cut_tiles, pl.parts_tiles);
  }
  ch.join = (ch.rt && pl.parts_rows > 1) || (ch.tiles && pl.parts_tiles > 1);
  return ch;
}

// Rows of the two regions of parts.
struct PartRows {
  int64_t tiles, rows;
};

PartRows part_rows(const pp_kv_pages& p, const pp_attention_args& a, const Plan& pl, const Choice& ch) {
  PartRows n{0, 0};
  if (ch.tiles && pl.parts_tiles > 1) n.tiles = (int64_t)pl.parts_tiles * a.tokens * a.q_heads;
  if (ch.rt && pl.parts_rows > 1) n.rows = (int64_t)pl.parts_rows * a.requests * p.heads * pl.few;
  return n;
}

template <class K>
hipError_t allow_lds(OnEachGpu& once, K kern, int bytes) {
  int gpu;
  const hipError_t e = hipGetDevice(&gpu);
  if (e != hipSuccess) return e;
  return once(gpu, [&] { return hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes); });
}

template <bool F16, bool NARROW, int D, int RT>
hipError_t go_rows(const pp_kv_pages& p, const pp_attention_args& a, const Plan& pl, hipStream_t st) {
  constexpr int lds = RowsShape<NARROW, D, RT>::kLds;
  static OnEachGpu once;
  const hipError_t ok = allow_lds(once, &k_rows<F16, NARROW, D, RT>, lds);
  if (ok != hipSuccess) return ok;
  const int64_t grid = (int64_t)a.requests * pl.parts_rows * p.heads;
  if (grid > INT32_MAX) return hipErrorInvalidConfiguration;
  k_rows<F16, NARROW, D, RT><<<(unsigned)grid, kWave * RowsShape<NARROW, D, RT>::kNW, lds, st>>>(p, a, pl);
  return hipGetLastError();
}

template <bool F16, bool NARROW, int D>
hipError_t go(const pp_kv_pages& p, const pp_attention_args& a, const Plan& pl, const Choice& ch, hipStream_t st) {
  if (ch.tiles) {
    constexpr int lds = kTilesLds<NARROW, D>;
    static OnEachGpu once;
    const hipError_t ok = allow_lds(once, &k_tiles<F16, NARROW, D>, lds);
    if (ok != hipSuccess) return ok;
    const int64_t grid = (int64_t)pl.slots * pl.parts_tiles * p.heads;
    if (grid > INT32_MAX) return hipErrorInvalidConfiguration;
    k_tiles<F16, NARROW, D><<<(unsigned)grid, 256, lds, st>>>(p, a, pl);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipError_t e = hipSuccess;
  if (ch.rt == 1) e = go_rows<F16, NARROW, D, 1>(p, a, pl, st);
  if (ch.rt == 2) e = go_rows<F16, NARROW, D, 2>(p, a, pl, st);
  if constexpr (D < 256)
    if (ch.rt == 4) e = go_rows<F16, NARROW, D, 4>(p, a, pl, st);
  if (e != hipSuccess) return e;
  if (ch.join) {
    constexpr int kRows = 256 / D;
    int64_t few_rows = 0, waves = (int64_t)a.tokens * ((a.q_heads + kRows - 1) / kRows);
    if (pl.parts_tiles == 1) {
      few_rows = (int64_t)a.max_new * pl.group < pl.few ? (int64_t)a.max_new * pl.group : pl.few;
      waves = (int64_t)a.requests * p.heads * ((few_rows + kRows - 1) / kRows);
    }
    k_join<F16, D><<<(unsigned)((waves + 3) / 4), 256, 0, st>>>(a, pl, (int32_t)few_rows, p.heads);
    e = hipGetLastError();
  }
  return e;
}

template <bool F16, bool NARROW>
hipError_t go_dim(const pp_kv_pages& p, const pp_attention_args& a, const Plan& pl, const Choice& ch, hipStream_t st) {
  if (p.dim == 64) return go<F16, NARROW, 64>(p, a, pl, ch, st);
  if (p.dim == 128) return go<F16, NARROW, 128>(p, a, pl, ch, st);
  return go<F16, NARROW, 256>(p, a, pl, ch, st);
}

}  // namespace

int64_t attention_workspace(const pp_kv_pages& p, const pp_attention_args& a) {
  Plan pl{};
  const Choice ch = choose(p, a, pl);
  const PartRows n = part_rows(p, a, pl, ch);
  return (n.tiles + n.rows) * (p.dim + 1) * 4;
}

hipError_t launch_attention(const pp_kv_pages& p, const pp_attention_args& a, hipStream_t st) {
  Plan pl{};
  const Choice ch = choose(p, a, pl);
  pl.negative = a.scale < 0;
  pl.c = (a.scale < 0 ? -a.scale : a.scale) * kLog2e;
  pl.part = (float*)a.workspace;
  const PartRows n = part_rows(p, a, pl, ch);
  pl.row_part = pl.part + n.tiles * p.dim;
  pl.part_lse = pl.row_part + n.rows * p.dim;
  pl.row_lse = pl.part_lse + n.tiles;
  const bool narrow = p.dtype == PP_E4M3;
  if (a.dtype == PP_F16) return narrow ? go_dim<true, true>(p, a, pl, ch, st) : go_dim<true, false>(p, a, pl, ch, st);
  return narrow ? go_dim<false, true>(p, a, pl, ch, st) : go_dim<false, false>(p, a, pl, ch, st);
}

}  // namespace pp

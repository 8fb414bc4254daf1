// pp_latent.hip -- attention of new tokens over pages of latent rows (gfx950).
//
// out = sum_j w_j C_j[0 .. C) / sum_j w_j, w_j = 2^(c s_j - c m), c = scale log2(e) k_scale, s = <q, C_j> over
// C + 64 elements: the scheme of pp_attend.hip (one pass with a running maximum, both products
// transposed, rows = token * heads + head) for rows that are key and value at once and that all query
// heads share.  A row of 1,152 bytes is brought into LDS once and read there twice: along the row for
// the scores, and transposed for the values.
//
// k_latent_rows takes requests of few rows (single tokens of 16 heads), which the reading of the pages
// bounds: its waves split the keys.  k_latent_tiles takes the others: 128 rows share a tile of keys;
// a wave has the scores of 32 rows, and then of all 128 rows the values of a quarter of the latent, so that the
// accumulators (128 x 512 floats, half the CU's registers) are there once.  Weights go from wave to wave
// through LDS.  Both cut the batch into equal shares for 256 blocks, and k_latent_join puts cut rows together.
//
// Weights are rounded to the queries' type for the second product, as in pp_attend.hip and for its reason; scores, sums
// and accumulators are 32 bits.  It costs less than a tenth of the output's own rounding (error against 64 bits 1.7e-3 in bf16
// and 2.1e-4 in f16, with it and without), but outputs near the middle of two values of their type go to the other one: they
// differ by 6e-4 to 1.2e-3 (f16 9e-5 to 1.8e-4) in all from those of weights in 32 bits.

#include "pp_attend.h"

#include <algorithm>

namespace pp {

namespace {

constexpr int kFew = 16;             // rows k_latent_rows takes
constexpr int kBlocks = 256;         // resident ones: one a CU
constexpr int kSlots = 1024;         // row tiles that k_latent_tiles cuts into equal shares, and requests
// What an item's start and end cost it, in tiles (stages of 16 or 32 keys, steps of 32), and the least that a block takes
// of them.  A start takes k_latent_rows some 11 us beside 1 us a tile of a wave, and k_latent_tiles 20 us beside 1.7 us a
// step.  With 4 and 8 (rows), 8 and 12 (tiles): 64 requests of 16 heads, 8 bits, 68.7 us where this takes 59.9, 48 requests of
// 128 heads 88.6 for 80.4, 512 short requests 78.4 for 65.3.
// A least share of 4 stages: lone requests of 4,097 and 16,384 keys 20.0 and 28.6 us, of 8 19.9 and 24.8 (fewer parts).
constexpr int kRowsStart = 16, kRowsShare = 8, kTilesStart = 16, kTilesShare = 8;
// Keys that requests of few rows may have beside prompts and still go with them through k_latent_tiles: 32 single tokens
// of 2,048 keys beside 512 new ones 89 us, with launches of their own 104; 16 of 16,384 361.7 for 360.5.
constexpr int kAlone = 131072;

// Rows that begin in block `block` and go on in the next ones up to `last`: `rows` of them from row `row` on of the
// request whose tokens begin at `first` (rows 0: none).
struct Cut {
  int32_t block, last, first, row, rows;
};

// A call's plan, and its parts in the workspace: [2 kBlocks][rows][C] (those of k_latent_tiles in its registers'
// order, part_at), their log sums, and the cuts.
struct Split : Plan {
  int32_t even;                      // k_latent_tiles cuts its slots
  int32_t by_slot;                   // its cuts are numbered by slots, which are fewer than blocks, else by the block they begin in
  float *slot_part, *slot_lse;
  Cut *row_cut, *slot_cut;
};

// Rows in LDS: the 16-byte unit u of a row lies at u ^ swizzle(row).  A row is 4.5 (16 bits, latent 512),
// 2.5 (256) or half of that many times 256 bytes, so neighbouring rows are already 128 (64) bytes apart in the
// banks, and the swizzle parts the rows that the transposing reads take together.
template <bool NARROW, int C>
struct Latent {
  static constexpr int kRB = (C + 64) * (NARROW ? 1 : 2);   // bytes of a row
  static constexpr int kUnits = kRB / 16;
  static constexpr int kKeys = NARROW ? 32 : 16;            // keys of a stage of k_latent_rows
  static constexpr int kStage = kKeys * kRB;
  static constexpr int kLoads = kStage / 1024;              // loads of 64 units
  static constexpr int kHalf = kLoads / 2;                  // those of kKeys / 2 keys
  static constexpr int kKS16 = (C + 64) / 32, kKS32 = (C + 64) / 16;   // steps of the scores
  static __device__ __forceinline__ int swizzle(int row) {
    return NARROW ? (row >> 2) & 3 : (row & 2) << 1 | (row & 4) >> 1 | (row & 8) >> 3;
  }
  // This lane's source of load i of kKeys / 2 rows from row `first` on (a multiple of that), in bytes from it.
  static __device__ __forceinline__ uint32_t source(int i, int lane, uint32_t tok_b, int first) {
    const int u = i * 64 + lane, row = u / kUnits;
    return row * tok_b + ((u % kUnits) ^ swizzle(row + first)) * 16;
  }
};

// What a row does not see does not touch it, whatever it holds.  In tiles that some row does not see whole, elements
// that are not finite are set to 0 in LDS between the scores and the values.  A row that sees one has a score of
// NaN or +infinity from it, and is NaN whole by its sum, or of -infinity, and then that element's weight of 0
// times an infinity makes it NaN: so mark_odd sets the row's element to NaN once it is stored.  In tiles seen whole
// the product itself does.  A row of which a wave or a block has seen nothing but scores of -infinity leaves 0 or such NaN
// there, which is added up with a factor of 0, so that where the batch is cut does not matter; the row is 0 only where that is
// all it has seen.
template <bool F16, bool NARROW>
__device__ __forceinline__ bool clean16(uint32_t at) {
  u32x4 x = *LDS_PTR(u32x4, at);
  uint32_t any = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (NARROW) {
      const uint32_t n = ((x[j] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
      any |= n;
      x[j] &= ~((n >> 7) * 0xffu);
    } else {
      const uint32_t n = not_finite<F16>(x[j]);
      any |= n;
      x[j] &= ~((n >> 15) * 0xffffu);
    }
  }
  if (any) *LDS_PTR(u32x4, at) = x;
  return any != 0;
}

// Whether some row sees a key of a tile that not all of them see: only such keys are odd, so that what lies behind the
// last token, or before a window, costs no time.
__device__ __forceinline__ bool seen_at_all(int32_t key, int32_t pos_lo, int32_t k1, int32_t window) {
  return (uint32_t)key < (uint32_t)k1 && (window == 0 || (int64_t)key > (int64_t)pos_lo - window);
}

// Rows row0 .. row0 + count - 1 of request r, keys k0 .. k1 - 1 of tiles of N, of which all rows see tiles sp.whole .. sp.tail - 1;
// sums: 0 for rows that stay as they are (of nothing but scores of -infinity, where that is known).
// `put` sets a row's element d to NaN.  All threads of the block, behind the rows' stores.  A walk over all of the keys took a batch
// of 64 requests of 16,001 keys and NaN behind each from 225 us to 5 ms.
template <bool F16, bool NARROW, int C, int N, class Put>
__device__ __forceinline__ void mark_odd(const pp_kv_pages& p, const pp_attention_args& a, const Plan& pl, int32_t r, int32_t start,
                                         int32_t row0, int32_t count, int32_t k0, int32_t k1, const Span3& sp, const float* sums, Put&& put) {
  const int32_t* blocks = a.block_table + r * a.row_stride;
  const int64_t es = NARROW ? 1 : 2;
#pragma unroll 1
  for (int32_t key = k0; key < k1; ++key) {
    const int32_t tile = (key - k0) / N;
    if (tile >= sp.whole && tile < sp.tail) {      // to the last key of the tiles seen whole
      key = k0 + (sp.tail * N - 1);
      continue;
    }
    const char* from = (const char*)p.k + page_of(p, a, pl, blocks, key) * p.page_stride * es +
                       (int64_t)(key & (p.page_size - 1)) * p.token_stride * es;
#pragma unroll 1
    for (int32_t d = threadIdx.x; d < C; d += 256) {
      uint32_t y;
      if constexpr (NARROW) y = (((const uint8_t*)from)[d] & 0x7f) == 0x7f;
      else y = not_finite<F16>(((const uint16_t*)from)[d]) & 0x8000u;
      if (!y) continue;
#pragma unroll 1
      for (int32_t i = 0; i < count; ++i)
        if (sees(start + (row0 + i) / pl.group, key, a.window) && sums[i] != 0) put(i, d);
    }
  }
}

// The last block of an item that begins in block b and whose costs end before `end`.  At most 255 are between them, so the
// quotient of floats is one off at most; a division of 64 bits takes a thousand cycles where its code is run once.
__device__ __forceinline__ int32_t last_block(int64_t end, int64_t share, int32_t b) {
  const int64_t behind = end - 1 - b * share;
  int32_t n = (int32_t)((float)behind / (float)share);
  if (n * share > behind) --n;
  if ((n + 1) * share <= behind) ++n;
  return b + n;
}

// What scores are multiplied by in the exponent: above 0 whatever the scales, so that -infinity times it is still that.
__device__ __forceinline__ float exponent_of(const Plan& pl, float k_scale) { return fmaxf(pl.c * k_scale, 0x1p-126f); }

// -------------------------------------------------------- k_latent_rows ---

template <bool NARROW, int C>
struct LatentRows : Latent<NARROW, C> {
  using L = Latent<NARROW, C>;
  static constexpr int kNW = 4;                             // waves
  static constexpr int kNS = C == 512 ? 2 : 3;              // stages of a wave's ring
  static constexpr int kRing = kNW * kNS * L::kStage;
  static constexpr int kRow = C + 4;                        // floats of a joined row
  static constexpr int kJoin = (kNW * 16 * (kRow + 3) + 16) * 4;
  static constexpr int kLds = kRing > kJoin ? kRing : kJoin;
};

template <bool F16>
__device__ __forceinline__ f32x4 mfma16x16(s16x4 a, s16x4 b, f32x4 c) {
  typedef __attribute__((__vector_size__(8))) _Float16 f16x4;
  if constexpr (F16)
    return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(f16x4, a), __builtin_bit_cast(f16x4, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a, b, c, 0, 0, 0);
}

// A value that all lanes have, where the compiler cannot know it.
__device__ __forceinline__ int64_t uniform(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)x >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}

// Sums over the 256 threads of a block: before this one, and of all.
__device__ __forceinline__ int64_t before(int64_t x, int64_t& all, int64_t* sums) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int64_t up = x;
  for (int o = 1; o < kWave; o <<= 1) {
    const int64_t y = __shfl_up(up, o);
    if (lane >= o) up += y;
  }
  __syncthreads();
  if (lane == kWave - 1) sums[wave] = up;
  __syncthreads();
  int64_t base = 0;
  all = 0;
  for (int w = 0; w < 4; ++w) {
    if (w < wave) base += sums[w];
    all += sums[w];
  }
  return base + up - x;
}

// All blocks together take the tiles of all items in order, `share` of the items' costs each.  An item at `at`
// in the row of costs has `start` for its start and end and then its tiles; block b has tiles from .. to - 1 of
// them (an item without tiles is whole in the block where it begins).  An item in several blocks leaves parts:
// that of its first block b is number 2 b + 1, the others 2 b, and a block has one of either at most.
struct Piece {
  int32_t from, to;
  bool here, first, last;
};

__device__ __forceinline__ Piece piece_of(int64_t at, int32_t start, int32_t tiles, int64_t share, int32_t b) {
  const int64_t lo = b * share - at - (tiles ? start : 0), hi = lo + share;
  Piece x;
  x.from = (int32_t)(lo > 0 ? lo : 0);
  x.to = (int32_t)(hi < tiles ? hi : tiles);
  x.first = lo <= 0;
  x.last = hi >= tiles;
  x.here = tiles ? x.from < x.to : lo <= 0 && hi > 0;
  return x;
}

// Requests of up to 16 rows.  All blocks together take the tiles of all requests in order, an equal share
// each, whatever the lengths: a block's share is of one request or of several.  Each wave has a ring of its own and
// keeps a stage in flight while it works on another, without a barrier.
// Bound by memory where there is much to read: 64 requests of 500 to 16,383 keys, 16 heads, 8 bits, 172 MB in 54 us, of
// which the finding of the first share takes 2.5, the queries and the first tiles 3.5 and the joining of the waves and
// the rows' stores 5; more keys go at 5.1 to 5.6 TB/s.  A lone request of 4,097 keys takes 15 us, 5 of them for two
// tiles a wave, the rest as before.
template <bool F16, bool NARROW, int C>
__global__ void __launch_bounds__(256, 1) k_latent_rows(pp_kv_pages p, pp_attention_args a, Split pl) {
  using Sh = LatentRows<NARROW, C>;
  constexpr int RB = Sh::kRB, NW = Sh::kNW, NS = Sh::kNS, KEYS = Sh::kKeys, KB = KEYS / 16;
  constexpr int DB = C / 16, KS = Sh::kKS16;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int grp = lane / 16, i16 = lane % 16, G = pl.group;
  if (threadIdx.x == 0) pl.row_cut[blockIdx.x].rows = 0;

  // what a request costs: its tiles and its start and end, nothing where it is not this kernel's
  struct Item {
    Request q;
    int32_t rows, tiles, cost;
  };
  auto item = [&](int32_t r) -> Item {
    Item x;
    x.q = request(a, pl, r);
    const int64_t rows = (int64_t)x.q.count * G;
    x.rows = rows <= kFew ? (int32_t)rows : 0;
    x.tiles = x.q.hi > x.q.lo ? (int32_t)(((int64_t)x.q.hi - x.q.lo + KEYS - 1) / KEYS) : 0;
    x.cost = x.rows ? x.tiles + kRowsStart : 0;
    return x;
  };
  int64_t share, at;
  int32_t r;
  {
    // thread i has requests i * each .. of them; the one whose costs hold the block's first looks it up
    int64_t* const sums = (int64_t*)g_lds;               // [4], then the block's first request and its place
    const int32_t each = (a.requests + 255) / 256, r0 = threadIdx.x * each;
    const int32_t r1 = r0 + each < a.requests ? r0 + each : a.requests;
    int64_t mine = 0, all;
    for (int32_t i = r0; i < r1; ++i) mine += item(i).cost;
    int64_t from = before(mine, all, sums);
    share = uniform((all + kBlocks - 1) / kBlocks);
    if (share < kRowsShare) share = kRowsShare;
    const int64_t x0 = blockIdx.x * share;
    if (x0 >= all) return;
    if (from <= x0 && x0 < from + mine) {
      int32_t i = r0;
      for (;; ++i) {
        const int32_t cost = item(i).cost;
        if (x0 < from + cost) break;
        from += cost;
      }
      sums[4] = i;
      sums[5] = from;
    }
    __syncthreads();
    r = __builtin_amdgcn_readfirstlane((int32_t)sums[4]);
    at = uniform(sums[5]);
  }

  const float vs = NARROW && p.k_scale ? p.k_scale[0] : 1.f;
  const float c = exponent_of(pl, vs);
  const int64_t es = NARROW ? 1 : 2;
  const int64_t page_b = p.page_stride * es;
  const uint32_t tok_b = (uint32_t)(p.token_stride * es);
  const char* rows_at = (const char*)p.k;
  const uint32_t ring = lds_base() + wave * (NS * Sh::kStage);
  uint32_t off[2][Sh::kHalf];
#pragma unroll
  for (int i = 0; i < Sh::kHalf; ++i) {
    off[0][i] = Sh::source(i, lane, tok_b, 0);
    off[1][i] = Sh::source(i, lane, tok_b, KEYS / 2);
  }
  // reads along a row: row i16, its units grp + 4 ks (16 bits) or grp / 2 + 2 ks; transposed ones: four
  // keys a 16-lane group, or eight.  The swizzle meets the steps' low bits only, the rest are offsets.
  const uint32_t kx = NARROW ? ((grp / 2) ^ Sh::swizzle(i16)) * 16 + (grp % 2) * 8 : (grp ^ Sh::swizzle(i16)) * 16;
  const int vrow = NARROW ? ((i16 / 2) / 4) * 16 + 4 * grp + (i16 / 2) % 4 : 4 * grp + i16 / 4;
  const uint32_t vx = NARROW ? Sh::swizzle(vrow) * 16 + (i16 % 2) * 8
                             : (((i16 % 4) / 2) ^ Sh::swizzle(vrow)) * 16 + (i16 % 2) * 8;
  uint32_t k_at[2], v_at[4];
#pragma unroll
  for (int i = 0; i < 2; ++i) k_at[i] = i16 * RB + (kx ^ (i * (NARROW ? 32 : 64)));
#pragma unroll
  for (int i = 0; i < 4; ++i) v_at[i] = vrow * RB + (vx ^ (i * (NARROW ? 16 : 32)));

#pragma unroll 1
  for (; r < a.requests && at < (blockIdx.x + 1) * share; ++r) {
    const Item x = item(r);
    const Request q = x.q;
    const int32_t rows = x.rows;
    const int64_t place = at;
    at += x.cost;
    const int32_t b = blockIdx.x;
    const Piece piece = piece_of(place, kRowsStart, x.tiles, share, b);
    if (!rows || !piece.here) continue;
    const bool parts = !piece.first || !piece.last;
    const int64_t to = 2 * b + piece.first;
    if (piece.first && parts && threadIdx.x == 0)
      pl.row_cut[b] = {b, last_block(place + x.cost, share, b), q.first, 0, rows};
    const int32_t k0 = q.lo + piece.from * KEYS;
    const int64_t end = (int64_t)q.lo + (int64_t)piece.to * KEYS;
    const int32_t k1 = end < q.hi ? (int32_t)end : q.hi;
    const int32_t tiles = piece.to - piece.from;
    const int32_t share_w = (tiles + NW - 1) / NW;
    const int32_t t0 = wave * share_w < tiles ? wave * share_w : tiles;
    const int32_t nt = t0 + share_w < tiles ? share_w : tiles - t0;
    const int32_t kbase = k0 + t0 * KEYS;
    const int32_t* blocks = a.block_table + r * a.row_stride;
    int32_t held = 0;
    auto issue = [&](int32_t t) {
      const uint32_t into = __builtin_amdgcn_readfirstlane(ring + (t % NS) * Sh::kStage);
      if ((t * KB & 63) == 0) held = page_of(p, a, pl, blocks, (int64_t)kbase + ((int64_t)t * KB + lane) * 16);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int32_t key = kbase + t * KEYS + half * (KEYS / 2);
        const int64_t page = __builtin_amdgcn_readlane(held, (t * KB + (KB - 1) * half) & 63);
        const char* from = rows_at + page * page_b + (int64_t)(key & (p.page_size - 1)) * tok_b;
        each<Sh::kHalf>([&](auto i) { load_lds(into + (half * Sh::kHalf + i) * 1024, off[half][i], from); });
      }
    };
    __syncthreads();                  // the ring was the last piece's join
    for (int32_t t = 0; t < NS - 1 && t < nt; ++t) issue(t);

    // this lane's row: its token's position, or -1
    const bool live = i16 < rows;
    const int32_t pos = live ? q.start + i16 / G : -1;
    s16x8 qf[KS];
    {
      const uint16_t* src = (const uint16_t*)a.q + (q.first + (live ? i16 / G : 0)) * a.q_token_stride +
                            (live ? i16 % G : 0) * a.q_head_stride + grp * 8;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        i32x4 y = *(const i32x4*)(src + ks * 32);
        y ^= pl.negative;
        qf[ks] = __builtin_bit_cast(s16x8, y);
      }
    }
    f32x4 acc[DB];
    float m = -INFINITY, l = 0;
    s16x8 nothing = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int d = 0; d < DB; ++d) {
      asm volatile("" : "+v"(nothing));     // cleared one by one, not copied
      acc[d] = mfma16<F16>(nothing, nothing, f32x4{0, 0, 0, 0});
    }
    const int32_t pos_lo = q.start;   // the first row's; rows of -1 see nothing in any case
    const int32_t pos_hi = q.start + q.count - 1;

    const Span3 sp = spans<KEYS>(kbase, nt, pos_lo, pos_hi, k1, a.window);
    bool odd = false;
    // One body for all tiles: a launch runs through little more than this once, and fetching code took
    // longer than its products (with a body each for tiles seen whole and in part a lone short request
    // took 16 us).
#pragma unroll 1
    for (int32_t t = 0; t < nt; ++t) {
      const bool masked = t < sp.whole || t >= sp.tail;   // some row does not see all of it
      if (t + NS - 1 < nt) {
        issue(t + NS - 1);
        wait_loads<(NS - 1) * Sh::kLoads>();
      } else if (NS > 2 && t + NS - 2 < nt) {
        wait_loads<(NS > 2 ? NS - 2 : 0) * Sh::kLoads>();
      } else {
        wait_loads<0>();
      }
      const uint32_t in = ring + (t % NS) * Sh::kStage;
      f32x4 s[KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        s[kb] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          s16x8 f;
          const uint32_t from = in + kb * 16 * RB + k_at[ks % 2] + ks / 2 * (NARROW ? 64 : 128);
          if constexpr (NARROW) f = widen8<F16>(*LDS_PTR(i32x2, from));
          else f = *LDS_PTR(s16x8, from);
          s[kb] = mfma16<F16>(f, qf[ks], s[kb]);
        }
      }
      float y[4 * KB], w[8];
#pragma unroll
      for (int j = 0; j < 4 * KB; ++j) y[j] = s[j / 4][j % 4];
      if (masked) {
        const int32_t key0 = kbase + t * KEYS + 4 * grp;   // of s[0][0]; + 16 kb + i
#pragma unroll
        for (int j = 0; j < 4 * KB; ++j) {
          const int32_t key = key0 + (j / 4) * 16 + j % 4;
          if (!(sees(pos, key, a.window) && (uint32_t)key < (uint32_t)k1)) y[j] = -INFINITY;
        }
        wait_lds();
#pragma unroll 1
        for (int i = lane; i < KEYS * (C * (int)es / 16); i += kWave) {
          const int row = i / (C * (int)es / 16);
          odd |= clean16<F16, NARROW>(in + row * RB + i % (C * (int)es / 16) * 16) &&
                 seen_at_all(kbase + t * KEYS + row, pos_lo, k1, a.window);
        }
        wait_lds();
      }
      float mx = y[0];
#pragma unroll
      for (int j = 1; j < 4 * KB; ++j) mx = fmaxf(mx, y[j]);
      mx = over_halves(over_rows(mx, Max()), Max());
      const bool grow = mx > m && (m == -INFINITY || (mx - m) * c > kLag<F16>);
      if (__any(grow)) {
        const float n = fmaxf(m, mx);
        const float al = m == -INFINITY ? 0.f : exp2_((m - n) * c);
        l *= al;
        if (__any(m != -INFINITY)) {      // else there is nothing yet
#pragma unroll
          for (int d = 0; d < DB; ++d) acc[d] *= al;
        }
        m = n;
      }
      const float mc = top_of<F16>(m, c);
      float sum = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        w[j] = j < 4 * KB ? exp2_(__builtin_fmaf(y[j < 4 * KB ? j : 0], c, -mc)) : 0.f;
        sum += w[j];
      }
      l += sum;
      const s16x8 pf = pack8<F16>(w);                    // of 16 keys: its first half
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        if constexpr (NARROW) {
          acc[db] = mfma16<F16>(widen8<F16>(__builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                                    LDS_PTR(i32x2, in + v_at[db % 4] + db / 4 * 64)))), pf, acc[db]);
        } else {
          acc[db] = mfma16x16<F16>(__builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, in + v_at[db % 4] + db / 4 * 128)),
                                   __builtin_shufflevector(pf, pf, 0, 1, 2, 3), acc[db]);
        }
      }
      wait_lds();   // this stage's reads are done before its next load is issued
    }

    // the waves' parts of the rows are joined in LDS
    float* js = (float*)g_lds;                       // [NW][16][kRow]
    float* jm = js + NW * 16 * Sh::kRow;             // [NW][16]
    float* jl = jm + NW * 16;
    const int any_odd = __syncthreads_or(odd);
    const float ls = over_halves(over_rows(l, Sum()), Sum());
    if (grp == 0) {
      jm[wave * 16 + i16] = m;
      jl[wave * 16 + i16] = ls;
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) *(f32x4*)&js[(wave * 16 + i16) * Sh::kRow + db * 16 + grp * 4] = acc[db];
    __syncthreads();
    // a factor for each wave's part of each row, 0 where it saw nothing, and the rows' sums
    float* const jf = jl + NW * 16;                  // [16][NW]
    float* const jt = jf + NW * 16;                  // [16]
    if (threadIdx.x < NW * 16) {
      const int w = threadIdx.x / 16, row = i16;
      float mm = -INFINITY, ll = 0;
#pragma unroll
      for (int v = 0; v < NW; ++v) mm = fmaxf(mm, jm[v * 16 + row]);
#pragma unroll
      for (int v = 0; v < NW; ++v) {
        const float mv = jm[v * 16 + row], lv = jl[v * 16 + row];
        if (lv != 0) ll += (mv == mm ? 1.f : exp2_((mv - mm) * c)) * lv;
      }
      const float mw = jm[w * 16 + row];
      jf[row * NW + w] = jl[w * 16 + row] == 0 ? 0.f : (mw == mm ? 1.f : exp2_((mw - mm) * c)) * (vs / ll);
      if (w == 0) jt[row] = parts ? 1.f : ll;        // what is 0 in a part need not be 0
      if (w == 0 && row < rows) {
        const float lse = ll == 0 ? -INFINITY : mm * c + (__log2f(ll) - kLift<F16>);
        if (parts) pl.row_lse[to * kFew + row] = lse;
        else if (a.lse) a.lse[(int64_t)(q.first + row / G) * a.q_heads + row % G] = lse / kLog2e;
      }
    }
    __syncthreads();
#pragma unroll 4
    for (int i = threadIdx.x; i < rows * (C / 4); i += NW * kWave) {
      const int row = i / (C / 4), d = i % (C / 4) * 4;
      const f32x4 f = *(const f32x4*)&jf[row * NW];
      f32x4 o = {0, 0, 0, 0};
#pragma unroll
      for (int w = 0; w < NW; ++w) o += f[w] * *(const f32x4*)&js[(w * 16 + row) * Sh::kRow + d];
      if (jt[row] == 0) o = f32x4{0, 0, 0, 0};
      if (parts) *(f32x4*)&pl.row_part[(to * kFew + row) * C + d] = o;
      else store4<F16>(a, q.first + row / G, row % G, d, o);
    }
    if (!any_odd) continue;
    __threadfence_block();
    __syncthreads();
    const Span3 all = spans<KEYS>(k0, tiles, pos_lo, pos_hi, k1, a.window);
    mark_odd<F16, NARROW, C, KEYS>(p, a, pl, r, q.start, 0, rows, k0, k1, all, jt, [&](int32_t i, int32_t d) {
      if (parts) pl.row_part[(to * kFew + i) * C + d] = __builtin_nanf("");
      else ((uint16_t*)a.out)[(q.first + i / G) * a.out_token_stride + i % G * a.out_head_stride + d] = F16 ? 0x7e00 : 0x7fc0;
    });
  }
}

// ------------------------------------------------------- k_latent_tiles ---

template <bool NARROW, int C>
struct LatentTiles : Latent<NARROW, C> {
  using L = Latent<NARROW, C>;
  static constexpr int kTile = 2 * L::kStage;               // 32 keys, or 64 in 8 bits
  static constexpr int kKeysTile = 2 * L::kKeys, kSubs = kKeysTile / 32;
  static constexpr int kNB = 3;                             // tiles in LDS
  static constexpr int kWeights = 4 * 2 * 1024;             // of 128 rows and 32 keys, as the products take them
  static constexpr int kOffsets = kNB * kTile + 2 * kWeights + 2 * 128 * 4 + 2 * 16;
  static constexpr int kTables = kOffsets + 2 * ((L::kHalf + 3) / 4) * 1024;   // of the even split
  static constexpr int kLds = kTables + kSlots * 16;
};

// x += a b (x = a b where FIRST) with x in vector registers: left alone the compiler keeps what matrix
// instructions write in accumulation registers, and the accumulators of 128 x 128 values take all 256 of
// a wave.  It cannot see the instruction's timing either: s_nop 1 covers operands that the vector unit wrote
// just before, and whoever reads x waits with settle() first.
template <bool F16, bool FIRST>
__device__ __forceinline__ void mfma32_vector(f32x16& x, s16x8 a, s16x8 b) {
  if constexpr (FIRST) {
    if constexpr (F16) asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_f16 %0, %1, %2, 0" : "=&v"(x) : "v"(a), "v"(b));
    else asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(x) : "v"(a), "v"(b));
  } else {
    if constexpr (F16) asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+v"(x) : "v"(a), "v"(b));
    else asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(x) : "v"(a), "v"(b));
  }
}

// x may be read 12 wait states after the last instruction that wrote it: the number that the compiler leaves where it sees one.
__device__ __forceinline__ void settle(f32x16& x) { asm volatile("s_nop 11" : "+v"(x)); }

// Where element d of row `row` of part `part` lies: runs of 256 floats have eight elements of 32 rows, as the
// accumulators' registers do.
template <int C>
__device__ __forceinline__ int64_t part_at(int64_t part, int32_t row, int32_t d) {
  return (part * 128 + row / 32 * 32) * C + d / 8 * 256 + (d / 4 % 2) * 128 + row % 32 * 4 + d % 4;
}

// This lane's number, without a register that keeps it.
__device__ __forceinline__ int this_lane() {
  int x;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=&v"(x));
  return x;
}

// 128 rows of one request and one part of its keys a block: a key's row is read from memory once for 128 rows and
// its values once from LDS (its scores four times, once a wave), where two blocks of 64 rows would need twice of both.
// Bound by the matrix cores: prompts of 1,024 to 2,048 tokens of 16 heads behind up to 16,384 in f16 1,326 us, 1.05
// PFLOP/s with the join, all behind 16,384 in bf16 1.19 (a product of 8,192 squared: 1.17 and 1.20).  A step takes 3,750 cycles
// (f16 3,950, whose maxima are followed more closely), its products 2,176, at 2.2 GHz: products alone draw so much power that the
// clock goes down to 1.7 GHz.  Without the reads of keys 6% less, without the loads of tiles 8%, without exponentials 1%;
// products of scores and values in turn took as long.  8-bit rows are widened once for the scores and once for the values: 5,250
// cycles, 0.99 PFLOP/s.
template <bool F16, bool NARROW, int C>
__global__ void __launch_bounds__(256, 1) k_latent_tiles(pp_kv_pages p, pp_attention_args a, Split pl) {
  using Sh = LatentTiles<NARROW, C>;
  constexpr int RB = Sh::kRB, KS = Sh::kKS32, SUBS = Sh::kSubs, TK = Sh::kKeysTile, NB = Sh::kNB;
  constexpr int DB = C / 128;                               // blocks of 32 of a wave's quarter of the latent
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int G = pl.group;
  // Blocks go to the eight XCDs in turn.  32 neighbouring shares or slots are one's, since their rows are most often of one
  // request, whose keys its L2 then holds for all of them.
  const int32_t block = (blockIdx.x | 255) < gridDim.x ? (int32_t)((blockIdx.x & ~255u) | (blockIdx.x & 7) << 5 | (blockIdx.x & 255) >> 3)
                                                       : (int32_t)blockIdx.x;

  // keys that the 128 rows of a request from row0 on see (there are less than 2^31 rows in all)
  struct Item {
    int32_t pos_lo, pos_hi, k0, k1, tiles;
  };
  auto item = [&](int32_t start, int32_t rows, int32_t lo, int32_t hi, int32_t row0) -> Item {
    Item x;
    const int32_t last = row0 + 127 < rows ? row0 + 127 : rows - 1;
    x.pos_lo = start + row0 / G;
    x.pos_hi = start + last / G;
    x.k0 = lo;
    if (a.window && (int64_t)x.pos_lo - a.window + 1 > x.k0) x.k0 = (x.pos_lo - a.window + 1) & ~63;
    x.k1 = x.pos_hi < hi ? x.pos_hi + 1 : hi;
    x.tiles = x.k1 > x.k0 ? (int32_t)(((int64_t)x.k1 - x.k0 + TK - 1) / TK) : 0;
    return x;
  };
  // Few slots of 128 rows: all blocks together take the tiles of all slots in order, an equal share each.
  // places: where slots begin in the row of costs; owners: their requests and their first rows.
  struct Owner {
    int32_t r, row;
  };
  int64_t* const places = (int64_t*)(g_lds + Sh::kTables);
  Owner* const owners = (Owner*)(places + kSlots);
  int64_t share = 1;
  int32_t slot = block, slots = 0;
  constexpr int kStart = kTilesStart / SUBS;
  if (pl.even) {
    if (!pl.by_slot && threadIdx.x == 0) pl.slot_cut[block].rows = 0;
    int64_t* const sums = (int64_t*)g_lds;                      // in the ring, as are
    int32_t* const begins = (int32_t*)(g_lds + 64);            // [kSlots]: the request that begins at a slot
    i32x4* const requests = (i32x4*)(g_lds + 64 + 4 * kSlots); // [kSlots]
    const int32_t most = a.requests > pl.slots ? a.requests : pl.slots, each = (most + 255) / 256;
    const int32_t i0 = threadIdx.x * each;
    int64_t all, sum = 0;
#pragma unroll 1
    for (int32_t i = i0; i < i0 + each; ++i) {
      begins[i] = 0;
      if (i >= a.requests) continue;
      const Request q = request(a, pl, i);
      requests[i] = i32x4{q.start, q.count * G, q.lo, q.hi};
      sum += q.count * G > pl.few ? (q.count * G + 127) / 128 : 0;
    }
    int32_t from = (int32_t)before(sum, all, sums);
    // requests that overlap may have more slots than there can be, and than there is room for: those are left out
    slots = (int32_t)uniform(all < pl.slots ? all : pl.slots);
    if (pl.by_slot && block == 0)       // the others are written where they begin
      for (int32_t i = slots + threadIdx.x; i < pl.slots; i += 256) pl.slot_cut[i].rows = 0;
#pragma unroll 1
    for (int32_t i = i0; i < i0 + each && i < a.requests; ++i) {
      const int32_t rows = requests[i][1];
      if (rows <= pl.few) continue;
      if (from < slots) begins[from] = i;
      owners[i].row = from;            // for now: the request's first slot
      from += (rows + 127) / 128;
    }
    __syncthreads();
    // the last request that begins at or before a slot
    int32_t last = 0;
    for (int32_t i = i0; i < i0 + each; ++i) last = begins[i] > last ? begins[i] : last;
    int32_t up = last;
    for (int o = 1; o < kWave; o <<= 1) {
      const int32_t y = __shfl_up(up, o);
      if (lane >= o && y > up) up = y;
    }
    if (lane == kWave - 1) ((int32_t*)sums)[8 + wave] = up;
    up = __shfl_up(up, 1);
    if (lane == 0) up = 0;
    __syncthreads();
    for (int w = 0; w < wave; ++w) {
      const int32_t y = ((int32_t*)sums)[8 + w];
      up = y > up ? y : up;
    }
    sum = 0;
    Owner mine[kSlots / 256];
    int32_t cost[kSlots / 256];
#pragma unroll
    for (int e = 0; e < kSlots / 256; ++e) {
      const int32_t i = i0 + e;
      if (e >= each || i >= slots) continue;
      up = begins[i] > up ? begins[i] : up;
      const i32x4 q = requests[up];
      mine[e] = {up, (i - owners[up].row) * 128};
      cost[e] = item(q[0], q[1], q[2], q[3], mine[e].row).tiles + kStart;
      sum += cost[e];
    }
    int64_t at = before(sum, all, sums);       // and every first slot is read
#pragma unroll
    for (int e = 0; e < kSlots / 256; ++e) {
      const int32_t i = i0 + e;
      if (e >= each || i >= slots) continue;
      places[i] = at;
      owners[i] = mine[e];
      at += cost[e];
    }
    __syncthreads();
    share = uniform((all + kBlocks - 1) / kBlocks);
    if (share < kTilesShare / SUBS) share = kTilesShare / SUBS;
    const int64_t x0 = block * share;
    if (x0 >= all) return;
    int32_t lo = 0, hi = slots - 1;         // the last slot at or before x0
    while (lo < hi) {
      const int32_t mid = (lo + hi + 1) / 2;
      if (places[mid] <= x0) lo = mid;
      else hi = mid - 1;
    }
    slot = __builtin_amdgcn_readfirstlane(lo);
  }

  const int half = lane / 32, l32 = lane % 32, i16 = lane % 16, dh = (lane / 16) % 2;
  // A block's first slot, of which it may have the end only, comes last: so the blocks begin with the first keys of
  // their requests together, and find in L2 what the others have read.
  int32_t left = -1;
  if (pl.even && slot + 1 < slots && places[slot] + kStart < block * share && places[slot + 1] < (block + 1) * share) left = slot++;
  left = __builtin_amdgcn_readfirstlane(left);
#pragma unroll 1
  for (bool more_slots = true; more_slots; ++slot) {
  int32_t r, row0;
  int64_t place = 0;
  if (pl.even) {
    if (slot >= slots || uniform(places[slot]) >= (block + 1) * share) {
      if (left < 0) return;
      slot = left;
      more_slots = false;
    }
    place = uniform(places[slot]);
    r = __builtin_amdgcn_readfirstlane(owners[slot].r);
    row0 = __builtin_amdgcn_readfirstlane(owners[slot].row);
  } else {
    more_slots = false;
    const Slot s = slot_of(a, pl, slot);
    r = s.r;
    if (r < 0 || (int64_t)(slot - s.first) * 128 >= (int64_t)a.tokens * G) return;
    row0 = (slot - s.first) * 128;
  }
  const Request q = request(a, pl, r);
  const int32_t rows = q.count * G;
  if (!pl.even && (rows <= pl.few || row0 >= rows)) return;
  const Item x = item(q.start, rows, q.lo, q.hi, row0);
  int32_t k0 = x.k0, k1 = x.k1;
  bool parts = false, cuts = false;
  int64_t to = 0;
  const int32_t count = rows - row0 < 128 ? rows - row0 : 128;
  if (pl.even) {
    const int32_t b = block;
    const Piece piece = piece_of(place, kStart, x.tiles, share, b);
    if (!piece.here) continue;
    const int64_t end = (int64_t)k0 + (int64_t)piece.to * TK;
    if (end < k1) k1 = (int32_t)end;
    k0 += piece.from * TK;
    parts = !piece.first || !piece.last;
    to = 2 * b + piece.first;
    cuts = piece.first && (parts || pl.by_slot);
  }
  k0 = __builtin_amdgcn_readfirstlane(k0);
  k1 = __builtin_amdgcn_readfirstlane(k1);
  const int32_t nt = k1 > k0 ? (int32_t)(((int64_t)k1 - k0 + TK - 1) / TK) : 0;
  const int32_t kbase = k0, pos_lo = x.pos_lo, pos_hi = x.pos_hi;
  const int32_t row = row0 + wave * 32 + l32;
  const bool live = row < rows;
  const int32_t tok = (live ? row : 0) / G, g = (live ? row : 0) % G;
  const int32_t pos = live ? q.start + tok : -1;
  barrier();                          // the last piece's sums are read

  const float vs = NARROW && p.k_scale ? p.k_scale[0] : 1.f;
  const float c = exponent_of(pl, vs);

  const int64_t es = NARROW ? 1 : 2;
  const int64_t page_b = p.page_stride * es;
  const uint32_t tok_b = (uint32_t)(p.token_stride * es);
  const uint32_t lds = lds_base(), weights = lds + NB * Sh::kTile, offsets = lds + Sh::kOffsets;
  float* const alphas = (float*)(g_lds + NB * Sh::kTile + 2 * Sh::kWeights);     // [2][128]
  int32_t* const grown = (int32_t*)(alphas + 2 * 128);                          // [2][4]
  // wave w brings a quarter of a tile's keys
  constexpr int kMine = TK / 4;
  const uint32_t own = __builtin_amdgcn_readfirstlane(lds + wave * kMine * RB);
  const int32_t* blocks = a.block_table + r * a.row_stride;
  int32_t held = nt ? page_of(p, a, pl, blocks, (int64_t)kbase + (int64_t)lane * TK + wave * kMine) : 0;   // of 64 tiles
  // where tile t comes from and goes to, or the last one again where there are no more
  struct Move {
    const char* from;
    uint32_t to;
  };
  auto move_of = [&](int32_t t) -> Move {
    const uint32_t to = own + t % NB * Sh::kTile;
    if (t && t < nt && (t & 63) == 0) held = page_of(p, a, pl, blocks, (int64_t)kbase + (int64_t)(t + lane) * TK + wave * kMine);
    if (t >= nt) t = nt - 1;
    const int64_t page = __builtin_amdgcn_readlane(held, t & 63);
    const char* from = (const char*)p.k + page * page_b + (int64_t)((kbase + t * TK + wave * kMine) & (p.page_size - 1)) * tok_b;
    return {(const char*)uniform((int64_t)from), (uint32_t)__builtin_amdgcn_readfirstlane(to)};
  };
  // this lane's sources wait in LDS: registers are short
  constexpr int kTable = (Sh::kHalf + 3) / 4 * 1024;         // rows 0 .. and 8 .. of 16 lie differently
  uint32_t my_offsets = offsets + wave % 2 * kTable + lane * 16;
  asm volatile("" : "+v"(my_offsets));
  auto sources = [&](auto i) {
    uint32_t x = my_offsets;
    asm volatile("" : "+v"(x));       // one register, and i as an offset
    return *LDS_PTR(u32x4, x + i * 1024);
  };
  auto bring = [&](auto i, u32x4 off, const Move& x) { load_lds_at<i * 1024>(x.to, off[i % 4], x.from); };

  // The queries and the first tiles are on their way together, and what follows up to the first step beside them.
  s16x8 qf[KS];
  {
    const uint16_t* src = (const uint16_t*)a.q + (q.first + tok) * a.q_token_stride + g * a.q_head_stride + half * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *(const s16x8*)(src + ks * 16);
  }
  if (nt) {
    if (wave < 2)
      each<(Sh::kHalf + 3) / 4>([&](auto i) {
        u32x4 x;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = Sh::source(i * 4 + j, lane, tok_b, wave * kMine);
        *LDS_PTR(u32x4, my_offsets + i * 1024) = x;
      });
    barrier();
#pragma unroll 1
    for (int32_t t = 0; t < 2; ++t) {
      const Move x = move_of(t);
      each<Sh::kHalf>([&](auto i) { bring(i, sources(std::integral_constant<int, i / 4>()), x); });
    }
  }
  if (cuts && threadIdx.x == 0)
    pl.slot_cut[pl.by_slot ? slot : block] = {block, last_block(place + x.tiles + kStart, share, block), q.first, row0, parts ? count : 0};

  // cleared by the matrix cores: 16 instructions instead of 256
  f32x16 acc[DB][4], zeros;
#pragma unroll
  for (int i = 0; i < 16; ++i) zeros[i] = 0;
  s16x8 nothing = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      asm volatile("" : "+v"(nothing));     // else the compiler clears one and copies it
      acc[d][e] = mfma32<F16>(nothing, nothing, zeros);
      if constexpr (C == 512) asm volatile("" : "+a"(acc[d][e]));
    }
  float m = -INFINITY, l = 0;

  // reads along a row: key l32, its units half + 2 ks (8 bits: the half of unit ks); transposed ones of
  // this wave's quarter
  const uint32_t kx = NARROW ? Sh::swizzle(l32) * 16 + half * 8 : (half ^ Sh::swizzle(l32)) * 16;
  const int vrow = NARROW ? ((i16 / 2) / 4) * 8 + 4 * half + (i16 / 2) % 4 : 4 * half + i16 / 4;
  const uint32_t vx = NARROW ? (dh ^ Sh::swizzle(vrow)) * 16 + (i16 % 2) * 8
                             : ((dh * 2 + (i16 % 4) / 2) ^ Sh::swizzle(vrow)) * 16 + (i16 % 2) * 8;
  // Rows and tiles begin at multiples of 128 bytes (64 of 8-bit rows), so the steps' low bits are exchanged in the whole address.
  static_assert(Sh::kTile % 128 == 0 && RB % (NARROW ? 64 : 128) == 0);
  uint32_t k_at = lds + l32 * RB + kx, v_at = lds + vrow * RB + vx + wave * (C * (int)es / 4);
  asm volatile("" : "+v"(k_at), "+v"(v_at));      // made for each slot: kept from one to the next they would go to memory
  auto k_frag = [&](uint32_t at, int ks) -> s16x8 {
    const uint32_t from = ((at + k_at) ^ (ks % 4 * (NARROW ? 16 : 32))) + ks / 4 * (NARROW ? 64 : 128);
    if constexpr (NARROW) return widen8<F16>(*LDS_PTR(i32x2, from));
    else return *LDS_PTR(s16x8, from);
  };
  // keys 8 (j / 4) + 4 half + j % 4 of 16, as the weights' registers have them
  auto v_frag = [&](uint32_t at, int db) -> s16x8 {
    const uint32_t from = (at + v_at) ^ (db % 2 * (NARROW ? 32 : 64));
    if constexpr (NARROW) {
      return widen8<F16>(__builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(LDS_PTR(i32x2, from + db / 2 * 64))));
    } else {                          // eight rows on the swizzle's lowest bit is another
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, from + db / 2 * 128));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, (from ^ 16) + 8 * RB + db / 2 * 128));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  };
  // Weights of rows 32 (i / 2) .., keys 16 (i % 2) .. lie at i * 1024 from where a buffer's begin for this lane.
  // The compiler is kept from a register for each i.
  uint32_t w_at = weights + lane * 16;
  asm volatile("" : "+v"(w_at));
  auto weights_of = [&](int b) -> uint32_t {
    uint32_t x = w_at + b * Sh::kWeights;
    asm volatile("" : "+v"(x));
    return x;
  };
  // The rows' maximum with that of 32 scores; where one grows too far, all waves have to know.
  auto peak = [&](float mx, int b) {
    mx = over_halves(mx, Max());
    const bool grows = __any(mx > m && (m == -INFINITY || (mx - m) * c > kLag<F16>));
    bool scaled = false;
    if (grows) {
      const float n = fmaxf(m, mx);
      const float al = m == -INFINITY ? 0.f : exp2_((m - n) * c);
      const int i = this_lane();
      if (i < 32) alphas[b * 128 + wave * 32 + i] = al;
      l *= al;
      scaled = __any(m != -INFINITY);     // else there is nothing yet
      m = n;
    }
    if (this_lane() == 0) grown[b * 4 + wave] = scaled;
  };
  auto rescale = [&](int b) {
    const i32x4 any = *(const i32x4*)&grown[b * 4];
    if (!__builtin_amdgcn_readfirstlane(any[0] | any[1] | any[2] | any[3])) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (!__builtin_amdgcn_readfirstlane(any[e])) continue;
      const float al = alphas[b * 128 + e * 32 + this_lane() % 32];
      each<DB>([&](auto d) {
        if constexpr (C == 512) asm volatile("" : "+a"(acc[d][e]));
        acc[d][e] *= al;
        if constexpr (C == 512) asm volatile("" : "+a"(acc[d][e]));
        __builtin_amdgcn_sched_barrier(0);
      });
    }
  };

  // Between a step's scores and its values, this wave's quarter of keys that some row does not see whole.
  constexpr int kQuarter = C / 4 * (NARROW ? 1 : 2) / 16;      // units
  bool odd = false;
  auto clean = [&](uint32_t at, int32_t key0) {
#pragma unroll 1
    for (int i = this_lane(); i < 32 * kQuarter; i += kWave) {
      const int row = i / kQuarter;
      odd |= clean16<F16, NARROW>(lds + at + row * RB + (wave * kQuarter + i % kQuarter) * 16) &&
             seen_at_all(key0 + row, pos_lo, k1, a.window);
    }
    wait_lds();
  };

  // The values of one step (at `cur`, weights in buffer b) and the scores and weights of the next.
  constexpr int kAhead = 2, NV = 2 * DB;
  auto step = [&](uint32_t cur, uint32_t next, int b, int32_t key0, uint32_t limit, bool masked, bool more,
                  const Move& tile) {
    rescale(b);
    s16x8 f[KS], w[8], v[NV];
    f32x16 y;
    u32x4 off[(Sh::kHalf + 3) / 4];
    auto read_v = [&](auto i) { v[i] = v_frag(cur + i / DB * 16 * RB, i % DB); };
    const uint32_t w_from = weights_of(b);
    auto read_w = [&](auto i) { w[i] = *LDS_PTR(s16x8, w_from + (i % 4 * 2 + i / 4) * 1024); };
    each<kAhead>([&](auto i) { f[i] = k_frag(next, i); });
    each<KS>([&](auto i) {
      if constexpr (i + kAhead < KS) f[i + kAhead] = k_frag(next, i + kAhead);
      if constexpr (i >= KS - 4) read_w(std::integral_constant<int, i - (KS - 4)>());
      if constexpr (i == KS - 2) read_v(std::integral_constant<int, 0>());
      mfma32_vector<F16, i == 0>(y, f[i], qf[i]);
      if constexpr (i % 8 == 0 && i / 8 < (Sh::kHalf + 3) / 4) off[i / 8] = sources(std::integral_constant<int, i / 8>());
      if constexpr (i >= 4 && i % 2 == 0 && i / 2 - 2 < Sh::kHalf)
        if (more) bring(std::integral_constant<int, i / 2 - 2>(), off[(i / 2 - 2) / 4], tile);
      __builtin_amdgcn_sched_barrier(0);
    });
    float mx = -INFINITY, mc = 0, sum = 0, x[16];
    uint32_t w_to = 0;
    constexpr int NM = NV * 4;
    each<NM>([&](auto at) {
      constexpr int i = decltype(at)::value, g = i / 4, e = i % 4;
      if constexpr (e == 0 && g + 1 < NV) read_v(std::integral_constant<int, g + 1>());
      acc[g % DB][e] = mfma32<F16>(v[g], w[g / DB * 4 + e], acc[g % DB][e]);
      if constexpr (g == DB - 1) read_w(std::integral_constant<int, 4 + e>());      // in place of the one just used
      // the next step's weights, a few instructions beside each product
      constexpr int kWait = 4, kMax = NM / 8, kPeak = kWait + kMax, kExp = kPeak + 1, kEnd = NM - NM / 8;
      if constexpr (i == kWait - 1) {
        settle(y);
        if (masked) {
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int32_t key = key0 + 4 * half + (j / 4) * 8 + j % 4;
            if (!(sees(pos, key, a.window) && (uint32_t)key < limit)) y[j] = -INFINITY;
          }
        }
      }
      if constexpr (i >= kWait && i < kPeak) {
#pragma unroll
        for (int j = (i - kWait) * 16 / kMax; j < (i - kWait + 1) * 16 / kMax; ++j) mx = fmaxf(mx, y[j]);
        asm volatile("" : "+v"(mx));
      }
      if constexpr (i == kPeak) {
        peak(mx, b ^ 1);
        mc = top_of<F16>(m, c);
        asm volatile("" : "+v"(mc));
      }
      if constexpr (i >= kExp && i < kEnd) {
#pragma unroll
        for (int j = (i - kExp) * 16 / (kEnd - kExp); j < (i + 1 - kExp) * 16 / (kEnd - kExp); ++j) {
          x[j] = exp2_(__builtin_fmaf(y[j], c, -mc));
          asm volatile("" : "+v"(x[j]));
          sum += x[j];
        }
        asm volatile("" : "+v"(sum));
      }
      if constexpr (i == kEnd) w_to = weights_of(b ^ 1) + wave * 2048;
      if constexpr (i == kEnd) *LDS_PTR(s16x8, w_to) = pack8<F16>(x);
      if constexpr (i == kEnd + 1) *LDS_PTR(s16x8, w_to + 1024) = pack8<F16>(x + 8);
      __builtin_amdgcn_sched_barrier(0);
    });
    l += sum;
  };

  // One barrier a step of 32 keys.  Before it the step's weights are written and the next step's keys
  // waited for; behind it every wave is past the values of the step before, whose tile is brought anew.
  // There is one body for all steps, since fetching code takes longer than running it: the first has the values of no
  // keys (zeros in the third tile and the second weights), the last the scores of keys that no row sees.
  const Span3 sp = spans<TK>(kbase, nt, pos_lo, pos_hi, k1, a.window);
#pragma unroll 1
  for (uint32_t i = threadIdx.x * 16; i < Sh::kTile; i += 4096) *LDS_PTR(i32x4, lds + 2 * Sh::kTile + i) = i32x4{0, 0, 0, 0};
#pragma unroll 1
  for (uint32_t i = threadIdx.x * 16; i < Sh::kWeights; i += 4096) *LDS_PTR(i32x4, weights + Sh::kWeights + i) = i32x4{0, 0, 0, 0};
  if (threadIdx.x < 4) grown[4 + threadIdx.x] = 0;
  __builtin_amdgcn_sched_barrier(0);
  if (pl.negative)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      i32x4 y = __builtin_bit_cast(i32x4, qf[ks]);
      y ^= pl.negative;
      qf[ks] = __builtin_bit_cast(s16x8, y);
    }
  wait_loads<0>();
  barrier();
  const int32_t steps = nt * SUBS, whole = sp.whole * SUBS, tail = sp.tail * SUBS;
  uint32_t cur = 2 * Sh::kTile;
#pragma unroll 1
  for (int32_t u = 0;; ++u) {
    const uint32_t next = u / SUBS % NB * Sh::kTile + u % SUBS * 32 * RB;
    const bool masked = u < whole || u >= tail;
    const bool more = u && (SUBS == 1 || !(u & 1));    // a tile's last step is over: two tiles on
    step(cur, next, (u & 1) ^ 1, kbase + u * 32, u < steps ? k1 : 0, masked, more, move_of(u / SUBS + 1));
    if (u == steps) break;
    if (SUBS == 1 || (u & 1)) wait_loads<0>();
    barrier();
    if (masked) clean(next, kbase + u * 32);
    cur = next;
  }
  wait_loads<0>();

  // The rows' sums and where they go, from their waves to all.  What a lane holds goes out from its registers: parts
  // as they lie, 1 KB a store, and rows in pieces of 32 bytes (32 rows at a time through LDS, in whole lines,
  // took 20,000 cycles where this takes 14,000).
  // Numbers of lanes are made anew: what the loop would have to keep for here it has no registers for.
  const int lane_ = this_lane(), half_ = lane_ / 32, l32_ = lane_ % 32;
  l = over_halves(l, Sum());
  const int any_odd = __syncthreads_or(odd);
  int64_t* const goes = (int64_t*)(g_lds + NB * Sh::kTile);          // [128], in place of the weights
  float* const inverse = (float*)(goes + 128);                       // [128]
  if (half_ == 0) {
    const int32_t i = wave * 32 + l32_, row_ = row0 + i;
    alphas[i] = parts ? 1.f : l;           // what is 0 in a part need not be 0
    inverse[i] = l == 0 ? 0.f : vs / l;
    if (row_ < rows) {
      const int32_t tok_ = row_ / G, g_ = row_ % G;
      goes[i] = (q.first + tok_) * a.out_token_stride + g_ * a.out_head_stride;
      const float lse = l == 0 ? -INFINITY : m * c + (__log2f(l) - kLift<F16>);
      if (parts) pl.slot_lse[to * 128 + i] = lse;
      else if (a.lse) a.lse[(int64_t)(q.first + tok_) * a.q_heads + g_] = lse / kLog2e;
    }
  }
  barrier();
  float inv = 0;
  int64_t row_at = 0;
#pragma unroll 1
  for (int32_t n = 0; n < 4 * DB && n / DB * 32 < count; ++n) {
    const int32_t e = n / DB, db = n % DB;
    if (db == 0) {
      inv = inverse[e * 32 + l32_];
      row_at = goes[e * 32 + l32_];
    }
    f32x16 o;
    each<4 * DB>([&](auto i) {
      if (i != n) return;
      o = acc[i % DB][i / DB];
      asm volatile("" : "+v"(o));
    });
#pragma unroll
    for (int j = 0; j < 16; ++j) o[j] *= inv;
    if (!parts && __any(inv == 0)) {    // of nothing but scores of -infinity: NaN, it may be
#pragma unroll
      for (int j = 0; j < 16; ++j) o[j] = inv == 0 ? 0.f : o[j];
    }
    if (parts) {
      float* const at = pl.slot_part + part_at<C>(to, e * 32, (wave * DB + db) * 32) + lane_ * 4;
#pragma unroll
      for (int b = 0; b < 4; ++b) *(f32x4*)(at + b * 256) = f32x4{o[4 * b], o[4 * b + 1], o[4 * b + 2], o[4 * b + 3]};
    } else if (e * 32 + l32_ < count) {
      // halves of the wave have four elements each in turn; after the exchange eight
      uint16_t* const at = (uint16_t*)a.out + row_at + (wave * DB + db) * 32 + half_ * 8;
#pragma unroll
      for (int b = 0; b < 4; b += 2) {
        const auto x = __builtin_amdgcn_permlane32_swap(pack2<F16>(o[4 * b], o[4 * b + 1]), pack2<F16>(o[4 * b + 4], o[4 * b + 5]), false, false);
        const auto y = __builtin_amdgcn_permlane32_swap(pack2<F16>(o[4 * b + 2], o[4 * b + 3]), pack2<F16>(o[4 * b + 6], o[4 * b + 7]), false, false);
        *(i32x4*)(at + b * 8) = i32x4{(int32_t)x[0], (int32_t)y[0], (int32_t)x[1], (int32_t)y[1]};
      }
    }
  }
  if (!any_odd) continue;
  __threadfence_block();
  __syncthreads();
  mark_odd<F16, NARROW, C, TK>(p, a, pl, r, q.start, row0, count, kbase, k1, spans<TK>(kbase, nt, pos_lo, pos_hi, k1, a.window), alphas, [&](int32_t i, int32_t d) {
    if (parts) pl.slot_part[part_at<C>(to, i, d)] = __builtin_nanf("");
    else ((uint16_t*)a.out)[goes[i] + d] = F16 ? 0x7e00 : 0x7fc0;
  });
  }
}

// --------------------------------------------------------- k_latent_join ---

// Cut rows, of the `each` at most of a cut.  Bound by the chain of its loads where parts are few (a lone request 4.3 us)
// and by memory where they are many (48 requests of 128 heads, 77 MB, 13.0 us): a wave reads eight parts at a time, their
// log sums with them, and WAVES waves share parts where they are many.  A wave has a row of k_latent_rows, or
// a 32nd of 32 rows of k_latent_tiles, as they lie.
template <bool F16, int C, int ROWS, int WAVES>
__global__ void __launch_bounds__(256) k_latent_join(pp_attention_args a, Split pl, int32_t each) {
  constexpr bool kTiles = ROWS != kFew;
  constexpr int kTurn = 8, kHalves = C / 256;
  __shared__ float tops[4][kWave], totals[4][kWave];
  __shared__ f32x4 outs[4][C / 4];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int32_t id = blockIdx.x * (4 / WAVES) + wave / WAVES, share = wave % WAVES;
  const int32_t cut = id / each, piece = id % each;
  const Cut at = (kTiles ? pl.slot_cut : pl.row_cut)[cut];
  if ((kTiles ? piece / 32 * 32 : piece) >= at.rows) return;         // all waves of the rows
  const int32_t row = kTiles ? piece / 32 * 32 + lane % 32 : piece;
  const float* const from = (kTiles ? pl.slot_part : pl.row_part) +
                            (kTiles ? (int64_t)(piece / 32 * 32) * C + piece % 32 * (kHalves * 256) : (int64_t)piece * C) + lane * 4;
  const float* const sums = (kTiles ? pl.slot_lse : pl.row_lse) + row;
  float m = -INFINITY, sum = 0;
  f32x4 o[kHalves];
#pragma unroll
  for (int h = 0; h < kHalves; ++h) o[h] = f32x4{0, 0, 0, 0};
  const int32_t count = at.last - at.block + 1, mine = (count + WAVES - 1) / WAVES;
  const int32_t p0 = at.block + share * mine, p1 = p0 + mine <= at.last ? p0 + mine : at.last + 1;
  for (int32_t base = p0; base < p1; base += kTurn) {
    float x[kTurn];
    f32x4 y[kTurn][kHalves];
#pragma unroll
    for (int j = 0; j < kTurn; ++j) {
      const int32_t i = base + j < p1 ? base + j : p1 - 1;
      const int64_t part = (2 * (int64_t)i + (i == at.block)) * ROWS;
      x[j] = sums[part];
#pragma unroll
      for (int h = 0; h < kHalves; ++h) y[j][h] = *(const f32x4*)(from + part * C + h * 256);
    }
    float n = m;
#pragma unroll
    for (int j = 0; j < kTurn; ++j) n = fmaxf(n, x[j]);
    const float al = m == -INFINITY ? 0.f : exp2_(m - n);
#pragma unroll
    for (int h = 0; h < kHalves; ++h) o[h] *= al;
    sum *= al;
    m = n;
#pragma unroll
    for (int j = 0; j < kTurn; ++j) {
      if (base + j >= p1) continue;
      const float w = x[j] == -INFINITY ? 0.f : x[j] == n ? 1.f : exp2_(x[j] - n);   // a part that saw nothing is 0 or NaN
      sum += w;
#pragma unroll
      for (int h = 0; h < kHalves; ++h) o[h] += w * y[j][h];
    }
  }
  if constexpr (WAVES > 1) {
    tops[wave][lane] = m;
    totals[wave][lane] = sum;
#pragma unroll
    for (int h = 0; h < kHalves; ++h) outs[wave][h * 64 + lane] = o[h];
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int v = 1; v < WAVES; ++v) {
      const float top = tops[v][lane], total = totals[v][lane];
      const float n = fmaxf(m, top);
      const float al = m == -INFINITY ? 0.f : exp2_(m - n), be = total == 0 ? 0.f : top == n ? 1.f : exp2_(top - n);
      sum = sum * al + total * be;
#pragma unroll
      for (int h = 0; h < kHalves; ++h) o[h] = o[h] * al + outs[v][h * 64 + lane] * be;
      m = n;
    }
  }
  if (row >= at.rows) return;
  const float inv = sum == 0 ? 0.f : 1.f / sum;
  const int32_t t = at.first + (at.row + row) / pl.group, g = (at.row + row) % pl.group;
#pragma unroll
  for (int h = 0; h < kHalves; ++h)
    store4<F16>(a, t, g, kTiles ? (piece % 32 * kHalves + h) * 8 + lane / 32 * 4 : h * 256 + lane * 4,
                sum == 0 ? f32x4{0, 0, 0, 0} : o[h] * inv);
  if (a.lse && (kTiles ? piece % 32 == 0 && lane < 32 : lane == 0))
    a.lse[(int64_t)t * a.q_heads + g] = sum == 0 ? -INFINITY : (m + __log2f(sum)) / kLog2e;
}

// -------------------------------------------------------------- dispatch ---

struct Choice {
  bool rows, tiles;
};

// Every rule here goes by sizes the host knows, so the workspace is known before the call.
Choice choose(const pp_kv_pages& p, const pp_attention_args& a, Split& pl) {
  Choice ch{};
  pl.group = a.q_heads;
  pl.shift = __builtin_ctz(p.page_size);
  if ((int64_t)a.max_new * pl.group <= kFew) {
    ch.rows = true;
  } else {
    ch.tiles = true;
    // requests of few rows apart, unless every request has max_new tokens, or those that can be of few rows have few keys
    if (pl.group <= kFew && (int64_t)a.requests * a.max_new != a.tokens) {
      const int64_t few = kFew / pl.group;      // tokens; max_new is above it
      const int64_t others = ((int64_t)a.tokens - few * a.requests + a.max_new - few - 1) / (a.max_new - few);
      const int64_t keys = std::min((int64_t)a.max_len, (int64_t)a.max_blocks << pl.shift);
      ch.rows = (a.requests - std::max<int64_t>(others, 0)) * keys > kAlone;
    }
  }
  pl.few = ch.rows ? kFew : 0;
  const int64_t slots = (int64_t)a.tokens * pl.group / 128 + a.requests;
  pl.slots = slots < INT32_MAX ? (int32_t)slots : INT32_MAX;
  pl.even = slots <= kSlots;
  pl.by_slot = slots < kBlocks;     // fewer blocks of k_latent_join without rows: 32 requests of 4 new tokens 78 us for 81
  return ch;
}

// Bytes of the workspace; its regions where `pl` is given one.
int64_t regions(int32_t value_dim, const pp_attention_args& a, const Choice& ch, Split& pl) {
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    char* const x = (char*)a.workspace + at;
    at += (bytes + 255) / 256 * 256;
    return x;
  };
  if (ch.rows) {
    pl.row_part = (float*)take((int64_t)2 * kBlocks * kFew * value_dim * 4);
    pl.row_lse = (float*)take((int64_t)2 * kBlocks * kFew * 4);
    pl.row_cut = (Cut*)take(kBlocks * sizeof(Cut));
  }
  if (ch.tiles && pl.even) {
    pl.slot_part = (float*)take((int64_t)2 * kBlocks * 128 * value_dim * 4);
    pl.slot_lse = (float*)take((int64_t)2 * kBlocks * 128 * 4);
    pl.slot_cut = (Cut*)take(kBlocks * sizeof(Cut));    // or one a slot, fewer
  }
  return at;
}

template <bool F16, bool NARROW, int C>
hipError_t go(const pp_kv_pages& p, const pp_attention_args& a, const Split& pl, const Choice& ch, hipStream_t st) {
  const int64_t most = (int64_t)a.max_new * pl.group;      // rows of a request
  if (ch.tiles) {
    constexpr int lds = LatentTiles<NARROW, C>::kLds;
    static OnEachGpu once;
    const hipError_t ok = allow_lds(once, &k_latent_tiles<F16, NARROW, C>, lds);
    if (ok != hipSuccess) return ok;
    if (!pl.even && pl.slots > most_blocks(256)) return hipErrorInvalidConfiguration;
    k_latent_tiles<F16, NARROW, C><<<pl.even ? kBlocks : pl.slots, 256, lds, st>>>(p, a, pl);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (pl.even) {
      const int32_t each = most < 128 ? ((int32_t)most + 31) / 32 * 32 : 128, cuts = pl.by_slot ? pl.slots : kBlocks;
      // few slots are in many parts
      if (pl.slots <= 64) k_latent_join<F16, C, 128, 4><<<cuts * each, 256, 0, st>>>(a, pl, each);
      else k_latent_join<F16, C, 128, 1><<<cuts * each / 4, 256, 0, st>>>(a, pl, each);
      const hipError_t e2 = hipGetLastError();
      if (e2 != hipSuccess) return e2;
    }
  }
  if (ch.rows) {
    constexpr int lds = LatentRows<NARROW, C>::kLds;
    static OnEachGpu once;
    const hipError_t ok = allow_lds(once, &k_latent_rows<F16, NARROW, C>, lds);
    if (ok != hipSuccess) return ok;
    k_latent_rows<F16, NARROW, C><<<kBlocks, 256, lds, st>>>(p, a, pl);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int32_t each = (int32_t)(most < kFew ? most : kFew);
    k_latent_join<F16, C, kFew, 4><<<kBlocks * each, 256, 0, st>>>(a, pl, each);
    return hipGetLastError();
  }
  return hipSuccess;
}

template <bool F16, bool NARROW>
hipError_t go_dim(const pp_kv_pages& p, int32_t value_dim, const pp_attention_args& a, const Split& pl, const Choice& ch,
                  hipStream_t st) {
  if (value_dim == 512) return go<F16, NARROW, 512>(p, a, pl, ch, st);
  return go<F16, NARROW, 256>(p, a, pl, ch, st);
}

}  // namespace

int64_t latent_workspace(const pp_kv_pages& p, int32_t value_dim, const pp_attention_args& a) {
  Split pl{};
  const Choice ch = choose(p, a, pl);
  return regions(value_dim, a, ch, pl);
}

hipError_t launch_latent(const pp_kv_pages& p, int32_t value_dim, const pp_attention_args& a, hipStream_t st) {
  Split pl{};
  const Choice ch = choose(p, a, pl);
  regions(value_dim, a, ch, pl);
  pl.negative = a.scale < 0 ? (int32_t)0x80008000 : 0;     // the queries' signs
  pl.c = std::fabs(a.scale) * kLog2e;
  const bool narrow = p.dtype == PP_E4M3;
  if (a.dtype == PP_F16) return narrow ? go_dim<true, true>(p, value_dim, a, pl, ch, st) : go_dim<true, false>(p, value_dim, a, pl, ch, st);
  return narrow ? go_dim<false, true>(p, value_dim, a, pl, ch, st) : go_dim<false, false>(p, value_dim, a, pl, ch, st);
}

}  // namespace pp

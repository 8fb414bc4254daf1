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
// through LDS.  Both leave parts of long requests to k_join.

#include "pp_attend.h"

namespace pp {

namespace {

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
    return NARROW ? (row >> 2) & 3 : (row & 2) << 1 | (row & 4) >> 1;
  }
  // This lane's source of load i of kKeys / 2 rows, in bytes from the first.
  static __device__ __forceinline__ uint32_t source(int i, int lane, uint32_t tok_b) {
    const int u = i * 64 + lane, row = u / kUnits;
    return row * tok_b + ((u % kUnits) ^ swizzle(row)) * 16;
  }
};

// What a row does not see does not touch it, whatever it holds.  In tiles that some row does not see
// whole, elements that are not finite go into the product as 0.  A row that sees one has a score of NaN or
// +infinity from it, and is NaN whole by its sum, or of -infinity, and then that element's weight of 0 times an
// infinity makes it NaN: so the row's element is set to NaN.
template <bool F16>
__device__ __forceinline__ s16x8 odd_ones(s16x8 v) {      // 1 where v is not finite
  s16x8 o;
  const uint16_t top = F16 ? 0x7c00 : 0x7f80;
#pragma unroll
  for (int j = 0; j < 8; ++j) o[j] = ((uint16_t)v[j] & top) == top ? (short)(F16 ? 0x3c00 : 0x3f80) : (short)0;
  return o;
}

// -------------------------------------------------------- k_latent_rows ---

template <bool NARROW, int C>
struct LatentRows : Latent<NARROW, C> {
  using L = Latent<NARROW, C>;
  static constexpr int kNW = 4;                             // waves
  static constexpr int kNS = C == 512 ? 2 : 3;              // stages of a wave's ring
  static constexpr int kRing = kNW * kNS * L::kStage;
  static constexpr int kRow = C + 4;                        // floats of a joined row
  static constexpr int kJoin = kNW * 16 * (kRow + 2) * 4;
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

template <bool F16, bool NARROW, int C, int RT>
__global__ void __launch_bounds__(256, 1) k_latent_rows(pp_kv_pages p, pp_attention_args a, Plan pl) {
  using Sh = LatentRows<NARROW, C>;
  constexpr int RB = Sh::kRB, NW = Sh::kNW, NS = Sh::kNS, KEYS = Sh::kKeys, KB = KEYS / 16;
  constexpr int DB = C / 16, KS = Sh::kKS16;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int part = blockIdx.x % pl.parts_rows;
  const int32_t r = blockIdx.x / pl.parts_rows;
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
  const int32_t tiles = k1 > k0 ? (int32_t)((k1 - k0 + KEYS - 1) / KEYS) : 0;
  const int32_t share = (tiles + NW - 1) / NW;
  const int32_t t0 = wave * share < tiles ? wave * share : tiles;
  const int32_t nt = t0 + share < tiles ? share : tiles - t0;
  const int32_t kbase = (int32_t)k0 + t0 * KEYS;
  const int grp = lane / 16, i16 = lane % 16;

  // this lane's row of each tile of rows: its token's position, or -1
  int32_t pos[RT];
  s16x8 qf[RT][KS];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int32_t row = rt * 16 + i16;
    const int32_t tok = row / G, g = row % G;
    pos[rt] = row < rows ? q.start + tok : -1;
    const uint16_t* src = (const uint16_t*)a.q + (q.first + (row < rows ? tok : 0)) * a.q_token_stride +
                          (row < rows ? g : 0) * a.q_head_stride + grp * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      i32x4 x = *(const i32x4*)(src + ks * 32);
      if (pl.negative) x ^= (int)0x80008000;
      qf[rt][ks] = __builtin_bit_cast(s16x8, x);
    }
  }
  const float vs = NARROW && p.k_scale ? p.k_scale[0] : 1.f;
  const float c = pl.c * vs;

  const int64_t es = NARROW ? 1 : 2;
  const int64_t page_b = p.page_stride * es;
  const uint32_t tok_b = (uint32_t)(p.token_stride * es);
  const char* rows_at = (const char*)p.k;
  const uint32_t ring = lds_base() + wave * (NS * Sh::kStage);
  uint32_t off[Sh::kHalf];
#pragma unroll
  for (int i = 0; i < Sh::kHalf; ++i) off[i] = Sh::source(i, lane, tok_b);
  const int32_t* blocks = a.block_table + r * a.row_stride;
  int32_t held = 0;
  auto issue = [&](int32_t t) {
    const uint32_t to = __builtin_amdgcn_readfirstlane(ring + (t % NS) * Sh::kStage);
    if ((t * KB & 63) == 0) held = page_of(p, a, pl, blocks, (int64_t)kbase + ((int64_t)t * KB + lane) * 16);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int32_t key = kbase + t * KEYS + half * (KEYS / 2);
      const int64_t page = __builtin_amdgcn_readlane(held, (t * KB + (KB - 1) * half) & 63);
      const char* from = rows_at + page * page_b + (int64_t)(key & (p.page_size - 1)) * tok_b;
      each<Sh::kHalf>([&](auto i) { load_lds(to + (half * Sh::kHalf + i) * 1024, off[i], from); });
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
  const int32_t pos_lo = q.start;   // the first row's; rows of -1 see nothing in any case
  const int32_t pos_hi = q.start + q.count - 1;

  auto tile = [&](int32_t t, auto masked) {
    constexpr bool kMasked = decltype(masked)::value;   // some row does not see all of it
    if (t + NS - 1 < nt) {
      issue(t + NS - 1);
      wait_loads<(NS - 1) * Sh::kLoads>();
    } else if (NS > 2 && t + NS - 2 < nt) {
      wait_loads<(NS > 2 ? NS - 2 : 0) * Sh::kLoads>();
    } else {
      wait_loads<0>();
    }
    const uint32_t at = ring + (t % NS) * Sh::kStage;
    f32x4 s[RT][KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) s[rt][kb] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        s16x8 f;
        const uint32_t from = at + kb * 16 * RB + k_at[ks % 2] + ks / 2 * (NARROW ? 64 : 128);
        if constexpr (NARROW) f = widen8<F16>(*LDS_PTR(i32x2, from));
        else f = *LDS_PTR(s16x8, from);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) s[rt][kb] = mfma16<F16>(f, qf[rt][ks], s[rt][kb]);
      }
    }
    const int32_t key0 = kbase + t * KEYS + 4 * grp;   // of s[.][0][0]; + 16 kb + i
    s16x8 pf[RT];                                      // of 16 keys: its first half
    uint32_t seen[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float x[4 * KB], w[8];
      seen[rt] = 0xff;
#pragma unroll
      for (int j = 0; j < 4 * KB; ++j) x[j] = s[rt][j / 4][j % 4];
      if constexpr (kMasked) {
        seen[rt] = 0;
#pragma unroll
        for (int j = 0; j < 4 * KB; ++j) {
          const int32_t key = key0 + (j / 4) * 16 + j % 4;
          const bool ok = sees(pos[rt], key, a.window) && key < k1;
          seen[rt] |= ok ? 1u << j : 0;
          if (!ok) x[j] = -INFINITY;
        }
      }
      float mx = x[0];
#pragma unroll
      for (int j = 1; j < 4 * KB; ++j) mx = fmaxf(mx, x[j]);
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
        w[j] = 0;
        if (j >= 4 * KB) continue;
        w[j] = exp2_(__builtin_fmaf(x[j], c, -mc));
        if (kMasked && !(seen[rt] >> j & 1)) w[j] = 0;
        sum += w[j];
      }
      l[rt] += sum;
      pf[rt] = pack8<F16>(w);
    }
    // the values of 32 (16 bits: two blocks of 16) elements of the latent
    auto v_frag = [&](int db) -> s16x8 {
      if constexpr (NARROW) {
        return widen8<F16>(__builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(
            LDS_PTR(i32x2, at + v_at[db % 4] + db / 4 * 64))));
      } else {
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, at + v_at[2 * db % 4] + 2 * db / 4 * 128));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, at + v_at[(2 * db + 1) % 4] + 2 * db / 4 * 128));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      }
    };
    constexpr int kPer = NARROW ? 1 : 2, NB = DB / kPer;
    auto product = [&](s16x8 v, s16x8 w, f32x4* o) {
      if constexpr (NARROW) {
        o[0] = mfma16<F16>(v, w, o[0]);
      } else {
        const s16x4 lo = __builtin_shufflevector(w, w, 0, 1, 2, 3);
        o[0] = mfma16x16<F16>(__builtin_shufflevector(v, v, 0, 1, 2, 3), lo, o[0]);
        o[1] = mfma16x16<F16>(__builtin_shufflevector(v, v, 4, 5, 6, 7), lo, o[1]);
      }
    };
    if constexpr (!kMasked) {
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const s16x8 f = v_frag(b);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) product(f, pf[rt], &acc[rt][b * kPer]);
      }
    } else {
      uint32_t odd = 0;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const s16x8 f = only_finite<F16>(v_frag(b), odd);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) product(f, pf[rt], &acc[rt][b * kPer]);
      }
      if (__any(odd != 0)) {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const s16x8 f = odd_ones<F16>(v_frag(b));
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            f32x4 n[kPer];
#pragma unroll
            for (int e = 0; e < kPer; ++e) n[e] = f32x4{0, 0, 0, 0};
            product(f, ones8<F16>(seen[rt]), n);
#pragma unroll
            for (int e = 0; e < kPer; ++e)
#pragma unroll
              for (int i = 0; i < 4; ++i) acc[rt][b * kPer + e][i] = n[e][i] != 0 ? __builtin_nanf("") : acc[rt][b * kPer + e][i];
          }
        }
      }
    }
    wait_lds();   // this stage's reads are done before its next load is issued
  };
  const Span3 sp = spans<KEYS>(kbase, nt, pos_lo, pos_hi, (int32_t)k1, a.window);
  for (int32_t t = 0; t < NS - 1 && t < nt; ++t) issue(t);
  int32_t t = 0;
  for (int pass = 0; pass < 2; ++pass) {
    for (const int32_t e = pass ? nt : sp.whole; t < e; ++t) tile(t, std::true_type());
    if (pass == 0)
      for (; t < sp.tail; ++t) tile(t, std::false_type());
  }

  // the waves' parts of 16 rows at a time are joined in LDS
  float* js = (float*)g_lds;                       // [NW][16][kRow]
  float* jm = js + NW * 16 * Sh::kRow;             // [NW][16]
  float* jl = jm + NW * 16;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    __syncthreads();
    const float ls = over_halves(over_rows(l[rt], Sum()), Sum());
    if (grp == 0) {
      jm[wave * 16 + i16] = m[rt];
      jl[wave * 16 + i16] = ls;
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) *(f32x4*)&js[(wave * 16 + i16) * Sh::kRow + db * 16 + grp * 4] = acc[rt][db];
    __syncthreads();
    const int left = rows - rt * 16 < 16 ? rows - rt * 16 : 16;
    for (int i = threadIdx.x; i < left * (C / 4); i += NW * kWave) {
      const int row = i / (C / 4), d = i % (C / 4) * 4;
      float mm = -INFINITY, ll = 0;
#pragma unroll
      for (int w = 0; w < NW; ++w) mm = fmaxf(mm, jm[w * 16 + row]);
      f32x4 o = {0, 0, 0, 0};
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float mw = jm[w * 16 + row], lw = jl[w * 16 + row];
        if (lw == 0) continue;      // it saw nothing
        const float f = mw == mm ? 1.f : exp2_((mw - mm) * c);
        ll += f * lw;
        o += f * *(const f32x4*)&js[(w * 16 + row) * Sh::kRow + d];
      }
      const float inv = ll == 0 ? 0.f : vs / ll;
      o *= inv;
      const float lse = ll == 0 ? -INFINITY : mm * c + (__log2f(ll) - kLift<F16>);
      const int32_t tk = q.first + (rt * 16 + row) / G, g = (rt * 16 + row) % G;
      if (parts == 1) {
        store4<F16>(a, tk, g, d, o);
        if (a.lse && d == 0) a.lse[(int64_t)tk * a.q_heads + g] = lse / kLog2e;
      } else {
        const int64_t to = ((int64_t)part * a.requests + r) * pl.few + rt * 16 + row;
        *(f32x4*)&pl.row_part[to * C + d] = o;
        if (d == 0) pl.row_lse[to] = lse;
      }
    }
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
  static constexpr int kLds = kNB * kTile + 2 * kWeights + 2 * 128 * 4 + 2 * 16;
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

// 16 passes of the last instruction that wrote x are over after 19 wait states.
__device__ __forceinline__ void settle(f32x16& x) { asm volatile("s_nop 15\n\ts_nop 7" : "+v"(x)); }

// 128 rows of one request and one part of its keys a block.
template <bool F16, bool NARROW, int C>
__global__ void __launch_bounds__(256, 1) k_latent_tiles(pp_kv_pages p, pp_attention_args a, Plan pl) {
  using Sh = LatentTiles<NARROW, C>;
  constexpr int RB = Sh::kRB, KS = Sh::kKS32, SUBS = Sh::kSubs, TK = Sh::kKeysTile, NB = Sh::kNB;
  constexpr int DB = C / 128;                               // blocks of 32 of a wave's quarter of the latent
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int part = blockIdx.x % pl.parts_tiles;
  const int32_t slot = blockIdx.x / pl.parts_tiles;
  const int G = pl.group;
  const Slot at_slot = slot_of(a, pl, slot);
  const int32_t r = at_slot.r;
  if (r < 0) return;
  const Request q = request(a, pl, r);
  const int64_t rows = (int64_t)q.count * G;
  const int64_t row0 = (int64_t)(slot - at_slot.first) * 128;
  if (rows <= pl.few || row0 >= rows) return;
  const int32_t parts = parts_of(q, pl.cut_tiles, pl.parts_tiles);
  if (part >= parts) return;

  const int half = lane / 32, l32 = lane % 32, i16 = lane % 16, dh = (lane / 16) % 2;
  const int64_t row = row0 + wave * 32 + l32;
  const bool live = row < rows;
  const int32_t tok = (int32_t)((live ? row : 0) / G), g = (int32_t)((live ? row : 0) % G);
  const int32_t pos = live ? q.start + tok : -1;

  // keys of this part that the tile's rows see
  const int32_t tok_lo = (int32_t)(row0 / G);
  const int64_t last = row0 + 127 < rows ? row0 + 127 : rows - 1;
  const int32_t pos_lo = q.start + tok_lo, pos_hi = q.start + (int32_t)(last / G);
  int64_t k0 = q.lo + (int64_t)part * pl.cut_tiles;
  int64_t k1 = part + 1 < parts ? k0 + pl.cut_tiles : q.hi;
  if (k1 > (int64_t)pos_hi + 1) k1 = (int64_t)pos_hi + 1;
  if (k1 > q.hi) k1 = q.hi;
  if (a.window && (int64_t)pos_lo - a.window + 1 > k0) k0 = (pos_lo - a.window + 1) & ~63;
  const int32_t nt = k1 > k0 ? (int32_t)((k1 - k0 + TK - 1) / TK) : 0;
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
  const float vs = NARROW && p.k_scale ? p.k_scale[0] : 1.f;
  const float c = pl.c * vs;

  const int64_t es = NARROW ? 1 : 2;
  const int64_t page_b = p.page_stride * es;
  const uint32_t tok_b = (uint32_t)(p.token_stride * es);
  const uint32_t lds = lds_base(), weights = lds + NB * Sh::kTile;
  float* const alphas = (float*)(g_lds + NB * Sh::kTile + 2 * Sh::kWeights);     // [2][128]
  int32_t* const grown = (int32_t*)(alphas + 2 * 128);                          // [2][4]
  // wave w brings a quarter of a tile's keys
  constexpr int kMine = TK / 4;
  const uint32_t own = __builtin_amdgcn_readfirstlane(lds + wave * kMine * RB);
  uint32_t off[Sh::kHalf];
#pragma unroll
  for (int i = 0; i < Sh::kHalf; ++i) off[i] = Sh::source(i, lane, tok_b);
  const int32_t* blocks = a.block_table + r * a.row_stride;
  int32_t held = 0;
  auto issue = [&](int32_t t) {
    if (t >= nt) return;
    if ((t & 63) == 0) held = page_of(p, a, pl, blocks, (int64_t)kbase + (int64_t)(t + lane) * TK + wave * kMine);
    const int64_t page = __builtin_amdgcn_readlane(held, t & 63);
    const char* from = (const char*)p.k + page * page_b + (int64_t)((kbase + t * TK + wave * kMine) & (p.page_size - 1)) * tok_b;
    const uint32_t to = own + t % NB * Sh::kTile;
    each<Sh::kHalf>([&](auto i) { load_lds_at<i * 1024>(to, off[i], from); });
  };

  f32x16 acc[DB][4];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[d][e][i] = 0;
  float m = -INFINITY, l = 0;

  // reads along a row: key l32, its units half + 2 ks (8 bits: the half of unit ks); transposed ones of
  // this wave's quarter
  const uint32_t kx = NARROW ? Sh::swizzle(l32) * 16 + half * 8 : (half ^ Sh::swizzle(l32)) * 16;
  const int vrow = NARROW ? ((i16 / 2) / 4) * 8 + 4 * half + (i16 / 2) % 4 : 4 * half + i16 / 4;
  const uint32_t vx = NARROW ? (dh ^ Sh::swizzle(vrow)) * 16 + (i16 % 2) * 8
                             : ((dh * 2 + (i16 % 4) / 2) ^ Sh::swizzle(vrow)) * 16 + (i16 % 2) * 8;
  uint32_t k_at[4], v_at[2];
#pragma unroll
  for (int i = 0; i < 4; ++i) k_at[i] = lds + l32 * RB + (kx ^ (i * (NARROW ? 16 : 32)));
#pragma unroll
  for (int i = 0; i < 2; ++i) v_at[i] = lds + vrow * RB + (vx ^ (i * (NARROW ? 32 : 64))) + wave * (RB - 64 * (int)es) / 4;
  auto k_frag = [&](uint32_t at, int ks) -> s16x8 {
    const uint32_t from = at + k_at[ks % 4] + ks / 4 * (NARROW ? 64 : 128);
    if constexpr (NARROW) return widen8<F16>(*LDS_PTR(i32x2, from));
    else return *LDS_PTR(s16x8, from);
  };
  // keys 8 (j / 4) + 4 half + j % 4 of 16, as the weights' registers have them
  auto v_frag = [&](uint32_t at, int db) -> s16x8 {
    const uint32_t from = at + v_at[db % 2] + db / 2 * (NARROW ? 64 : 128);
    if constexpr (NARROW) {
      return widen8<F16>(__builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(LDS_PTR(i32x2, from))));
    } else {
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, from));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, from + 8 * RB));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  };
  auto scores = [&](uint32_t at) -> f32x16 {       // of 32 keys
    f32x16 x;
    each<KS>([&](auto ks) { mfma32_vector<F16, ks == 0>(x, k_frag(at, ks), qf[ks]); });
    settle(x);
    return x;
  };

  auto p_frag = [&](int b, int i) -> s16x8 {       // weights of rows 32 (i / 2) .., keys 16 (i % 2) ..
    return *LDS_PTR(s16x8, weights + b * Sh::kWeights + i * 1024 + lane * 16);
  };
  auto put_weights = [&](int b, int k, s16x8 w) {
    *LDS_PTR(s16x8, weights + b * Sh::kWeights + (wave * 2 + k) * 1024 + lane * 16) = w;
  };
  // The rows' maximum with that of 32 scores; where one grows too far, all waves have to know.
  auto peak = [&](float mx, int b) {
    mx = over_halves(mx, Max());
    const bool grows = __any(mx > m && (m == -INFINITY || (mx - m) * c > kLag<F16>));
    if (grows) {
      const float n = fmaxf(m, mx);
      const float al = m == -INFINITY ? 0.f : exp2_((m - n) * c);
      l *= al;
      m = n;
      if (half == 0) alphas[b * 128 + wave * 32 + l32] = al;
    }
    if (lane == 0) grown[b * 4 + wave] = grows;
  };
  auto rescale = [&](int b) {
    const i32x4 any = *(const i32x4*)&grown[b * 4];
    if (!__builtin_amdgcn_readfirstlane(any[0] | any[1] | any[2] | any[3])) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (!__builtin_amdgcn_readfirstlane(any[e])) continue;
      const float al = alphas[b * 128 + e * 32 + l32];
      each<DB>([&](auto d) {
        if constexpr (C == 512) asm volatile("" : "+a"(acc[d][e]));
        acc[d][e] *= al;
        if constexpr (C == 512) asm volatile("" : "+a"(acc[d][e]));
        __builtin_amdgcn_sched_barrier(0);
      });
    }
  };

  // A step's scores and weights, and its values, of 32 keys that some row may not see whole.
  uint32_t odd = 0;
  auto weigh = [&](uint32_t at, int32_t key0, int b) {
    f32x16 s = scores(at);
    uint32_t seen = 0;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const int32_t key = key0 + 4 * half + (j / 4) * 8 + j % 4;
      const bool ok = sees(pos, key, a.window) && key < k1;
      seen |= ok ? 1u << j : 0;
      if (!ok) s[j] = -INFINITY;
    }
    float mx = s[0];
#pragma unroll
    for (int j = 1; j < 16; ++j) mx = fmaxf(mx, s[j]);
    peak(mx, b);
    const float mc = top_of<F16>(m, c);
    float w[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      w[j] = (seen >> j & 1) ? exp2_(__builtin_fmaf(s[j], c, -mc)) : 0.f;
      l += w[j];
    }
    put_weights(b, 0, pack8<F16>(w));
    put_weights(b, 1, pack8<F16>(w + 8));
  };
  auto values = [&](uint32_t at, int b) {
    rescale(b);
    each<2>([&](auto k) {
      s16x8 w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = p_frag(b, e * 2 + k);
      each<DB>([&](auto d) {
        const s16x8 f = only_finite<F16>(v_frag(at + k * 16 * RB, d), odd);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[d][e] = mfma32<F16>(f, w[e], acc[d][e]);
        __builtin_amdgcn_sched_barrier(0);
      });
    });
  };

  // The values of one step (at `cur`, weights in buffer b) and the scores and weights of the next, of keys
  // that every row sees.
  constexpr int kAhead = 4, NV = 2 * DB;
  auto step = [&](uint32_t cur, uint32_t next, int b) {
    rescale(b);
    s16x8 f[KS], w[8], v[NV];
    f32x16 y;
    auto read_v = [&](auto i) { v[i] = v_frag(cur + i / DB * 16 * RB, i % DB); };
    auto read_w = [&](auto i) { w[i] = p_frag(b, i % 4 * 2 + i / 4); };
    each<kAhead>([&](auto i) { f[i] = k_frag(next, i); });
    each<KS>([&](auto i) {
      if constexpr (i + kAhead < KS) f[i + kAhead] = k_frag(next, i + kAhead);
      else read_w(std::integral_constant<int, i + kAhead - KS>());
      if constexpr (i == KS - 2) read_v(std::integral_constant<int, 0>());
      mfma32_vector<F16, i == 0>(y, f[i], qf[i]);
      __builtin_amdgcn_sched_barrier(0);
    });
    float mx = -INFINITY, mc = 0, sum = 0, x[16];
    constexpr int NM = NV * 4;
    each<NM>([&](auto at) {
      constexpr int i = decltype(at)::value, g = i / 4, e = i % 4;
      if constexpr (e == 0 && g + 1 < NV) read_v(std::integral_constant<int, g + 1>());
      if constexpr (g >= 1 && g <= 2 && (e == 1 || e == 2) && DB > 2) read_w(std::integral_constant<int, 4 + (g - 1) * 2 + e - 1>());
      if constexpr (DB == 2 && g == 1) read_w(std::integral_constant<int, 4 + e>());
      acc[g % DB][e] = mfma32<F16>(v[g], w[g / DB * 4 + e], acc[g % DB][e]);
      // the next step's weights, a few instructions beside each product
      constexpr int kWait = 4, kMax = NM / 8, kPeak = kWait + kMax, kExp = kPeak + 1, kEnd = NM - NM / 8;
      if constexpr (i == kWait - 1) settle(y);
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
      if constexpr (i == kEnd) put_weights(b ^ 1, 0, pack8<F16>(x));
      if constexpr (i == kEnd + 1) put_weights(b ^ 1, 1, pack8<F16>(x + 8));
      __builtin_amdgcn_sched_barrier(0);
    });
    l += sum;
  };

  const Span3 sp = spans<TK>(kbase, nt, pos_lo, pos_hi, (int32_t)k1, a.window);
  issue(0);
  issue(1);
  // One barrier a step of 32 keys.  Before it the step's weights are written and the next step's keys
  // waited for; behind it every wave is past the values of the step before, whose tile is brought anew.
  if (nt > 1) wait_loads<Sh::kHalf>();
  else wait_loads<0>();
  barrier();
  const int32_t steps = nt * SUBS, whole = sp.whole * SUBS, tail = sp.tail * SUBS;
  auto turn = [&](int32_t u) {       // step u's weights are on their way
    const bool end = SUBS == 1 || (u & 1);
    if (end) wait_loads<0>();
    barrier();
    if (end) issue(u / SUBS + 2);
  };
  auto place = [&](int32_t u) -> uint32_t { return u / SUBS % NB * Sh::kTile + u % SUBS * 32 * RB; };
  int32_t u = 0;
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {
#pragma unroll 1
    for (const int32_t e = pass ? steps : whole; u < e; ++u) {
      weigh(place(u), kbase + u * 32, u & 1);
      turn(u);
      values(place(u), u & 1);
    }
    if (pass || u >= tail) continue;
    weigh(place(u), kbase + u * 32, u & 1);
    turn(u);
    uint32_t cur = place(u);
#pragma unroll 1
    for (; u + 1 < tail; ++u) {
      const uint32_t next = place(u + 1);
      step(cur, next, u & 1);
      turn(u + 1);
      cur = next;
    }
    values(cur, u & 1);
    ++u;
  }

  // sums and log sums from the rows' waves to all
  l = over_halves(l, Sum());
  barrier();
  if (half == 0) alphas[wave * 32 + l32] = l;
  if (half == 0 && live) {
    const float lse = l == 0 ? -INFINITY : m * c + (__log2f(l) - kLift<F16>);
    const int64_t at = (int64_t)(q.first + tok) * a.q_heads + g;
    if (parts > 1) pl.part_lse[(int64_t)part * a.tokens * a.q_heads + at] = lse;
    else if (a.lse) a.lse[at] = lse / kLog2e;
  }
  barrier();
  each<4>([&](auto e) {
    const int64_t other = row0 + e * 32 + l32;
    if (other >= rows) return;
    const int32_t tk = q.first + (int32_t)(other / G), og = (int32_t)(other % G);
    const float le = alphas[e * 32 + l32], inv = vs / le;
    const int64_t at = ((int64_t)part * a.tokens + tk) * a.q_heads + og;
    each<DB>([&](auto db) {
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        f32x4 o = {acc[db][e][4 * b], acc[db][e][4 * b + 1], acc[db][e][4 * b + 2], acc[db][e][4 * b + 3]};
        // where l is 0 the products may still hold 0 times an infinity
        o = le == 0 ? f32x4{0, 0, 0, 0} : o * inv;
        const int d = (wave * DB + db) * 32 + b * 8 + half * 4;
        if (parts == 1) store4<F16>(a, tk, og, d, o);
        else *(f32x4*)&pl.part[at * C + d] = o;
      }
      __builtin_amdgcn_sched_barrier(0);
    });
  });
  if (!__any(odd != 0)) return;
  // Elements that are not finite, in keys that some row does not see: a wave marks its own quarter of
  // the rows that see them, behind its own stores.
  __threadfence_block();
  const int32_t all = (int32_t)(rows - row0 < 128 ? rows - row0 : 128);
#pragma unroll 1
  for (int32_t v = 0; v < steps; ++v) {
    if (v >= whole && v < tail) continue;
#pragma unroll 1
    for (int32_t key = kbase + v * 32; key < kbase + v * 32 + 32 && key < k1; ++key) {
      const char* from = (const char*)p.k + page_of(p, a, pl, blocks, key) * page_b + (int64_t)(key & (p.page_size - 1)) * tok_b;
#pragma unroll 1
      for (int32_t d = wave * DB * 32 + lane; d < (wave + 1) * DB * 32; d += kWave) {
        uint32_t x;
        if constexpr (NARROW) x = (((const uint8_t*)from)[d] & 0x7f) == 0x7f;
        else x = not_finite<F16>(((const uint16_t*)from)[d]) & 0x8000u;
        if (!x) continue;
#pragma unroll 1
        for (int32_t i = 0; i < all; ++i) {
          const int32_t tk = (int32_t)((row0 + i) / G), og = (int32_t)((row0 + i) % G);
          if (!sees(q.start + tk, key, a.window) || alphas[i] == 0) continue;
          if (parts == 1)
            ((uint16_t*)a.out)[(q.first + tk) * a.out_token_stride + og * a.out_head_stride + d] = F16 ? 0x7e00 : 0x7fc0;
          else
            pl.part[(((int64_t)part * a.tokens + q.first + tk) * a.q_heads + og) * C + d] = __builtin_nanf("");
        }
      }
    }
  }
}

// -------------------------------------------------------------- dispatch ---

int64_t round_up(int64_t x, int32_t m) { return (x + m - 1) / m * m; }

struct Choice {
  int rt;                       // tiles of 16 rows in k_latent_rows, 0 = not launched
  bool tiles, join;
};

// Every rule here goes by sizes the host knows, so the workspace is known before the call.
Choice choose(const pp_kv_pages& p, int32_t value_dim, const pp_attention_args& a, Plan& pl) {
  Choice ch{};
  pl.group = a.q_heads;
  pl.shift = __builtin_ctz(p.page_size);
  constexpr int kMost = 32;                     // rows k_latent_rows has registers for
  const int64_t rows = (int64_t)a.max_new * pl.group;
  if (rows <= kMost) {
    ch.rt = rows <= 16 ? 1 : 2;
  } else {
    ch.tiles = true;
    // single tokens apart, unless every request has max_new tokens
    if (pl.group <= kMost && (int64_t)a.requests * a.max_new != a.tokens) ch.rt = pl.group <= 16 ? 1 : 2;
  }
  pl.few = ch.rt * 16;
  // keys that a request's rows see, at most; tokens past a row of the block table do not exist
  int64_t keys = (int64_t)a.max_blocks * p.page_size;
  if (a.max_len < keys) keys = a.max_len;
  if (keys < 1) keys = 1;
  if (a.window && (int64_t)a.window + a.max_new + 64 < keys) keys = (int64_t)a.window + a.max_new + 64;
  // n parts at most; the last one is open, so a size held to 31 bits loses no key
  auto cut = [&](int64_t n, int32_t& size, int32_t& parts) {
    const int64_t x = round_up((keys + n - 1) / n, 128), most = INT32_MAX / 128 * 128;
    size = (int32_t)(x < most ? x : most);
    const int64_t count = (keys + size - 1) / size;
    parts = (int32_t)(count < n ? count : n);
  };
  cut(1, pl.cut_rows, pl.parts_rows);
  cut(1, pl.cut_tiles, pl.parts_tiles);
  if (ch.rt) {
    int64_t n = (2048 + a.requests - 1) / a.requests;
    if (n > keys / 256) n = keys / 256;
    cut(n > 1 ? n : 1, pl.cut_rows, pl.parts_rows);
  }
  pl.slots = (int32_t)((int64_t)a.tokens * pl.group / 128) + a.requests;
  if (ch.tiles) {
    // as many parts as end soonest: rounds of resident blocks, each of its share of the tiles and some
    // tiles' time to start and end, and the join's reading and writing of every part
    const double blocks = (double)a.tokens * pl.group / 128 + 1, tiles = keys / 32.0;
    const double tile_us = 1.5 * value_dim / 512;
    const double part_us = (double)a.tokens * a.q_heads * value_dim * 8 / 4e6;
    double best = 0;
    int32_t n = 1;
    const double part_bytes = (double)a.tokens * a.q_heads * value_dim * 4;
    // 512 MiB of parts at most
    for (int32_t i = 1; i <= 64 && (i == 1 || (tiles / i >= 8 && i * part_bytes <= 0x1p29)); ++i) {
      const double t = std::ceil(blocks * i / 256) * (tiles / i + 6) * tile_us + (i > 1 ? 4 + i * part_us : 0);
      if (i == 1 || t < best) {
        best = t;
        n = i;
      }
    }
    cut(n, pl.cut_tiles, pl.parts_tiles);
  }
  ch.join = (ch.rt && pl.parts_rows > 1) || (ch.tiles && pl.parts_tiles > 1);
  return ch;
}

// Rows of the two regions of parts.
struct PartRows {
  int64_t tiles, rows;
};

PartRows part_rows(const pp_attention_args& a, const Plan& pl, const Choice& ch) {
  PartRows n{0, 0};
  if (ch.tiles && pl.parts_tiles > 1) n.tiles = (int64_t)pl.parts_tiles * a.tokens * a.q_heads;
  if (ch.rt && pl.parts_rows > 1) n.rows = (int64_t)pl.parts_rows * a.requests * pl.few;
  return n;
}

template <bool F16, bool NARROW, int C, int RT>
hipError_t go_rows(const pp_kv_pages& p, const pp_attention_args& a, const Plan& pl, hipStream_t st) {
  constexpr int lds = LatentRows<NARROW, C>::kLds;
  static OnEachGpu once;
  const hipError_t ok = allow_lds(once, &k_latent_rows<F16, NARROW, C, RT>, lds);
  if (ok != hipSuccess) return ok;
  const int64_t grid = (int64_t)a.requests * pl.parts_rows;
  if (grid > INT32_MAX) return hipErrorInvalidConfiguration;
  k_latent_rows<F16, NARROW, C, RT><<<(unsigned)grid, 256, lds, st>>>(p, a, pl);
  return hipGetLastError();
}

template <bool F16, bool NARROW, int C>
hipError_t go(const pp_kv_pages& p, const pp_attention_args& a, const Plan& pl, const Choice& ch, hipStream_t st) {
  if (ch.tiles) {
    constexpr int lds = LatentTiles<NARROW, C>::kLds;
    static OnEachGpu once;
    const hipError_t ok = allow_lds(once, &k_latent_tiles<F16, NARROW, C>, lds);
    if (ok != hipSuccess) return ok;
    const int64_t grid = (int64_t)pl.slots * pl.parts_tiles;
    if (grid > INT32_MAX) return hipErrorInvalidConfiguration;
    k_latent_tiles<F16, NARROW, C><<<(unsigned)grid, 256, lds, st>>>(p, a, pl);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipError_t e = hipSuccess;
  if (ch.rt == 1) e = go_rows<F16, NARROW, C, 1>(p, a, pl, st);
  if (ch.rt == 2) e = go_rows<F16, NARROW, C, 2>(p, a, pl, st);
  if (e != hipSuccess) return e;
  if (ch.join) {
    int64_t few_rows = 0, waves = (int64_t)a.tokens * a.q_heads;
    if (pl.parts_tiles == 1) {
      few_rows = (int64_t)a.max_new * pl.group < pl.few ? (int64_t)a.max_new * pl.group : pl.few;
      waves = (int64_t)a.requests * few_rows;
    }
    k_join<F16, C><<<(unsigned)((waves + 3) / 4), 256, 0, st>>>(a, pl, (int32_t)few_rows, 1);
    e = hipGetLastError();
  }
  return e;
}

template <bool F16, bool NARROW>
hipError_t go_dim(const pp_kv_pages& p, int32_t value_dim, const pp_attention_args& a, const Plan& pl, const Choice& ch,
                  hipStream_t st) {
  if (value_dim == 512) return go<F16, NARROW, 512>(p, a, pl, ch, st);
  return go<F16, NARROW, 256>(p, a, pl, ch, st);
}

}  // namespace

int64_t latent_workspace(const pp_kv_pages& p, int32_t value_dim, const pp_attention_args& a) {
  Plan pl{};
  const Choice ch = choose(p, value_dim, a, pl);
  const PartRows n = part_rows(a, pl, ch);
  return (n.tiles + n.rows) * (value_dim + 1) * 4;
}

hipError_t launch_latent(const pp_kv_pages& p, int32_t value_dim, const pp_attention_args& a, hipStream_t st) {
  Plan pl{};
  const Choice ch = choose(p, value_dim, a, pl);
  pl.negative = a.scale < 0;
  pl.c = (a.scale < 0 ? -a.scale : a.scale) * kLog2e;
  pl.part = (float*)a.workspace;
  const PartRows n = part_rows(a, pl, ch);
  pl.row_part = pl.part + n.tiles * value_dim;
  pl.part_lse = pl.row_part + n.rows * value_dim;
  pl.row_lse = pl.part_lse + n.tiles;
  const bool narrow = p.dtype == PP_E4M3;
  if (a.dtype == PP_F16) return narrow ? go_dim<true, true>(p, value_dim, a, pl, ch, st) : go_dim<true, false>(p, value_dim, a, pl, ch, st);
  return narrow ? go_dim<false, true>(p, value_dim, a, pl, ch, st) : go_dim<false, false>(p, value_dim, a, pl, ch, st);
}

}  // namespace pp

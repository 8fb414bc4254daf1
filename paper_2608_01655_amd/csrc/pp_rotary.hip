// pp_rotary.hip -- norms, rotary positions and page writes in one pass (gfx950).
//
// y = x / sqrt(mean x^2 + eps) * weight, (a, b) -> amplitude (a cos t - b sin t, a sin t + b cos t), in 32 bits from
// the rows' read to their one rounding.  Bound by memory: a row is read once and written once, 16 bytes a lane, whatever
// is done to it between.  65,536 tokens of 32 query and 8 key heads of 128, half of each rotated, into 8-bit pages take
// 282 us, 1.48 GB at 5.2 TB/s, what a large copy reaches; rotation and write in torch operations 4,341.  61 tokens of
// 28 and 4 normed heads take 4.2 us, a chain of slot, row and store behind the launch, and 9.5 with the call's checks.

#include "pp_rows.h"

namespace pp {

namespace {

constexpr int kWave = 64;

// One kind of rows (queries, keys or values) and how a wave takes them: `lanes` lanes a row, two
// chunks of 8 elements a lane.  The chunks of a lane hold the pairs that rotate together, so a rotation
// needs no other lane: lane i < rot / 16 has chunks first / 8 + i and + rot / 16 (halves), or
// first / 8 + 2 i and the next (interleaved); the other lanes have the chunks that do not rotate.
struct Rows {
  const uint16_t *in, *weight;
  uint16_t* out;
  int64_t token, head, out_token, out_head;
  int32_t heads, chunks, first, norm, rot;    // the last four in chunks
  int32_t lanes_log2;
  int32_t groups;                             // wave's worth of rows a token
};

struct Work {
  Rows q, k, v;
  const int32_t* position;
  const uint64_t* turns;
  const int64_t* slot;
  int32_t tokens, interleaved, paged;
  int32_t groups, each, waves;                // a token's, a wave's, and waves a token
  int32_t shift;
  float eps, amplitude;
};

struct Angles {
  float c[8], s[8];
};

// position * turns modulo 2^64 is the angle exactly.  Its upper 32 bits are taken to the nearest quarter turn in
// whole numbers, and the rest, at most pi / 4, goes into the Taylor polynomials of sine and cosine (what they
// leave out is below 2^-28 and 2^-31): both are off by 2^-22 at most, at any position.
__device__ __forceinline__ void angle(uint64_t t, float& cosine, float& sine) {
  const uint32_t u = (uint32_t)(t >> 32) + 0x20000000u, quarter = u >> 30;
  const float x = (float)((int32_t)(u & 0x3fffffffu) - 0x20000000) * 1.4629180792671596e-9f;   // 2 pi / 2^32
  const float y = x * x;
  float s = __builtin_fmaf(y, 2.7557319e-6f, -1.9841270e-4f), c = __builtin_fmaf(y, -2.7557319e-7f, 2.4801587e-5f);
  s = __builtin_fmaf(y, s, 8.3333333e-3f);
  s = __builtin_fmaf(y, s, -1.6666667e-1f);
  s = __builtin_fmaf(x * y, s, x);
  c = __builtin_fmaf(y, c, -1.3888889e-3f);
  c = __builtin_fmaf(y, c, 4.1666667e-2f);
  c = __builtin_fmaf(y, c, -0.5f);
  c = __builtin_fmaf(y, c, 1.f);
  cosine = quarter & 1 ? s : c;
  sine = quarter & 1 ? c : s;
  if (quarter == 1 || quarter == 2) cosine = -cosine;
  if (quarter >= 2) sine = -sine;
}

__device__ __forceinline__ void angles(const Work& w, int32_t position, int lane, int32_t rot, Angles& a) {
  if (lane >= rot / 2) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    angle((uint64_t)(int64_t)position * w.turns[lane * 8 + j], a.c[j], a.s[j]);
    a.c[j] *= w.amplitude;
    a.s[j] *= w.amplitude;
  }
}

template <bool F16>
__device__ __forceinline__ void widen(i32x4 x, float* f) {
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] = widen1<F16>((uint16_t)(x[j / 2] >> (16 * (j % 2))));
}

// A lane's two chunks of its row of a group of one kind, for one token, as they are read.
struct Chunks {
  i32x4 x[2], w[2];
  int32_t at[2];       // their numbers
  int64_t to;          // their row's place, in elements
  int32_t head;
  bool has[2], turns, skipped;
};

template <bool TO_PAGES, bool PLAIN>
__device__ __forceinline__ Chunks read_chunks(const Work& w, const Rows& r, const pp_kv_pages& p, int32_t t, int32_t g) {
  Chunks c;
  const int lane = threadIdx.x % kWave, sub = lane & ((1 << r.lanes_log2) - 1);
  const int32_t h = (g << (6 - r.lanes_log2)) + (lane >> r.lanes_log2), turning = PLAIN ? 0 : r.rot;
  c.head = h;
  c.turns = sub < turning / 2;
  if (c.turns) {
    c.at[0] = r.first + (w.interleaved ? 2 * sub : sub);
    c.at[1] = c.at[0] + (w.interleaved ? 1 : turning / 2);
  } else {
    const int32_t u = 2 * (sub - turning / 2), first = PLAIN ? r.chunks : r.first;
    c.at[0] = u < first ? u : u + turning;
    c.at[1] = u + 1 < first ? u + 1 : u + 1 + turning;
  }
  const uint16_t* from = r.in + t * r.token + h * r.head;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    c.has[j] = h < r.heads && c.at[j] < r.chunks;
    c.x[j] = c.w[j] = i32x4{0, 0, 0, 0};
    if (c.has[j]) c.x[j] = *(const i32x4*)(from + c.at[j] * 8);
    if (!PLAIN && c.has[j] && c.at[j] < r.norm) c.w[j] = *(const i32x4*)(r.weight + c.at[j] * 8);
  }
  c.skipped = false;
  if (TO_PAGES) {
    const int64_t at = w.slot[t];
    c.skipped = at < 0 || at >> w.shift >= p.n_pages;        // for the whole wave
    c.to = (at >> w.shift) * p.page_stride + h * p.head_stride + (at & (p.page_size - 1)) * p.token_stride;
  } else {
    c.to = t * r.out_token + h * r.out_head;
  }
  return c;
}

template <bool F16, bool NARROW, bool PLAIN>
__device__ __forceinline__ void write_chunks(const Work& w, const Rows& r, const Chunks& c, void* base, const float* scales,
                                             const Angles& an) {
  if (c.skipped) return;
  if constexpr (PLAIN && !NARROW) {                           // as it is
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (c.has[j]) *(i32x4*)((uint16_t*)base + c.to + c.at[j] * 8) = c.x[j];
    return;
  }
  float y[16];
  widen<F16>(c.x[0], y);
  widen<F16>(c.x[1], y + 8);
  if (!PLAIN && r.norm) {
    float sum = 0;
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (c.has[j] && c.at[j] < r.norm)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(y[8 * j + i], y[8 * j + i], sum);
    for (int o = 1; o < 1 << r.lanes_log2; o <<= 1) sum += __shfl_xor(sum, o);
    const float f = 1.f / sqrtf(sum / (r.norm * 8) + w.eps);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (!(c.has[j] && c.at[j] < r.norm)) continue;
      float v[8];
      widen<F16>(c.w[j], v);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[8 * j + i] = y[8 * j + i] * f * v[i];
    }
  }
  if (!PLAIN && c.turns) {
    if (w.interleaved) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float x0 = y[2 * j], x1 = y[2 * j + 1];
        y[2 * j] = x0 * an.c[j] - x1 * an.s[j];
        y[2 * j + 1] = x0 * an.s[j] + x1 * an.c[j];
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float x0 = y[j], x1 = y[j + 8];
        y[j] = x0 * an.c[j] - x1 * an.s[j];
        y[j + 8] = x0 * an.s[j] + x1 * an.c[j];
      }
    }
  }
  const Scale s = scale_of(NARROW && scales && c.head < r.heads ? scales[c.head] : 1.f);
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    if (!c.has[j]) continue;
    if constexpr (NARROW) *(i32x2*)((uint8_t*)base + c.to + c.at[j] * 8) = narrow8(y + 8 * j, s);
    else *(i32x4*)((uint16_t*)base + c.to + c.at[j] * 8) = round8<F16>(y + 8 * j);
  }
}

template <bool F16, bool NARROW, bool PAGED>
__global__ void __launch_bounds__(256) k_rotary(Work w, pp_kv_pages p) {
  const int64_t id = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int32_t t = (int32_t)(id / w.waves);
  if (t >= w.tokens) return;
  const int32_t g0 = (int32_t)(id % w.waves) * w.each;
  const int32_t g1 = g0 + w.each < w.groups ? g0 + w.each : w.groups, kg = w.q.groups + w.k.groups;
  const int lane = threadIdx.x % kWave;
  const int32_t position = w.position ? w.position[t] : 0;
  Angles an;
  int32_t g = g0;
  // a group's rows are on their way before the angles are worked out
  for (; g < g1 && g < w.q.groups; ++g) {
    const Chunks c = read_chunks<false, false>(w, w.q, p, t, g);
    if (g == g0) angles(w, position, lane & ((1 << w.q.lanes_log2) - 1), w.q.rot, an);
    write_chunks<F16, false, false>(w, w.q, c, w.q.out, nullptr, an);
  }
  for (; g < g1 && g < kg; ++g) {
    const Chunks c = read_chunks<PAGED, false>(w, w.k, p, t, g - w.q.groups);
    if (g == g0 || (g == w.q.groups && w.k.lanes_log2 != w.q.lanes_log2))
      angles(w, position, lane & ((1 << w.k.lanes_log2) - 1), w.k.rot, an);
    write_chunks<F16, NARROW && PAGED, false>(w, w.k, c, PAGED ? p.k : w.k.out, PAGED ? p.k_scale : nullptr, an);
  }
  if constexpr (PAGED)
    for (; g < g1; ++g) {
      const Chunks c = read_chunks<true, true>(w, w.v, p, t, g - kg);
      write_chunks<F16, NARROW, true>(w, w.v, c, p.v, p.v_scale, an);
    }
}

int log2_up(int32_t n) {
  int l = 0;
  while (1 << l < n) ++l;
  return l;
}

Rows rows(const void* in, const void* weight, void* out, int64_t token, int64_t head, int64_t out_token, int64_t out_head,
          int32_t heads, int32_t dim, int32_t first, int32_t norm, int32_t rot) {
  Rows r{};
  r.in = (const uint16_t*)in;
  r.weight = (const uint16_t*)weight;
  r.out = (uint16_t*)out;
  r.token = token;
  r.head = head;
  r.out_token = out_token;
  r.out_head = out_head;
  r.heads = heads;
  r.chunks = dim / 8;
  r.first = first / 8;
  r.norm = norm / 8;
  r.rot = rot / 8;
  r.lanes_log2 = log2_up((r.chunks + 1) / 2);
  const int32_t per = 64 >> r.lanes_log2;
  r.groups = (heads + per - 1) / per;
  return r;
}

}  // namespace

hipError_t launch_rotary(const pp_rotary_args& a, const pp_kv_pages* pages, hipStream_t st) {
  Work w{};
  if (a.q_heads)
    w.q = rows(a.q, a.q_weight, a.q_out, a.q_token_stride, a.q_head_stride, a.q_out_token_stride, a.q_out_head_stride, a.q_heads,
               a.q_dim, a.q_first, a.q_norm, a.rot_dim);
  if (a.k_heads) {
    w.k = rows(a.k, a.k_weight, a.k_out, a.k_token_stride, a.k_head_stride, a.k_out_token_stride, a.k_out_head_stride, a.k_heads,
               a.k_dim, a.k_first, a.k_norm, a.rot_dim);
    if (a.v) w.v = rows(a.v, nullptr, nullptr, a.v_token_stride, a.v_head_stride, 0, 0, a.k_heads, a.k_dim, 0, 0, 0);
  }
  w.position = a.position;
  w.turns = a.turns;
  w.slot = a.slot_map;
  w.tokens = a.tokens;
  w.interleaved = a.interleaved;
  w.eps = a.eps;
  w.amplitude = a.amplitude;
  w.groups = w.q.groups + w.k.groups + w.v.groups;
  const int64_t most = (int64_t)a.tokens * w.groups;
  // A wave a group while there are few, so that a token's rows are not taken one after the other; else 8,192 waves at least,
  // and angles are worked out once a wave.
  int64_t each = most / 8192;
  w.each = (int32_t)(each < 1 ? 1 : each > w.groups ? w.groups : each);
  w.waves = (w.groups + w.each - 1) / w.each;
  pp_kv_pages p{};
  if (pages) {
    p = *pages;
    w.shift = __builtin_ctz(p.page_size);
  }
  const bool f16 = a.dtype == PP_F16, narrow = pages && p.dtype == PP_E4M3;
  auto kern = !pages ? (f16 ? k_rotary<true, false, false> : k_rotary<false, false, false>)
              : narrow ? (f16 ? k_rotary<true, true, true> : k_rotary<false, true, true>)
                       : (f16 ? k_rotary<true, false, true> : k_rotary<false, false, true>);
  // as many tokens at a time as a launch takes (waves are few where there are more)
  const int64_t turn = most_blocks(256) * 4 / w.waves;
  for (int64_t t = 0; t < a.tokens; t += turn) {
    w.tokens = (int32_t)(a.tokens - t < turn ? a.tokens - t : turn);
    kern<<<(unsigned)(((int64_t)w.tokens * w.waves + 3) / 4), 256, 0, st>>>(w, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (t + turn >= a.tokens) break;
    for (Rows* r : {&w.q, &w.k, &w.v}) {
      if (r->in) r->in += turn * r->token;
      if (r->out) r->out += turn * r->out_token;
    }
    if (w.position) w.position += turn;
    if (w.slot) w.slot += turn;
  }
  return hipSuccess;
}

}  // namespace pp

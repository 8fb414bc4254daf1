// pp_attend.hip -- attention of new tokens over paged keys and values (gfx950).

#include "pp_serve.h"

namespace pp {

namespace {

constexpr int kWave = 64;

__device__ __forceinline__ float widen(const void* p, int64_t i, int32_t type) {
  if (type == PP_F16) return (float)((const _Float16*)p)[i];
  if (type == PP_BF16) return __builtin_bit_cast(float, (uint32_t)((const uint16_t*)p)[i] << 16);
  return __builtin_amdgcn_cvt_f32_fp8(((const uint8_t*)p)[i], 0);
}

// One wave a (token, query head), key by key.
__global__ void __launch_bounds__(kWave) k_attend_row(pp_kv_pages p, pp_attention_args a, int shift) {
  const int lane = threadIdx.x;
  const int32_t t = blockIdx.x / a.q_heads, g = blockIdx.x % a.q_heads;
  int32_t r = 0;
  while (r + 1 < a.requests && a.query_start[r + 1] <= t) ++r;
  const int32_t first = a.query_start[r], u = a.query_start[r + 1] - first;
  if (t < first || t >= first + u) return;
  const int64_t room = (int64_t)a.max_blocks << shift;
  const int32_t pos = a.length[r] - u + (t - first);
  const int h = g / (a.q_heads / p.heads);
  const int64_t from = a.window && pos >= a.window ? pos - a.window + 1 : 0;
  const int64_t to = pos + 1 < room ? pos + 1 : room;
  const float ks = p.k_scale ? p.k_scale[h] : 1.f, vs = p.v_scale ? p.v_scale[h] : 1.f;
  float q[4], o[4] = {0, 0, 0, 0}, m = -INFINITY, l = 0;
  for (int j = 0; j < p.dim / kWave; ++j)
    q[j] = widen(a.q, t * a.q_token_stride + g * a.q_head_stride + j * kWave + lane, a.dtype);
  for (int64_t k = from; k < to; ++k) {
    int32_t page = a.block_table[r * a.row_stride + (k >> shift)];
    page = page < 0 ? 0 : page < p.n_pages ? page : p.n_pages - 1;
    const int64_t at = page * p.page_stride + h * p.head_stride +
                       (k & (p.page_size - 1)) * p.token_stride + lane;
    float s = 0;
    for (int j = 0; j < p.dim / kWave; ++j) s += q[j] * widen(p.k, at + j * kWave, p.dtype);
    for (int x = kWave / 2; x; x >>= 1) s += __shfl_xor(s, x);
    s *= a.scale * ks;
    const float n = fmaxf(m, s);
    if (n == -INFINITY && s == s) continue;
    const float w = m == -INFINITY ? 0.f : expf(m - n), e = expf(s - n);
    l = l * w + e;
    for (int j = 0; j < p.dim / kWave; ++j) o[j] = o[j] * w + e * widen(p.v, at + j * kWave, p.dtype);
    m = n;
  }
  for (int j = 0; j < p.dim / kWave; ++j) {
    const float x = l == 0 ? 0.f : o[j] / l * vs;
    const int64_t i = t * a.out_token_stride + g * a.out_head_stride + j * kWave + lane;
    if (a.dtype == PP_F16) ((_Float16*)a.out)[i] = (_Float16)x;
    else ((__bf16*)a.out)[i] = (__bf16)x;
  }
  if (a.lse && lane == 0) a.lse[(int64_t)t * a.q_heads + g] = l == 0 ? -INFINITY : m + logf(l);
}

}  // namespace

int64_t attention_workspace(const pp_kv_pages&, const pp_attention_args&) { return 0; }

hipError_t launch_attention(const pp_kv_pages& p, const pp_attention_args& a, hipStream_t st) {
  k_attend_row<<<a.tokens * a.q_heads, kWave, 0, st>>>(p, a, __builtin_ctz(p.page_size));
  return hipGetLastError();
}

}  // namespace pp

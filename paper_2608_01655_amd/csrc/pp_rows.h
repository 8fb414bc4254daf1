// pp_rows.h -- device helpers of the kernels that write rows into pages: widening, rounding and
// scaling of elements.
#pragma once

#include "pp_serve.h"

namespace pp {

namespace {

typedef __attribute__((__vector_size__(16))) int i32x4;
typedef __attribute__((__vector_size__(8))) int i32x2;

template <bool F16>
__device__ __forceinline__ float widen1(uint16_t x) {
  if constexpr (F16) return (float)__builtin_bit_cast(_Float16, x);
  else return __builtin_bit_cast(float, (uint32_t)x << 16);
}

// Two values rounded to nearest into the rows' type, eight of them.
template <bool F16>
__device__ __forceinline__ i32x4 round8(const float* y) {
  typedef __attribute__((__vector_size__(4))) __bf16 bf16x2;
  typedef __attribute__((__vector_size__(4))) _Float16 f16x2;
  i32x4 o;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (F16) o[j] = __builtin_bit_cast(int, f16x2{(_Float16)y[2 * j], (_Float16)y[2 * j + 1]});
    else o[j] = __builtin_bit_cast(int, bf16x2{(__bf16)y[2 * j], (__bf16)y[2 * j + 1]});
  }
  return o;
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

// Eight values / scale as e4m3.
__device__ __forceinline__ i32x2 narrow8(const float* x, const Scale& s) {
  float f[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] = shrink(x[j], s);
  i32x2 o;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int q = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * j], f[4 * j + 1], 0, false);
    o[j] = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * j + 2], f[4 * j + 3], q, true);
  }
  return o;
}

}  // namespace

}  // namespace pp

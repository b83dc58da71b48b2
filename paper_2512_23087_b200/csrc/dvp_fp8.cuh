// 8-bit values of a block that shares a scale: q = e4m3(y / c), the float32 quotient rounded to nearest, ties to even.
#pragma once

#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace dvp {
namespace fp8 {

constexpr float kMax = 448.f;              // the largest value
constexpr float kLeastAmax = 1.262177448e-29f;  // 2^-96: a block of zeros has a scale that can be divided by

__device__ __forceinline__ float scale_of(float amax) { return amax / kMax; }

__device__ __forceinline__ uint32_t pair_of(float lo, float hi) {
  return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}

// Two products with one factor.
__device__ __forceinline__ uint32_t pair_of_products(float lo, float hi, float r) {
  asm("{\n\t.reg .b64 v, f;\n\t"
      "mov.b64 v, {%0, %1};\n\t"
      "mov.b64 f, {%2, %2};\n\t"
      "mul.rn.f32x2 v, v, f;\n\t"
      "mov.b64 {%0, %1}, v;\n\t}"
      : "+f"(lo), "+f"(hi)
      : "f"(r));
  return pair_of(lo, hi);
}
static __device__ __noinline__ uint32_t divided(float a, float b, float c, float d, float by) {
  return pair_of(a / by, b / by) | pair_of(c / by, d / by) << 16;
}

// Eight or four quotients.  The conversion is monotone, so where products with a bound of 1 / c on either side become the same value, the
// quotient does too: the special-function unit's reciprocal is good to 2^-23, two roundings on the way add 2^-24 each, and the
// quotient's own is one more, less than the 2^-21 between the bounds and it.  Only what lies so near a border is divided:
// one four in some twenty thousand (16,384 x 4,096 bfloat16, norm to 8 bits: 111 us; with a division each 131; with products by the
// approximate reciprocal alone, which put some values on the border's other side, 102).
template <int N>
__device__ __forceinline__ void quotients(const float (&y)[N], float c, uint32_t (&q)[N / 4]) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(c));
  const float under = r * (1.f - 4.76837158203125e-7f), over = r * (1.f + 4.76837158203125e-7f);  // 2^-21
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const float a = y[4 * i], b = y[4 * i + 1], d = y[4 * i + 2], e = y[4 * i + 3];
    q[i] = pair_of_products(a, b, under) | pair_of_products(d, e, under) << 16;
    if (q[i] != (pair_of_products(a, b, over) | pair_of_products(d, e, over) << 16)) q[i] = divided(a, b, d, e, c);
  }
}

}  // namespace fp8
}  // namespace dvp

// The 8-bit float format of the block-scaled path (trdq_fp8_*): e4m3 codes, one fp32 scale per 128 consecutive channels
// of a row (activations) or per 128 x 128 block (weights).
//   a = max |v| over the block,   scale = fl(a * fl(1/448)),   code = e4m3(fl(v * fl(448 * fl(1/a))))
// 448 is the largest e4m3 number, the conversion rounds to nearest with ties to even.  One division per block; the two roundings of the factor move
// v by 2^-23 of its value, and the block's largest value always becomes 448 or -448.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace trdq {

constexpr float kFp8Max = 448.0f;
constexpr float kFp8InvMax = 1.0f / 448.0f;
// Block maxima below 2^-100 are scaled as if they were 2^-100: the factor stays finite (and a product with a zero a zero).
constexpr float kFp8Tiny = 7.888609052210118e-31f;

struct Fp8Factor {
  float scale;  // stored: value = code * scale
  float mul;    // v * mul is rounded to the code
};
// amax: the block's maximum; a NaN among the values leaves no trace in it, but becomes a NaN code by itself.
__device__ __forceinline__ Fp8Factor fp8_factor(float amax) {
  const float a = fmaxf(amax, kFp8Tiny);
  return Fp8Factor{amax > 0.0f ? __fmul_rn(a, kFp8InvMax) : 0.0f, __fmul_rn(__frcp_rn(a), kFp8Max)};
}

// Two codes, lo in the low byte; magnitudes beyond 448 (one rounding of v * mul) become 448.
__device__ __forceinline__ uint32_t fp8_pack2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t fp8_pack4(float2 a, float2 b) {
  return __byte_perm(fp8_pack2(a.x, a.y), fp8_pack2(b.x, b.y), 0x5410);
}

}  // namespace trdq

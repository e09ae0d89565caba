// Pieces shared by the forward and the backward kernel of trdq_gated_norm: rows in 16-byte chunks of eight channels, and sums over the
// warps that hold a row.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "internal.h"

namespace trdq {

// Eight channels as fp32 pairs.
struct Chunk {
  float2 p[4];
};

__device__ __forceinline__ float2 widen_bf16x2(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
__device__ __forceinline__ Chunk widen(const uint4& w) { return Chunk{{widen_bf16x2(w.x), widen_bf16x2(w.y), widen_bf16x2(w.z), widen_bf16x2(w.w)}}; }
__device__ __forceinline__ uint32_t narrow_bf16x2(float2 v) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint4 narrow(const Chunk& c) {
  return make_uint4(narrow_bf16x2(c.p[0]), narrow_bf16x2(c.p[1]), narrow_bf16x2(c.p[2]), narrow_bf16x2(c.p[3]));
}
__device__ __forceinline__ uint4 zero4() { return make_uint4(0u, 0u, 0u, 0u); }

// A chunk of the residual stream (bf16 or fp32) as it lies in memory.
template <bool F32>
struct StreamChunk;
template <>
struct StreamChunk<false> {
  uint4 w;
  __device__ __forceinline__ void clear() { w = zero4(); }
  __device__ __forceinline__ void load(const void* row, int chunk) { w = *(static_cast<const uint4*>(row) + chunk); }
  __device__ __forceinline__ void store(void* row, int chunk) const { *(static_cast<uint4*>(row) + chunk) = w; }
  __device__ __forceinline__ Chunk value() const { return widen(w); }
  __device__ __forceinline__ void set(const Chunk& c) { w = narrow(c); }  // rounds
};
template <>
struct StreamChunk<true> {
  float4 lo, hi;
  __device__ __forceinline__ void clear() { lo = hi = make_float4(0.0f, 0.0f, 0.0f, 0.0f); }
  __device__ __forceinline__ void load(const void* row, int chunk) {
    lo = *(static_cast<const float4*>(row) + 2 * chunk);
    hi = *(static_cast<const float4*>(row) + 2 * chunk + 1);
  }
  __device__ __forceinline__ void store(void* row, int chunk) const {
    *(static_cast<float4*>(row) + 2 * chunk) = lo;
    *(static_cast<float4*>(row) + 2 * chunk + 1) = hi;
  }
  __device__ __forceinline__ Chunk value() const {
    return Chunk{{make_float2(lo.x, lo.y), make_float2(lo.z, lo.w), make_float2(hi.x, hi.y), make_float2(hi.z, hi.w)}};
  }
  __device__ __forceinline__ void set(const Chunk& c) {
    lo = make_float4(c.p[0].x, c.p[0].y, c.p[1].x, c.p[1].y);
    hi = make_float4(c.p[2].x, c.p[2].y, c.p[3].x, c.p[3].y);
  }
};

__device__ __forceinline__ const void* stream_row(const void* base, int64_t row, int64_t ld, bool f32) {
  return static_cast<const char*>(base) + row * ld * (f32 ? 4 : 2);
}
__device__ __forceinline__ void* stream_row(void* base, int64_t row, int64_t ld, bool f32) { return static_cast<char*>(base) + row * ld * (f32 ? 4 : 2); }

// Chunk of a bf16 parameter row that may be absent.
__device__ __forceinline__ uint4 load_param(const uint16_t* row, int chunk) { return __ldg(reinterpret_cast<const uint4*>(row) + chunk); }

__device__ __forceinline__ float chunk_sum(const Chunk& c) {
  const float2 s = __fadd2_rn(__fadd2_rn(c.p[0], c.p[1]), __fadd2_rn(c.p[2], c.p[3]));
  return __fadd_rn(s.x, s.y);
}
__device__ __forceinline__ float chunk_dot(const Chunk& a, const Chunk& b) {
  float2 s = __fmul2_rn(a.p[0], b.p[0]);
#pragma unroll
  for (int i = 1; i < 4; ++i) s = __ffma2_rn(a.p[i], b.p[i], s);
  return __fadd_rn(s.x, s.y);
}
__device__ __forceinline__ Chunk chunk_mul(const Chunk& a, const Chunk& b) {
  Chunk r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.p[i] = __fmul2_rn(a.p[i], b.p[i]);
  return r;
}
__device__ __forceinline__ Chunk chunk_scale(const Chunk& a, float f) {
  const float2 f2 = make_float2(f, f);
  return Chunk{{__fmul2_rn(a.p[0], f2), __fmul2_rn(a.p[1], f2), __fmul2_rn(a.p[2], f2), __fmul2_rn(a.p[3], f2)}};
}
__device__ __forceinline__ Chunk chunk_shift(const Chunk& a, float d) {
  const float2 d2 = make_float2(d, d);
  return Chunk{{__fadd2_rn(a.p[0], d2), __fadd2_rn(a.p[1], d2), __fadd2_rn(a.p[2], d2), __fadd2_rn(a.p[3], d2)}};
}
__device__ __forceinline__ Chunk chunk_fma(const Chunk& a, const Chunk& b, const Chunk& c) {
  Chunk r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.p[i] = __ffma2_rn(a.p[i], b.p[i], c.p[i]);
  return r;
}

// Sums over the W warps that hold a row, in a fixed order, the result in every lane.  `slots`: shared, 2 x NV x W floats of this
// team; consecutive sums alternate between the two halves, so that one barrier a sum is enough.
template <int W>
struct TeamSum {
  float* slots;
  int team, warp;  // of the team, of the warp in it
  int turn = 0;
  static constexpr int kMost = 2;  // values summed at once
  static constexpr int kFloats = 2 * kMost * W;
  __device__ __forceinline__ TeamSum(float* s, int t, int w) : slots(s), team(t), warp(w) {}
  template <int NV>
  __device__ __forceinline__ void sum(float (&v)[NV]) {
    static_assert(NV <= kMost, "slots");
#pragma unroll
    for (int d = 16; d > 0; d >>= 1)
#pragma unroll
      for (int i = 0; i < NV; ++i) v[i] = __fadd_rn(v[i], __shfl_xor_sync(0xffffffffu, v[i], d));
    if constexpr (W > 1) {
      float* const here = slots + turn * kMost * W;
      turn ^= 1;
      if ((threadIdx.x & 31) == 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) here[i * W + warp] = v[i];
      }
      asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "n"(32 * W) : "memory");
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        float s = here[i * W];
#pragma unroll
        for (int k = 1; k < W; ++k) s = __fadd_rn(s, here[i * W + k]);
        v[i] = s;
      }
    }
  }
  __device__ __forceinline__ float sum(float a) {
    float v[1] = {a};
    sum(v);
    return v[0];
  }
};

}  // namespace trdq

// Pieces shared by the forward and the backward kernel of trdq_gated_norm: rows in 16-byte chunks of eight channels and sums over the
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
  __device__ __forceinline__ void load(const void* at) { w = *static_cast<const uint4*>(at); }
  __device__ __forceinline__ void load_pieces(const float4* at, int) { load(at); }  // 16-byte pieces, `step` of them from one to the next
  __device__ __forceinline__ void store(void* at) const { *static_cast<uint4*>(at) = w; }
  __device__ __forceinline__ Chunk value() const { return widen(w); }
  __device__ __forceinline__ void set(const Chunk& c) { w = narrow(c); }  // rounds
};
template <>
struct StreamChunk<true> {
  float4 lo, hi;
  __device__ __forceinline__ void clear() { lo = hi = make_float4(0.0f, 0.0f, 0.0f, 0.0f); }
  __device__ __forceinline__ void load(const void* at) {
    lo = static_cast<const float4*>(at)[0];
    hi = static_cast<const float4*>(at)[1];
  }
  __device__ __forceinline__ void load_pieces(const float4* at, int step) {
    lo = at[0];
    hi = at[step];
  }
  __device__ __forceinline__ void store(void* at) const {
    static_cast<float4*>(at)[0] = lo;
    static_cast<float4*>(at)[1] = hi;
  }
  __device__ __forceinline__ Chunk value() const {
    return Chunk{{make_float2(lo.x, lo.y), make_float2(lo.z, lo.w), make_float2(hi.x, hi.y), make_float2(hi.z, hi.w)}};
  }
  __device__ __forceinline__ void set(const Chunk& c) {
    lo = make_float4(c.p[0].x, c.p[0].y, c.p[1].x, c.p[1].y);
    hi = make_float4(c.p[2].x, c.p[2].y, c.p[3].x, c.p[3].y);
  }
};

__device__ __forceinline__ const char* stream_at(const void* base, int64_t row, int64_t ld, int chunk, bool f32) {
  return static_cast<const char*>(base) + (row * ld + 8 * chunk) * (f32 ? 4 : 2);
}
__device__ __forceinline__ char* stream_at(void* base, int64_t row, int64_t ld, int chunk, bool f32) {
  return static_cast<char*>(base) + (row * ld + 8 * chunk) * (f32 ? 4 : 2);
}

// Chunk of a bf16 parameter row that may be absent.
__device__ __forceinline__ uint4 load_param(const uint16_t* row, int chunk) { return __ldg(reinterpret_cast<const uint4*>(row) + chunk); }

__device__ __forceinline__ void prefetch_l1(const void* at) { asm volatile("prefetch.global.L1 [%0];" ::"l"(at)); }

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

// A CTA holds one row: CH chunks a thread, thread t the chunks t, t + blockDim.x.
constexpr int kRowWarps = 16;  // most warps of a CTA; with two chunks a thread D <= 8192

inline int row_chunks(int32_t D) { return D / 8 > 32 * kRowWarps ? 2 : 1; }
inline int row_threads(int32_t D) { return (D / 8 + 32 * row_chunks(D) - 1) / (32 * row_chunks(D)) * 32; }

// Sums over a row, in a fixed order: the lanes of a warp, then the warps through shared memory with one barrier.  Consecutive sums of a kind
// use different halves of its slots, so that a half is not written again before every warp has passed a barrier behind its last reading.
struct RowSum {
  static constexpr int kSlots = 2 * (kRowWarps / 4) + 2 * (kRowWarps / 2);
  float4* slots;  // [2][kRowWarps / 4] one value a warp, [2][kRowWarps / 2] two values; zeros for the warps that are not there
  int warps, turn1 = 0, turn2 = 0;
  __device__ __forceinline__ explicit RowSum(float4* s) : slots(s), warps(static_cast<int>(blockDim.x) >> 5) {
    if (threadIdx.x < kSlots) s[threadIdx.x] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    __syncthreads();
  }
  static __device__ __forceinline__ float4 add(const float4& a, const float4& b) {
    return make_float4(__fadd_rn(a.x, b.x), __fadd_rn(a.y, b.y), __fadd_rn(a.z, b.z), __fadd_rn(a.w, b.w));
  }
  __device__ __forceinline__ float one(float v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v = __fadd_rn(v, __shfl_xor_sync(0xffffffffu, v, d));
    if (warps == 1) return v;
    float4* const here = slots + turn1;
    turn1 ^= kRowWarps / 4;
    if ((threadIdx.x & 31) == 0) reinterpret_cast<float*>(here)[threadIdx.x >> 5] = v;
    __syncthreads();
    float4 s = here[0];
    for (int k = 4; k < warps; k += 4) s = add(s, here[k >> 2]);
    return __fadd_rn(__fadd_rn(s.x, s.z), __fadd_rn(s.y, s.w));
  }
  __device__ __forceinline__ float2 two(float2 v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v = __fadd2_rn(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, d), __shfl_xor_sync(0xffffffffu, v.y, d)));
    if (warps == 1) return v;
    float4* const here = slots + 2 * (kRowWarps / 4) + turn2;
    turn2 ^= kRowWarps / 2;
    if ((threadIdx.x & 31) == 0) reinterpret_cast<float2*>(here)[threadIdx.x >> 5] = v;
    __syncthreads();
    float4 s = here[0];
    for (int k = 2; k < warps; k += 2) s = add(s, here[k >> 1]);
    return make_float2(__fadd_rn(s.x, s.z), __fadd_rn(s.y, s.w));
  }
};
static_assert(RowSum::kSlots <= 32, "a CTA of one warp clears the slots");

// 1 / sqrt(a) for a > 0 to about one unit of the last place: the hardware's estimate and a Newton step.  0 and infinity as they come.
__device__ __forceinline__ float inverse_root(float a) {
  const float y = rsqrtf(a);
  const float e = __fmaf_rn(__fmul_rn(-a, y), y, 1.0f);
  return a > 0.0f && a < __uint_as_float(0x7F800000u) ? __fmaf_rn(__fmul_rn(0.5f, e), y, y) : y;
}

// v -> v - mean (LayerNorm) or v (root mean square); returns 1 / sqrt(mean square of the result + eps).  Chunks outside the row (`in` false) are
// zero and stay so.  Two sums and not one of (mean, squared deviations) per warp joined afterwards, which saves a barrier but costs
// more instructions than it hides.
template <int CH>
__device__ __forceinline__ float row_centre(Chunk (&v)[CH], const bool (&in)[CH], int kind, float inv_d, float eps, RowSum& row) {
  if (kind == TRDQ_NORM_LAYER) {
    float s = chunk_sum(v[0]);
#pragma unroll
    for (int j = 1; j < CH; ++j) s = __fadd_rn(s, chunk_sum(v[j]));
    const float mean = __fmul_rn(row.one(s), inv_d);
#pragma unroll
    for (int j = 0; j < CH; ++j) v[j] = chunk_shift(v[j], in[j] ? -mean : 0.0f);
  }
  float q = chunk_dot(v[0], v[0]);
#pragma unroll
  for (int j = 1; j < CH; ++j) q = __fadd_rn(q, chunk_dot(v[j], v[j]));
  return inverse_root(__fmaf_rn(row.one(q), inv_d, eps));
}

}  // namespace trdq

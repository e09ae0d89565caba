// bf16 -> block-scaled e4m3 (fp8.cuh), plain or behind the rotation of Eq. 10: activations with a scale per row and 128 channels,
// weights with a scale per 128 x 128 block.  The rotation's block is the scale's block, so nothing but the block itself has
// to be known before its codes are written: no reduction over a row, one pass.
//
// Four lanes own one block of one row (lane_group.cuh: 32 values each as fp32 pairs, three butterfly stages in a thread, two by
// shuffle, two more in the thread).
#include <algorithm>

#include "fp8.cuh"
#include "internal.h"
#include "lane_group.cuh"
#include "ptx.cuh"

namespace trdq {
namespace {

constexpr int kThreads = 256;
constexpr int kRowsPerWarp = 32 / kFastLanes;

__device__ __forceinline__ void fp8_store_lanes4(const float2 (&v)[16], float mul, uint8_t* dst) {
  const float2 mul2 = make_float2(mul, mul);
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    float2 q[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = __fmul2_rn(v[4 * c + j], mul2);
    *reinterpret_cast<uint2*>(dst + 32 * c) = make_uint2(fp8_pack4(q[0], q[1]), fp8_pack4(q[2], q[3]));
  }
}

__device__ __forceinline__ void load_chunks(const uint16_t* src, bool valid, uint4 (&raw)[4]) {
#pragma unroll
  for (int c = 0; c < 4; ++c) raw[c] = valid ? __ldg(reinterpret_cast<const uint4*>(src) + 4 * c) : make_uint4(0u, 0u, 0u, 0u);
}

// A warp takes one 128-block of `steps` times eight consecutive rows: its lanes share the block's part of the fused vector, which stays in registers, and
// the eight scales of a step are consecutive floats of scales[b][m].  The next step's values are requested before this one's are used.  Plain it is bound by
// memory (5.8 TB/s at 32768 x 1152); rotated by instruction issue, 144 packed operations on 32 values beside 64 shuffles (24.9 us, 4.6 TB/s; read again
// for each step the vector cost as much of the first-level cache as the values: 28.6 us).  Two CTAs an SM: with the registers of three it spills, 38 us.
template <bool ROTATE>
__global__ void __launch_bounds__(kThreads, 2) fp8_quantize_kernel(const uint16_t* __restrict__ x, int64_t ldx, int32_t M, int32_t K,
                                                                const float* __restrict__ vec, uint8_t* __restrict__ codes,
                                                                float* __restrict__ scales, int32_t steps) {
  const int nb = K / TRDQ_BLOCK;
  const int lane4 = threadIdx.x & (kFastLanes - 1);
  const int64_t item = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) >> 5;
  const int b = static_cast<int>(item % nb);
  int64_t row = item / nb * kRowsPerWarp * steps + ((threadIdx.x & 31) / kFastLanes);
  const int col0 = b * TRDQ_BLOCK + lane4 * 8;
  griddep_launch_dependents();
  griddep_wait();  // x may be written, and the codes still read, by the kernel before
  uint4 raw[4];
  load_chunks(x + row * ldx + col0, row < M, raw);
  float2 by[16];
  if constexpr (ROTATE) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float4 f = __ldg(reinterpret_cast<const float4*>(vec + col0 + 32 * c) + h);
        by[4 * c + 2 * h] = make_float2(f.x, f.y);
        by[4 * c + 2 * h + 1] = make_float2(f.z, f.w);
      }
    }
  }
  for (int i = 0; i < steps; ++i, row += kRowsPerWarp) {
    float2 v[16];
    widen_chunks_lanes4(raw, v);
    if (i + 1 < steps) load_chunks(x + (row + kRowsPerWarp) * ldx + col0, row + kRowsPerWarp < M, raw);
    if constexpr (ROTATE) {
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] = __fmul2_rn(v[j], by[j]);
      wht128_lanes4(v, lane4);
    }
    const Fp8Factor f = fp8_factor(absmax_lanes4(v));
    if (row < M) {
      fp8_store_lanes4(v, f.mul, codes + row * K + col0);
      if (lane4 == 0) scales[static_cast<int64_t>(b) * M + row] = f.scale;
    }
  }
}

// One CTA per 128 x 128 block of the weights, four threads a row: the scale needs the whole block, which stays in registers meanwhile.  4608 x 1152: 6.6 us, the
// launch, two latencies and the issue of the 324 blocks on 148 SMs.  (Registers for three CTAs an SM instead of two: spills, 7.3 us.
// A block in clusters of four CTAs, for a finer grain: 7.8 us, 16384 x 4096 69 instead of 57.)
template <bool ROTATE>
__global__ void __launch_bounds__(512) fp8_quantize_weights_kernel(const uint16_t* __restrict__ w, int32_t N, int32_t K, const float* __restrict__ vec,
                                                                   uint8_t* __restrict__ codes, float* __restrict__ scales) {
  __shared__ float warp_max[16];
  const int nb = K / TRDQ_BLOCK;
  const int lane4 = threadIdx.x & (kFastLanes - 1);
  const int kb = blockIdx.x % nb, rb = blockIdx.x / nb;
  const int64_t row = static_cast<int64_t>(rb) * TRDQ_BLOCK + threadIdx.x / kFastLanes;
  const bool valid = row < N;
  const int col0 = kb * TRDQ_BLOCK + lane4 * 8;
  griddep_launch_dependents();
  griddep_wait();
  uint4 raw[4];
  load_chunks(w + row * K + col0, valid, raw);
  float2 v[16];
  if constexpr (ROTATE) {
    scale_chunks_lanes4(raw, reinterpret_cast<const float2*>(vec + col0), v);
    wht128_lanes4(v, lane4);
  } else {
    widen_chunks_lanes4(raw, v);
  }
  float m = absmax_lanes4(v);
  for (int d = 4; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
  if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = m;
  __syncthreads();
  m = warp_max[threadIdx.x & 15];
  for (int d = 1; d < 16; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
  const Fp8Factor f = fp8_factor(m);
  if (valid) fp8_store_lanes4(v, f.mul, codes + row * K + col0);
  if (threadIdx.x == 0) scales[blockIdx.x] = f.scale;
}

}  // namespace

trdq_status launch_fp8_quantize(const void* x_bf16, int64_t ldx, int32_t M, int32_t K, const float* vec, uint8_t* codes, float* scales,
                                cudaStream_t stream) {
  const int64_t groups = (static_cast<int64_t>(M) + kRowsPerWarp - 1) / kRowsPerWarp;
  // More steps a warp while every SM still has its sixteen warps.  Eight against one: 32768 x 1152 rotated 24.9 us, 36.8; plain, where there is no vector
  // to keep, four: 19.8 us, 21.8 for one and 23.0 for eight.
  int32_t steps = 1;
  while (steps < (vec ? 8 : 4) && groups * (K / TRDQ_BLOCK) / (2 * steps) >= 148 * 16) steps *= 2;
  const int64_t warps = (groups + steps - 1) / steps * (K / TRDQ_BLOCK);
  const int64_t grid = (warps * 32 + kThreads - 1) / kThreads;
  if (grid > 0x7FFFFFFF) return TRDQ_ERR_SHAPE;
  const cudaError_t e = launch_overlapped(vec ? fp8_quantize_kernel<true> : fp8_quantize_kernel<false>, dim3(static_cast<unsigned>(grid)), dim3(kThreads), 0,
                                          stream, static_cast<const uint16_t*>(x_bf16), ldx, M, K, vec, codes, scales, steps);
  return e == cudaSuccess ? TRDQ_OK : TRDQ_ERR_CUDA;
}

trdq_status launch_fp8_quantize_weights(const void* w_bf16, int32_t N, int32_t K, const float* vec, uint8_t* codes, float* scales,
                                        cudaStream_t stream) {
  const int64_t grid = (static_cast<int64_t>(N) + TRDQ_BLOCK - 1) / TRDQ_BLOCK * (K / TRDQ_BLOCK);
  if (grid > 0x7FFFFFFF) return TRDQ_ERR_SHAPE;
  const cudaError_t e = launch_overlapped(vec ? fp8_quantize_weights_kernel<true> : fp8_quantize_weights_kernel<false>, dim3(static_cast<unsigned>(grid)),
                                          dim3(512), 0, stream, static_cast<const uint16_t*>(w_bf16), N, K, vec, codes, scales);
  return e == cudaSuccess ? TRDQ_OK : TRDQ_ERR_CUDA;
}

}  // namespace trdq

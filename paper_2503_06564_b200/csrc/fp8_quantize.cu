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

// A warp takes one 128-block of eight consecutive rows: its lanes share the block's part of the fused vector, and its eight
// scales are consecutive floats of scales[b][m].
template <bool ROTATE>
__global__ void __launch_bounds__(kThreads) fp8_quantize_kernel(const uint16_t* __restrict__ x, int64_t ldx, int32_t M, int32_t K,
                                                                const float* __restrict__ vec, uint8_t* __restrict__ codes,
                                                                float* __restrict__ scales) {
  const int nb = K / TRDQ_BLOCK;
  const int lane4 = threadIdx.x & (kFastLanes - 1);
  const int64_t item = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) >> 5;
  const int b = static_cast<int>(item % nb);
  const int64_t row = item / nb * kRowsPerWarp + ((threadIdx.x & 31) / kFastLanes);
  const bool valid = row < M;
  const int col0 = b * TRDQ_BLOCK + lane4 * 8;
  griddep_launch_dependents();
  griddep_wait();  // x may be written, and the codes still read, by the kernel before
  uint4 raw[4];
  load_chunks(x + row * ldx + col0, valid, raw);
  float2 v[16];
  if constexpr (ROTATE) {
    scale_chunks_lanes4(raw, reinterpret_cast<const float2*>(vec + col0), v);
    wht128_lanes4(v, lane4);
  } else {
    widen_chunks_lanes4(raw, v);
  }
  const Fp8Factor f = fp8_factor(absmax_lanes4(v));
  if (!valid) return;
  fp8_store_lanes4(v, f.mul, codes + row * K + col0);
  if (lane4 == 0) scales[static_cast<int64_t>(b) * M + row] = f.scale;
}

// One CTA per 128 x 128 block of the weights, four threads a row.
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
  const int64_t warps = (static_cast<int64_t>(M) + kRowsPerWarp - 1) / kRowsPerWarp * (K / TRDQ_BLOCK);
  const int64_t grid = (warps * 32 + kThreads - 1) / kThreads;
  if (grid > 0x7FFFFFFF) return TRDQ_ERR_SHAPE;
  const cudaError_t e = launch_overlapped(vec ? fp8_quantize_kernel<true> : fp8_quantize_kernel<false>, dim3(static_cast<unsigned>(grid)), dim3(kThreads), 0,
                                          stream, static_cast<const uint16_t*>(x_bf16), ldx, M, K, vec, codes, scales);
  return e == cudaSuccess ? TRDQ_OK : TRDQ_ERR_CUDA;
}

trdq_status launch_fp8_quantize_weights(const void* w_bf16, int32_t N, int32_t K, const float* vec, uint8_t* codes, float* scales,
                                        cudaStream_t stream) {
  const int64_t grid = (static_cast<int64_t>(N) + TRDQ_BLOCK - 1) / TRDQ_BLOCK * (K / TRDQ_BLOCK);
  if (grid > 0x7FFFFFFF) return TRDQ_ERR_SHAPE;
  const auto kernel = vec ? fp8_quantize_weights_kernel<true> : fp8_quantize_weights_kernel<false>;
  kernel<<<static_cast<unsigned>(grid), 512, 0, stream>>>(static_cast<const uint16_t*>(w_bf16), N, K, vec, codes, scales);
  return cudaGetLastError() == cudaSuccess ? TRDQ_OK : TRDQ_ERR_CUDA;
}

}  // namespace trdq

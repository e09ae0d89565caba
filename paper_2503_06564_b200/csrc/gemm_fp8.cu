// Product of block-scaled e4m3 codes (trdq_fp8_linear):
//   y[m,n] = bf16(act( sum_b sx[b][m] * sw[n / 128][b] * (sum_{k in block b} q[m,k] * qw[n,k]) + bias[n] ))
// The inner sums are tensor-core accumulations (tcgen05 kind::f8f6f4, fp32) of one 128-wide k-block each; the sum over the blocks is fp32
// in registers: acc = fma(p_b, fl(sx sw), acc), b ascending.
//
// The product is formed TRANSPOSED: 128 output channels are the M operand (the lanes of tensor memory), T tokens the N operand,
// so that few tokens cost a tile of few columns, and the weight scale of a k-block is one number for the whole tile.  The k-blocks of a
// tile are cut among the CTAs of a cluster; their sums are joined through distributed shared memory, in CTA order, by the CTA that writes
// the outputs, so the result does not depend on scheduling and no workspace or second launch is needed.
//   warp 0      TMA of the weight tile (128 x 128 bytes) and the token tile (T x 128 bytes)
//   warp 1      four tcgen05.mma (128 x T x 32) per k-block into an accumulator slot of T columns of its own
//   warp 2      the tokens' scales of the k-block, by asynchronous 4-byte copies
//   warps 4 ..  one output channel per thread: accumulators * scales -> registers
// Every wait is bounded.
#include <cuda_bf16.h>

#include <algorithm>

#include "epilogue.cuh"
#include "internal.h"
#include "pair.cuh"
#include "ptx.cuh"

namespace trdq {
namespace {

constexpr int kTileCh = 128;
constexpr int kTileK = 128;  // one scale block
constexpr int kWBytes = kTileCh * kTileK;

template <int T>
struct Cfg {
  static constexpr int kCtasPerSm = T == 128 ? 1 : 2;
  static constexpr int kDrainWarps = T == 128 ? 8 : 4;
  static constexpr int kTokPerWarp = T == 128 ? 64 : T;
  static constexpr int kThreads = 128 + 32 * kDrainWarps;
  static constexpr int kSlots = T >= 64 ? 4 : 8;
  static constexpr int kTmemCols = T * kSlots;  // 128, 256, 256, 512
  static constexpr int kStageBytes = kWBytes + T * kTileK;
  static constexpr int kStages = T == 128 ? 6 : (110 * 1024 - 8 * T * 4) / kStageBytes;
  static constexpr int kSxBytes = kSlots * T * 4;
  static constexpr int kBarrierBytes = 512;
  static constexpr int kSxOff = kStages * kStageBytes;
  static constexpr int kBarOff = kSxOff + kSxBytes;
  static constexpr int kSmemBytes = 1024 + kBarOff + kBarrierBytes;
  static_assert(kSmemBytes <= (kCtasPerSm == 2 ? 113 : 227) * 1024, "shared memory");
  static_assert(T * kTileCh * 4 <= kStages * kStageBytes, "the partial sums lie where the stages were");
  static_assert((2 * kStages + 3 * kSlots) * 8 + 4 <= kBarrierBytes, "barriers");
  static_assert(kTmemCols * kCtasPerSm <= 512, "tensor memory");
};

struct alignas(64) Fp8Params {
  CUtensorMap tmap_w, tmap_x;  // boxes 128 B x 128 rows, 128 B x T rows, 128-byte swizzle
  const float* sx;
  const float* sw;
  const __nv_bfloat16* bias;
  __nv_bfloat16* out;
  int64_t ld;
  int32_t M, N, num_kb, tiles_m, splits;
  uint32_t* status;
};

__device__ __forceinline__ void umma_fp8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t"
      ".reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t"
      "}\n" ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// kind::f8f6f4: fp32 D, e4m3 A and B (format 0), both K-major, M = 128.
__host__ __device__ constexpr uint32_t umma_idesc_e4m3(int n) {
  return (1u << 4) | (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(128 >> 4) << 24);
}

__device__ __forceinline__ float4 ld_cluster_v4(uint32_t cluster_addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(cluster_addr) : "memory");
  return v;
}

struct Ring {
  int idx = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void advance(int n) {
    if (++idx == n) {
      idx = 0;
      phase ^= 1;
    }
  }
};

template <int T, bool ACT>
__global__ void __launch_bounds__(Cfg<T>::kThreads, Cfg<T>::kCtasPerSm) gemm_fp8_kernel(const __grid_constant__ Fp8Params p) {
  using C = Cfg<T>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (smem_base - smem_u32(smem_raw));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::kBarOff);
  const uint32_t bar_full = smem_u32(bars);               // [kStages] both tiles landed
  const uint32_t bar_empty = bar_full + 8 * C::kStages;   // [kStages] the MMAs have read the stage
  const uint32_t bar_tfull = bar_empty + 8 * C::kStages;  // [kSlots]  accumulators complete
  const uint32_t bar_tempty = bar_tfull + 8 * C::kSlots;  // [kSlots]  accumulators and scales of the slot used
  const uint32_t bar_sfull = bar_tempty + 8 * C::kSlots;  // [kSlots]  scales landed
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * C::kStages + 3 * C::kSlots);

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const int rank = static_cast<int>(blockIdx.x % p.splits);  // = the CTA's rank in its cluster
  const int tile = static_cast<int>(blockIdx.x / p.splits);
  const int nt = tile / p.tiles_m;
  const int m0 = (tile - nt * p.tiles_m) * T;
  const int n0 = nt * kTileCh;
  const int kb0 = static_cast<int>(static_cast<int64_t>(p.num_kb) * rank / p.splits);
  const int kb1 = static_cast<int>(static_cast<int64_t>(p.num_kb) * (rank + 1) / p.splits);

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(bar_full + 8 * s, 1);
      mbar_init(bar_empty + 8 * s, 1);
    }
    for (int a = 0; a < C::kSlots; ++a) {
      mbar_init(bar_tfull + 8 * a, 1);
      mbar_init(bar_tempty + 8 * a, C::kDrainWarps);
      mbar_init(bar_sfull + 8 * a, 32);
    }
    fence_mbar_init();
    prefetch_tensormap(&p.tmap_w);
    prefetch_tensormap(&p.tmap_x);
  }
  if (warp == 3) {
    tmem_alloc(smem_u32(tmem_slot), C::kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  griddep_launch_dependents();
  griddep_wait();  // codes, scales and weights may all come from the kernel before

  if (warp == 0) {
    if (elect_one()) {
      BoundedWaiter w(p.status, kStatusTimeoutProducer);
      Ring st;
      for (int kb = kb0; kb < kb1; ++kb) {
        w.wait(bar_empty + 8 * st.idx, st.phase ^ 1);
        const uint32_t full = bar_full + 8 * st.idx, dst = smem_base + st.idx * C::kStageBytes;
        mbar_arrive_expect_tx(full, C::kStageBytes);
        tma_load_2d(dst, &p.tmap_w, kb * kTileK, n0, full);
        tma_load_2d(dst + kWBytes, &p.tmap_x, kb * kTileK, m0, full);
        st.advance(C::kStages);
      }
      w.settle();
    }
  } else if (warp == 1) {
    if (elect_one()) {
      BoundedWaiter w(p.status, kStatusTimeoutMma);
      constexpr uint32_t idesc = umma_idesc_e4m3(T);
      Ring st, slot;
      for (int kb = kb0; kb < kb1; ++kb) {
        w.wait(bar_tempty + 8 * slot.idx, slot.phase ^ 1);
        w.wait(bar_full + 8 * st.idx, st.phase);
        tc_fence_after();
        const uint32_t w_addr = smem_base + st.idx * C::kStageBytes;
        const uint64_t a_desc = umma_desc_k_sw128(w_addr), b_desc = umma_desc_k_sw128(w_addr + kWBytes);
#pragma unroll
        for (int k = 0; k < kTileK / 32; ++k) umma_fp8(tmem_base + slot.idx * T, a_desc + 2 * k, b_desc + 2 * k, idesc, k != 0 ? 1u : 0u);
        umma_commit(bar_empty + 8 * st.idx);
        umma_commit(bar_tfull + 8 * slot.idx);
        st.advance(C::kStages);
        slot.advance(C::kSlots);
      }
      w.settle();
    }
  } else if (warp == 2) {
    BoundedWaiter w(p.status, kStatusTimeoutUnpack);
    Ring slot;
    for (int kb = kb0; kb < kb1; ++kb) {
      w.wait(bar_tempty + 8 * slot.idx, slot.phase ^ 1);
      const float* const src = p.sx + static_cast<int64_t>(kb) * p.M;
#pragma unroll
      for (int i = 0; i < (T + 31) / 32; ++i) {
        const int j = i * 32 + lane;
        const bool valid = m0 + j < p.M;
        if (j < T) cp_async4(smem_base + C::kSxOff + (slot.idx * T + j) * 4, src + (valid ? m0 + j : 0), valid ? 4u : 0u);
      }
      cp_async_arrive(bar_sfull + 8 * slot.idx);
      slot.advance(C::kSlots);
    }
    w.settle();
  } else if (warp >= 4) {
    BoundedWaiter w(p.status, kStatusTimeoutEpilogue);
    const int q = warp & 3;  // the lane quarter of tensor memory this warp may read
    const int tok0 = ((warp - 4) >> 2) * C::kTokPerWarp;
    const uint32_t t_lane = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + tok0;
    const float* const swp = p.sw + static_cast<int64_t>(nt) * p.num_kb;
    float2 acc[C::kTokPerWarp / 2];
#pragma unroll
    for (int j = 0; j < C::kTokPerWarp / 2; ++j) acc[j] = make_float2(0.0f, 0.0f);
    Ring slot;
    float sw_next = __ldg(swp + kb0);
    for (int kb = kb0; kb < kb1; ++kb) {
      const float2 sw2 = make_float2(sw_next, sw_next);
      if (kb + 1 < kb1) sw_next = __ldg(swp + kb + 1);
      w.wait(bar_sfull + 8 * slot.idx, slot.phase);
      w.wait(bar_tfull + 8 * slot.idx, slot.phase);
      __syncwarp();
      tc_fence_after();
      const float4* const sx4 = reinterpret_cast<const float4*>(smem + C::kSxOff) + (slot.idx * T + tok0) / 4;
#pragma unroll
      for (int c = 0; c < C::kTokPerWarp / 16; ++c) {
        uint32_t r[16];
        tmem_ld_32x16(t_lane + slot.idx * T + c * 16, r);
        tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float4 s = sx4[c * 4 + j];
          float2* const a = acc + c * 8 + j * 2;
          a[0] = __ffma2_rn(make_float2(__uint_as_float(r[4 * j]), __uint_as_float(r[4 * j + 1])), __fmul2_rn(make_float2(s.x, s.y), sw2), a[0]);
          a[1] = __ffma2_rn(make_float2(__uint_as_float(r[4 * j + 2]), __uint_as_float(r[4 * j + 3])), __fmul2_rn(make_float2(s.z, s.w), sw2), a[1]);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_tempty + 8 * slot.idx);
      slot.advance(C::kSlots);
    }
    w.settle();
    // the sums of this CTA's k-blocks, [token][channel], where the stages were: every MMA has been waited for
    float* const part = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int j = 0; j < C::kTokPerWarp / 2; ++j) {
      part[(tok0 + 2 * j) * kTileCh + q * 32 + lane] = acc[j].x;
      part[(tok0 + 2 * j + 1) * kTileCh + q * 32 + lane] = acc[j].y;
    }
  }

  tc_fence_before();
  __syncthreads();
  if (p.splits > 1) cluster_sync_all();
  if (warp == 3) {
    tc_fence_after();
    tmem_dealloc(tmem_base, C::kTmemCols);
  }
  // This CTA's share of the tile's tokens: a warp takes a token, a lane four channels.
  const int share = T / p.splits;
  const int n = n0 + 4 * lane;
  float4 bias = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (p.bias && n < p.N) {
    const uint2 raw = __ldg(reinterpret_cast<const uint2*>(p.bias + n));
    bias = make_float4(__uint_as_float(raw.x << 16), __uint_as_float(raw.x & 0xFFFF0000u), __uint_as_float(raw.y << 16), __uint_as_float(raw.y & 0xFFFF0000u));
  }
  for (int i = warp; i < share; i += C::kThreads / 32) {
    const int tok = rank * share + i;
    if (m0 + tok >= p.M) break;
    const uint32_t at = smem_base + (tok * kTileCh + 4 * lane) * 4;
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int k = 0; k < p.splits; ++k) {
      const float4 v = p.splits > 1 ? ld_cluster_v4(map_to_cta(at, k)) : *reinterpret_cast<const float4*>(smem + (at - smem_base));
      s = make_float4(__fadd_rn(s.x, v.x), __fadd_rn(s.y, v.y), __fadd_rn(s.z, v.z), __fadd_rn(s.w, v.w));
    }
    float2 lo = make_float2(__fadd_rn(s.x, bias.x), __fadd_rn(s.y, bias.y)), hi = make_float2(__fadd_rn(s.z, bias.z), __fadd_rn(s.w, bias.w));
    if constexpr (ACT) {
      lo = gelu_tanh2<false>(lo);
      hi = gelu_tanh2<false>(hi);
    }
    if (n < p.N) *reinterpret_cast<uint2*>(p.out + static_cast<int64_t>(m0 + tok) * p.ld + n) = make_uint2(pack_bf16(lo), pack_bf16(hi));
  }
  if (p.splits > 1) cluster_sync_all();  // no CTA leaves while another still reads its sums
}

template <int T>
trdq_status launch_tokens(const Fp8Linear& a, int sms, int dev, cudaStream_t stream) {
  using C = Cfg<T>;
  static PerDeviceFlag configured;
  if (!configured.get(dev)) {
    for (const auto kernel : {gemm_fp8_kernel<T, false>, gemm_fp8_kernel<T, true>})
      if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmemBytes) != cudaSuccess) return TRDQ_ERR_CUDA;
    configured.set(dev, true);
  }
  Fp8Params p;
  trdq_status st = encode_tmap_u8_sw128(&p.tmap_w, a.w_codes, a.K, a.N, a.K, kTileK, kTileCh);
  if (st == TRDQ_OK) st = encode_tmap_u8_sw128(&p.tmap_x, a.codes, a.K, a.M, a.K, kTileK, T);
  if (st != TRDQ_OK) return st;
  p.sx = a.scales;
  p.sw = a.w_scales;
  p.bias = static_cast<const __nv_bfloat16*>(a.bias_bf16);
  p.out = static_cast<__nv_bfloat16*>(a.out);
  p.ld = a.ld;
  p.M = a.M;
  p.N = a.N;
  p.num_kb = a.K / kTileK;
  p.tiles_m = static_cast<int32_t>((static_cast<int64_t>(a.M) + T - 1) / T);
  p.status = device_status_word();
  if (!p.status) return TRDQ_ERR_CUDA;
  const int64_t tiles = static_cast<int64_t>(p.tiles_m) * ((a.N + kTileCh - 1) / kTileCh);
  p.splits = 1;
  while (p.splits < 8 && 2 * p.splits <= p.num_kb && 2 * p.splits * tiles <= C::kCtasPerSm * sms) p.splits *= 2;
  if (tiles * p.splits > 0x7FFFFFFF) return TRDQ_ERR_SHAPE;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(tiles * p.splits));
  cfg.blockDim = dim3(C::kThreads);
  cfg.dynamicSmemBytes = C::kSmemBytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = p.splits;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.splits > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, a.act ? gemm_fp8_kernel<T, true> : gemm_fp8_kernel<T, false>, p) == cudaSuccess ? TRDQ_OK : TRDQ_ERR_CUDA;
}

}  // namespace

trdq_status launch_gemm_fp8(const Fp8Linear& a, cudaStream_t stream) {
  int dev = 0, sms = 148;
  if (cudaGetDevice(&dev) != cudaSuccess) return TRDQ_ERR_CUDA;
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (a.M > 512) {
    const trdq_status st = launch_gemm_fp8_pair(a, stream);
    if (st != TRDQ_ERR_SHAPE) return st;
  }
  if (a.M <= 16) return launch_tokens<16>(a, sms, dev, stream);
  if (a.M <= 32) return launch_tokens<32>(a, sms, dev, stream);
  if (a.M <= 64) return launch_tokens<64>(a, sms, dev, stream);
  return launch_tokens<128>(a, sms, dev, stream);
}

}  // namespace trdq

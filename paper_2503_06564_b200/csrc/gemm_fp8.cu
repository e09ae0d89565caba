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
// A k-block passes from the copy over the MMAs to the drain in 0.21, 0.25 and 0.32 us for 16, 32 and 64 tokens: too short a step for anything but its
// latencies, so a call is bounded by the blocks of the longest CTA (and by the weights' bytes where all SMs are busy), and the cut of K is what
// pays.  Measured (device time, M x K x N): 8 x 4608 x 1152 9.9 us uncut, 4.9 cut in eight; 64 x 4096 x 4096 9.8, 7.9; 8 x 4096 x 16384 14.4, the 67 MB of
// weights at 4.7 TB/s.
// Tried and left out: 128 tokens a tile (the pair kernel is faster from there on); two sets of drain warps that take every second k-block (4 % faster
// uncut, 0.3 to 0.9 us slower in a cluster, which has twice the sums to join).
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>
#include <cstdio>

#include "epilogue.cuh"
#include "internal.h"
#include "pair.cuh"
#include "ptx.cuh"

namespace trdq {
namespace {

constexpr int kTileCh = 128;
constexpr int kTileK = 128;  // one scale block
constexpr int kWBytes = kTileCh * kTileK;

constexpr int kMostLog = 3;  // clusters of up to 2^3 CTAs

// T tokens a tile, drained by four warps (one per lane quarter of tensor memory); 64 tokens by two times four, half of the tokens each, since a thread's 64
// sums would not fit the registers of two CTAs an SM.
template <int T>
struct Cfg {
  static constexpr int kTokPerWarp = T == 64 ? 32 : T;
  static constexpr int kDrainWarps = 4 * (T / kTokPerWarp);
  static constexpr int kThreads = 128 + 32 * kDrainWarps;
  static constexpr int kSlots = T == 64 ? 4 : 8;
  static constexpr int kTmemCols = T * kSlots;  // 128, 256, 256
  static constexpr int kStageBytes = kWBytes + T * kTileK;
  static constexpr int kSxBytes = kSlots * T * 4;
  static constexpr int kBarrierBytes = 512;
  static constexpr int kOverhead = 1024 + kSxBytes + kBarrierBytes;
  // Stages for one or two CTAs an SM.  Two CTAs that share an SM halve each other's pace, and the hardware places them so although other SMs are free
  // (64 x 4096 x 16384 in 128 CTAs: 21.7 us, 17.3 when the stages leave room for one only).
  static constexpr int stages(int per_sm) { return ((per_sm == 1 ? 227 : 113) * 1024 - kOverhead) / kStageBytes; }
  static constexpr int smem(int per_sm) { return kOverhead + stages(per_sm) * kStageBytes; }
  static_assert(T * kTileCh * 4 <= stages(2) * kStageBytes, "the sums lie where the stages were");
  static_assert((2 * stages(1) + 3 * kSlots) * 8 + 4 <= kBarrierBytes, "barriers");
  static_assert(2 * kTmemCols <= 512, "tensor memory of two CTAs");
};

struct alignas(64) Fp8Params {
  CUtensorMap tmap_w, tmap_x;  // boxes 128 B x 128 rows, 128 B x T rows, 128-byte swizzle
  const float* sx;
  const float* sw;
  const __nv_bfloat16* bias;
  __nv_bfloat16* out;
  int64_t ld;
  int32_t M, N, num_kb, tiles_m, splits, stages;
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
__global__ void __launch_bounds__(Cfg<T>::kThreads, 2) gemm_fp8_kernel(const __grid_constant__ Fp8Params p) {
  using C = Cfg<T>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (smem_base - smem_u32(smem_raw));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + p.stages * C::kStageBytes + C::kSxBytes);
  const uint32_t sx_off = p.stages * C::kStageBytes;
  const uint32_t bar_full = smem_u32(bars);               // [stages] both tiles landed
  const uint32_t bar_empty = bar_full + 8 * p.stages;     // [stages] the MMAs have read the stage
  const uint32_t bar_tfull = bar_empty + 8 * p.stages;    // [kSlots]  accumulators complete
  const uint32_t bar_tempty = bar_tfull + 8 * C::kSlots;  // [kSlots]  accumulators and scales of the slot used
  const uint32_t bar_sfull = bar_tempty + 8 * C::kSlots;  // [kSlots]  scales landed
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * p.stages + 3 * C::kSlots);

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
    for (int s = 0; s < p.stages; ++s) {
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
        st.advance(p.stages);
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
        st.advance(p.stages);
        slot.advance(C::kSlots);
      }
      w.settle();
    }
  } else if (warp == 2) {
    BoundedWaiter w(p.status, kStatusTimeoutScales);
    Ring slot;
    for (int kb = kb0; kb < kb1; ++kb) {
      w.wait(bar_tempty + 8 * slot.idx, slot.phase ^ 1);
      const float* const src = p.sx + static_cast<int64_t>(kb) * p.M;
#pragma unroll
      for (int i = 0; i < (T + 31) / 32; ++i) {
        const int j = i * 32 + lane;
        const bool valid = m0 + j < p.M;
        if (j < T) cp_async4(smem_base + sx_off + (slot.idx * T + j) * 4, src + (valid ? m0 + j : 0), valid ? 4u : 0u);
      }
      cp_async_arrive(bar_sfull + 8 * slot.idx);
      slot.advance(C::kSlots);
    }
    w.settle();
  } else if (warp >= 4) {
    BoundedWaiter w(p.status, kStatusTimeoutEpilogue);
    const int q = warp & 3;  // the lane quarter of tensor memory this warp may read
    const int set = (warp - 4) >> 2;
    const int tok0 = set * C::kTokPerWarp;
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
      const float4* const sx4 = reinterpret_cast<const float4*>(smem + sx_off) + (slot.idx * T + tok0) / 4;
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
    // The sums, [token][channel], where the stages were: the last k-block is complete, so every copy has landed and every MMA has read its stage.
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
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int k = 0; k < p.splits; ++k) {
      const uint32_t at = (tok * kTileCh + 4 * lane) * 4;
      const float4 v = p.splits > 1 ? ld_cluster_v4(map_to_cta(smem_base + at, k)) : *reinterpret_cast<const float4*>(smem + at);
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

// Clusters of 2^log_splits CTAs that the device holds at once with one CTA an SM; 0: the kernel cannot run here.  With two an SM it is twice that: the
// registers of the launch bounds, smem(2) and the tensor memory leave room for two, though the runtime's own count stays at one for that size too.
template <int T>
int resident_clusters(int dev, int log_splits) {
  using C = Cfg<T>;
  static PerDevice<int> cached[kMostLog + 1];
  PerDevice<int>& slot = cached[log_splits];
  const int known = slot.get(dev);
  if (known != 0) return known > 0 ? known : 0;
  bool ok = true;
  for (const auto kernel : {gemm_fp8_kernel<T, false>, gemm_fp8_kernel<T, true>})
    ok = ok && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::smem(1)) == cudaSuccess;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(1u << log_splits);
  cfg.blockDim = dim3(C::kThreads);
  cfg.dynamicSmemBytes = C::smem(1);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 1u << log_splits;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int n = 0;
  ok = ok && cudaOccupancyMaxActiveClusters(&n, gemm_fp8_kernel<T, false>, &cfg) == cudaSuccess && n > 0;
  if (!ok) cudaGetLastError();
  slot.set(dev, ok ? n : -1);
  return ok ? n : 0;
}

// How a call is cut: the tokens of a tile (0: the pair kernel), the CTAs that share a tile's k-blocks, the CTAs an SM.  us: its expected time.
struct Cut {
  int tokens = 0, log_splits = 0, per_sm = 1;
  double us = HUGE_VAL;
};

int64_t tiles_of(const Fp8Linear& a, int tokens, int channels) {
  return ((static_cast<int64_t>(a.M) + tokens - 1) / tokens) * ((static_cast<int64_t>(a.N) + channels - 1) / channels);
}

// The times are lines through those measured (8 to 256 rows, 9 to 64 k-blocks, 9 to 128 column tiles; most within 15 % of them, but for calls that the weights' bytes
// bound): a call's fixed part, what joining a cluster's sums adds, and the k-blocks that the busiest CTA goes through at the pace of a CTA that has its SM
// (us_alone) or shares it (us_shared).  CTAs that have to wait for others to leave cost their start as well.  The weights' bytes are in none of the lines: every
// cut reads them once, so a call that they bound takes longer than expected (1 x 4096 x 16384 14.4 us for 9.0; 10.2 of it the 67 MB) whichever it gets.
template <int T>
void consider(const Fp8Linear& a, int dev, Cut& best) {
  constexpr double us_alone = T == 16 ? 0.21 : T == 32 ? 0.25 : 0.315, us_shared = T == 16 ? 0.38 : T == 32 ? 0.45 : 0.65, us_fixed = T == 64 ? 3.4 : 2.3;
  const int num_kb = a.K / kTileK;
  const int64_t tiles = tiles_of(a, T, kTileCh);
  for (int log = 0; log <= kMostLog && (1 << log) <= num_kb; ++log) {
    const int alone = resident_clusters<T>(dev, log);
    if (alone == 0) continue;
    const int per_sm = tiles <= alone ? 1 : 2, resident = per_sm * alone;
    const double waves = static_cast<double>((tiles + resident - 1) / resident), kb = (num_kb + (1 << log) - 1) >> log;
    const double us = us_fixed + (log ? 0.6 + 0.25 * log : 0.0) + waves * kb * (per_sm == 1 ? us_alone : us_shared) + (waves - 1.0) * (log ? 3.0 : 2.0);
    if (us < best.us) best = Cut{T, log, per_sm, us};
  }
}

template <int T>
trdq_status launch_tokens(const Fp8Linear& a, const Cut& cut, cudaStream_t stream) {
  using C = Cfg<T>;
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
  p.splits = 1 << cut.log_splits;
  p.stages = C::stages(cut.per_sm);
  p.status = device_status_word();
  if (!p.status) return TRDQ_ERR_CUDA;
  const int64_t ctas = tiles_of(a, T, kTileCh) << cut.log_splits;
  if (ctas > 0x7FFFFFFF) return TRDQ_ERR_SHAPE;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(ctas));
  cfg.blockDim = dim3(C::kThreads);
  cfg.dynamicSmemBytes = C::smem(cut.per_sm);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(p.splits);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cut.log_splits ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, a.act ? gemm_fp8_kernel<T, true> : gemm_fp8_kernel<T, false>, p) == cudaSuccess ? TRDQ_OK : TRDQ_ERR_CUDA;
}

}  // namespace

// Few rows go to the kernel above, in the cheapest cut; the pair kernel (tiles of 256 rows and 128 columns, 0.28 us a k-block, no cut of K) takes over where
// it is expected to be faster.  Measured, us, this kernel against the pair's: 64 x 4096 x 16384 17.3, 25; 256 x 4608 x 1152 10.0, 12.8;
// 128 x 4096 x 16384 22, 29; 256 x 4096 x 4096 13.8, 12.3; 256 x 4096 x 16384 42, 25; wide outputs, where the pair kernel has many rounds of tiles that are
// nearly empty of rows: 1 x 4096 x 65536 47, 221; 64 x 4096 x 65536 54, 77; 64 x 4096 x 131072 106, 142.
static Cut choose(const Fp8Linear& a, int dev) {
  const int pairs = fp8_pair_clusters(dev);
  const int64_t rounds = pairs > 0 ? (tiles_of(a, 256, 128) + pairs - 1) / pairs : 0;
  Cut cut;
  if (pairs > 0) cut.us = (rounds > 1 ? 6.0 : 4.0) + static_cast<double>(rounds) * (a.K / kTileK * 0.28 + 0.3);
  consider<16>(a, dev, cut);
  consider<32>(a, dev, cut);
  consider<64>(a, dev, cut);
  return cut;
}

trdq_status describe_gemm_fp8_kernel(int32_t M, int32_t K, int32_t N, int dev, char* name, size_t bytes) {
  Fp8Linear a = {};
  a.M = M, a.K = K, a.N = N;
  const Cut cut = choose(a, dev);
  if (cut.tokens > 0) {
    snprintf(name, bytes, "gemm_fp8_kernel<%d>, %d a cluster, %d an SM", cut.tokens, 1 << cut.log_splits, cut.per_sm);
  } else if (fp8_pair_clusters(dev) > 0) {
    snprintf(name, bytes, "gemm_fp8_pair_kernel");
  } else {
    return TRDQ_ERR_CUDA;
  }
  return TRDQ_OK;
}

trdq_status launch_gemm_fp8(const Fp8Linear& a, cudaStream_t stream) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return TRDQ_ERR_CUDA;
  const Cut cut = choose(a, dev);
  switch (cut.tokens) {
    case 16: return launch_tokens<16>(a, cut, stream);
    case 32: return launch_tokens<32>(a, cut, stream);
    case 64: return launch_tokens<64>(a, cut, stream);
    default: return fp8_pair_clusters(dev) > 0 ? launch_gemm_fp8_pair(a, stream) : TRDQ_ERR_CUDA;
  }
}

}  // namespace trdq

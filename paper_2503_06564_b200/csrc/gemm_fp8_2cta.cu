// Product of block-scaled e4m3 codes (gemm_fp8.cu has the formula), CTA-PAIR variant for many rows (tcgen05 cta_group::2).
//
// Two CTAs of a cluster compute one 256 x BN tile of Y: each loads its own 128 rows of the activation codes and half of the weight tile, one
// thread of the leader issues the MMAs of both.  A k-block of the pipeline is one scale block, so every k-block's sums are complete numbers in an
// accumulator slot of their own, and the epilogue warps add them up in registers, acc = fma(p, fl(sx sw), acc), while the next k-block is
// multiplied:
//   warp 0       TMA of both operands (both CTAs)
//   warp 1       MMAs (leader)
//   warps 4-11   drain: a thread owns one row and half of the tile's columns; its row scale changes with the k-block, the weight scale with
//                k-block and 128-column block.  At the end of a tile bias, activation, bf16, staging tile, TMA store.
// Synchronisation as in gemm_i8_2cta.cu, with the accumulator barriers per k-block; every wait bounded.
#include <cuda_bf16.h>

#include "epilogue.cuh"
#include "internal.h"
#include "pair.cuh"
#include "ptx.cuh"

namespace trdq {
namespace {

constexpr int kTileM = 128;  // rows per CTA; the pair covers 256
constexpr int kTileK = 128;  // one scale block
constexpr int kUmmaK = 32;
constexpr int kTmemCols = 512;
constexpr int kDrainWarps = 8;
constexpr int kThreads = 128 + 32 * kDrainWarps;
constexpr int kSmemBudget = 227 * 1024;
// Registers: the drain holds up to 128 sums and a double-buffered tensor-memory load a thread, the other warpgroup little.
constexpr int kRegsLaunch = 168, kRegsDrain = 208, kRegsOther = 80;
static_assert(32 * kDrainWarps * kRegsDrain + 128 * kRegsOther <= kThreads * kRegsLaunch, "register split exceeds the launch's allocation");

template <int BN>
struct Cfg {
  static constexpr int kSlotStride = BN == 128 ? 128 : 256;
  static constexpr int kSlots = kTmemCols / kSlotStride;
  static constexpr int kABytes = kTileM * kTileK;
  static constexpr int kBBytes = (BN / 2) * kTileK;  // this CTA's half of the weight tile
  static constexpr int kStageBytes = kABytes + kBBytes;
  static constexpr int kOutBytes = kDrainWarps * 4096;  // a 32 x 64 bf16 tile per drain warp
  static constexpr int kBarrierBytes = 512;
  static constexpr int kStages = (kSmemBudget - 1024 - kOutBytes - kBarrierBytes) / kStageBytes;
  static constexpr int kSmemBytes = 1024 + kStages * kStageBytes + kOutBytes + kBarrierBytes;
  static constexpr int kCols = BN / 2;  // of a drain thread
  static_assert(kStageBytes % 1024 == 0 && kStages >= 4, "stages");
  static_assert((2 * kStages + 2 * kSlots) * 8 + 4 <= kBarrierBytes, "barriers");
};

struct alignas(64) Fp8PairParams {
  CUtensorMap tmap_a;      // activation codes, box 128 B x 128 rows
  CUtensorMap tmap_b;      // weight codes, box 128 B x BN/2 rows
  CUtensorMap tmap_out;    // bf16 output, box 64 x 32, 128-byte swizzle
  CUtensorMap tmap_out32;  // box 32 x 32, 64-byte swizzle: the odd chunk of BN = 192
  const float* sx;
  const float* sw;
  const __nv_bfloat16* bias;
  int32_t M, N, num_kb, tiles_m, tiles_n, band;
  uint32_t* status;
};

__device__ __forceinline__ void umma_fp8_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t"
      ".reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t"
      "}\n" ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// kind::f8f6f4: fp32 D, e4m3 A and B (format 0), both K-major, M = 256.
__host__ __device__ constexpr uint32_t umma_idesc_e4m3_pair(int n) {
  return (1u << 4) | (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(256 >> 4) << 24);
}

struct Tile {
  int m0, n0;
};
// Bands of `band` row tiles, column block by column block inside a band: the clusters that run at once cover a rectangle and share panels in L2.
__device__ __forceinline__ Tile tile_at(const Fp8PairParams& p, int tile, int bn) {
  const int per_band = p.band * p.tiles_n;
  const int b = tile / per_band;
  const int r = tile - b * per_band;
  const int rows = min(p.band, p.tiles_m - b * p.band);
  const int nt = r / rows;
  return Tile{(b * p.band + (r - nt * rows)) * 2 * kTileM, nt * bn};
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

// Waits for this thread's tensor-memory loads; every use of the registers stays behind the wait.
__device__ __forceinline__ void tmem_wait_ld_regs(uint32_t (&r)[16]) {
  tmem_wait_ld();
#pragma unroll
  for (int i = 0; i < 16; ++i) asm volatile("" : "+r"(r[i]));
}

template <int BN, bool ACT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) gemm_fp8_pair_kernel(const __grid_constant__ Fp8PairParams p) {
  using C = Cfg<BN>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (smem_base - smem_u32(smem_raw));
  const uint32_t out_base = smem_base + C::kStages * C::kStageBytes;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::kStages * C::kStageBytes + C::kOutBytes);
  const uint32_t bar_full = smem_u32(bars);               // [kStages] used in the leader: both CTAs' tiles landed
  const uint32_t bar_empty = bar_full + 8 * C::kStages;   // [kStages] each CTA's own: the MMAs have read the stage
  const uint32_t bar_tfull = bar_empty + 8 * C::kStages;  // [kSlots]  each CTA's own: the k-block's sums are complete
  const uint32_t bar_tempty = bar_tfull + 8 * C::kSlots;  // [kSlots]  used in the leader: both CTAs have read them
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * C::kStages + 2 * C::kSlots);

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const bool leader = rank == 0;
  const int cluster_id = blockIdx.x >> 1;
  const int num_clusters = gridDim.x >> 1;
  const int total_tiles = p.tiles_m * p.tiles_n;

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(bar_full + 8 * s, 2);   // one arrive.expect_tx from each CTA's producer
      mbar_init(bar_empty + 8 * s, 1);  // one multicast commit
    }
    for (int a = 0; a < C::kSlots; ++a) {
      mbar_init(bar_tfull + 8 * a, 1);
      mbar_init(bar_tempty + 8 * a, 2 * kDrainWarps);
    }
    fence_mbar_init();
    prefetch_tensormap(&p.tmap_a);
    prefetch_tensormap(&p.tmap_b);
    prefetch_tensormap(&p.tmap_out);
    if (BN == 192) prefetch_tensormap(&p.tmap_out32);
  }
  if (warp == 2) {
    tmem_alloc_pair(smem_u32(tmem_slot), kTmemCols);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // the peer's barriers are initialised and its tensor memory allocated before anything is signalled
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  griddep_launch_dependents();
  griddep_wait();  // codes, scales and weights may all come from the kernel before

  if (warp >= 4) {
    // ------------------------------------------------------------------- drain (both CTAs, own 128 rows)
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsDrain));
    const int dw = warp - 4;
    const int q = dw & 3;  // = warp % 4: the lane quarter of tensor memory this warp may read
    const int half = dw >> 2;
    const uint32_t my_stage = out_base + dw * 4096;
    const uint32_t t_lane = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + half * C::kCols;
    const uint32_t leader_tempty = map_to_cta(bar_tempty, 0);
    const int last_block = (p.N - 1) / kTileK;
    BoundedWaiter w(p.status, kStatusTimeoutEpilogue);
    Ring slot;
    for (int tile = cluster_id; tile < total_tiles; tile += num_clusters) {
      const Tile t = tile_at(p, tile, BN);
      const int m0 = t.m0 + static_cast<int>(rank) * kTileM + q * 32;
      const int c0 = t.n0 + half * C::kCols;
      const bool row_in = m0 + lane < p.M;
      const float* sxp = p.sx + (row_in ? m0 + lane : 0);
      // weight scales of the thread's columns: one 128-column block, or (BN = 192) two
      const float* swp = p.sw + static_cast<int64_t>(min(c0 / kTileK, last_block)) * p.num_kb;
      const float* swp2 = p.sw + static_cast<int64_t>(min((c0 + C::kCols - 1) / kTileK, last_block)) * p.num_kb;
      float2 acc[C::kCols / 2];
#pragma unroll
      for (int j = 0; j < C::kCols / 2; ++j) acc[j] = make_float2(0.0f, 0.0f);
      float sx = __ldg(sxp), sw = __ldg(swp), sw2 = BN == 192 ? __ldg(swp2) : 0.0f;
#pragma unroll 1
      for (int kb = 0; kb < p.num_kb; ++kb) {
        const float s0 = __fmul_rn(sx, sw), s1 = BN == 192 ? __fmul_rn(sx, sw2) : s0;
        if (kb + 1 < p.num_kb) {
          sxp += p.M;
          sx = __ldg(sxp);
          sw = __ldg(swp + kb + 1);
          if (BN == 192) sw2 = __ldg(swp2 + kb + 1);
        }
        w.wait(bar_tfull + 8 * slot.idx, slot.phase);
        __syncwarp();
        tc_fence_after();
        const uint32_t t_row = t_lane + slot.idx * C::kSlotStride;
        uint32_t r[2][16];
        tmem_ld_32x16(t_row, r[0]);
#pragma unroll
        for (int c = 0; c < C::kCols / 16; ++c) {
          tmem_wait_ld_regs(r[c & 1]);
          if (c + 1 < C::kCols / 16) {
            tmem_ld_32x16(t_row + (c + 1) * 16, r[(c + 1) & 1]);
          } else {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_remote_arrive(leader_tempty + 8 * slot.idx);
          }
          const float s = BN == 192 && (c0 + 16 * c) / kTileK != c0 / kTileK ? s1 : s0;
          const float2 s2 = make_float2(s, s);
#pragma unroll
          for (int j = 0; j < 8; ++j)
            acc[c * 8 + j] = __ffma2_rn(make_float2(__uint_as_float(r[c & 1][2 * j]), __uint_as_float(r[c & 1][2 * j + 1])), s2, acc[c * 8 + j]);
        }
        slot.advance(C::kSlots);
      }
      // bias, activation, bf16; 64 columns per store (32 in the odd chunk of BN = 192)
#pragma unroll
      for (int c = 0; c < C::kCols; c += 64) {
        const bool wide = c + 64 <= C::kCols;
        if (lane == 0) bulk_wait_group_read<0>();  // the previous store has finished reading the staging tile
        __syncwarp();
#pragma unroll
        for (int v = 0; v < (wide ? 8 : 4); ++v) {
          const int n = c0 + c + 8 * v;
          uint2 b[2] = {make_uint2(0u, 0u), make_uint2(0u, 0u)};
          if (p.bias && n < p.N) {
            b[0] = __ldg(reinterpret_cast<const uint2*>(p.bias + n));
            b[1] = __ldg(reinterpret_cast<const uint2*>(p.bias + n) + 1);
          }
          uint32_t packed[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t bw = j & 1 ? b[j / 2].y : b[j / 2].x;
            float2 y = __fadd2_rn(acc[(c + 8 * v) / 2 + j], make_float2(__uint_as_float(bw << 16), __uint_as_float(bw & 0xFFFF0000u)));
            if constexpr (ACT) y = gelu_tanh2<false>(y);
            packed[j] = pack_bf16(y);
          }
          const uint32_t at = wide ? my_stage + lane * 128 + ((v ^ (lane & 7)) << 4) : my_stage + lane * 64 + ((v ^ ((lane >> 1) & 3)) << 4);
          st_shared_v4(at, packed[0], packed[1], packed[2], packed[3]);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0 && m0 < p.M && c0 + c < p.N) {
          tma_store_2d(wide ? &p.tmap_out : &p.tmap_out32, c0 + c, m0, my_stage);  // rows >= M and columns >= N are clipped
          bulk_commit_group();
        }
      }
    }
    if (lane == 0) bulk_wait_group_read<0>();
    w.settle();
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
    if (warp == 0) {
      if (elect_one()) {
        BoundedWaiter w(p.status, kStatusTimeoutProducer);
        const uint32_t leader_full = map_to_cta(bar_full, 0);
        Ring st;
        for (int tile = cluster_id; tile < total_tiles; tile += num_clusters) {
          const Tile t = tile_at(p, tile, BN);
          for (int kb = 0; kb < p.num_kb; ++kb) {
            w.wait(bar_empty + 8 * st.idx, st.phase ^ 1);
            const uint32_t a_dst = smem_base + st.idx * C::kStageBytes, full = leader_full + 8 * st.idx;
            mbar_remote_arrive_expect_tx(full, C::kStageBytes);
            tma_load_2d_pair(a_dst, &p.tmap_a, kb * kTileK, t.m0 + rank * kTileM, full);
            tma_load_2d_pair(a_dst + C::kABytes, &p.tmap_b, kb * kTileK, t.n0 + rank * (BN / 2), full);
            st.advance(C::kStages);
          }
        }
        w.settle();
      }
    } else if (warp == 1) {
      if (leader && elect_one()) {
        BoundedWaiter w(p.status, kStatusTimeoutMma);
        constexpr uint32_t idesc = umma_idesc_e4m3_pair(BN);
        Ring st, slot;
        for (int tile = cluster_id; tile < total_tiles; tile += num_clusters) {
          for (int kb = 0; kb < p.num_kb; ++kb) {
            w.wait(bar_tempty + 8 * slot.idx, slot.phase ^ 1);
            w.wait(bar_full + 8 * st.idx, st.phase);
            tc_fence_after();
            const uint32_t a_addr = smem_base + st.idx * C::kStageBytes;
            const uint64_t a_desc = umma_desc_k_sw128(a_addr), b_desc = umma_desc_k_sw128(a_addr + C::kABytes);
#pragma unroll
            for (int k = 0; k < kTileK / kUmmaK; ++k)
              umma_fp8_pair(tmem_base + slot.idx * C::kSlotStride, a_desc + 2 * k, b_desc + 2 * k, idesc, k != 0 ? 1u : 0u);
            umma_commit_pair(bar_empty + 8 * st.idx);
            umma_commit_pair(bar_tfull + 8 * slot.idx);
            st.advance(C::kStages);
            slot.advance(C::kSlots);
          }
        }
        w.settle();
      }
    }
    __syncwarp();
  }

  // Neither CTA may release its shared or tensor memory while the other's MMAs or copies can still touch it.
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  if (warp == 2) {
    tc_fence_after();
    tmem_dealloc_pair(tmem_base, kTmemCols);
  }
}

// Clusters of two CTAs that can be resident at once; 0: the kernel cannot run here.
template <int BN>
int resident_clusters(int dev) {
  static PerDevice<int> cached;
  int known = cached.get(dev);
  if (known != 0) return known > 0 ? known : 0;
  using C = Cfg<BN>;
  bool ok = true;
  for (const auto kernel : {gemm_fp8_pair_kernel<BN, false>, gemm_fp8_pair_kernel<BN, true>}) {
    cudaFuncAttributes attr;
    // the register split draws on what the launch allocates
    ok = ok && cudaFuncGetAttributes(&attr, kernel) == cudaSuccess && attr.numRegs == kRegsLaunch &&
         cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmemBytes) == cudaSuccess;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = C::kSmemBytes;
  int n = 0;
  ok = ok && cudaOccupancyMaxActiveClusters(&n, gemm_fp8_pair_kernel<BN, false>, &cfg) == cudaSuccess && n > 0;
  if (!ok) cudaGetLastError();
  cached.set(dev, ok ? n : -1);
  return ok ? n : 0;
}

template <int BN, bool ACT>
cudaError_t launch_pair(const Fp8PairParams& p, int clusters, cudaStream_t stream) {
  return launch_overlapped(gemm_fp8_pair_kernel<BN, ACT>, dim3(2 * clusters), dim3(kThreads), Cfg<BN>::kSmemBytes, stream, p);
}

}  // namespace

trdq_status launch_gemm_fp8_pair(const Fp8Linear& a, cudaStream_t stream) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return TRDQ_ERR_CUDA;
  const int64_t tiles_m = (static_cast<int64_t>(a.M) + 2 * kTileM - 1) / (2 * kTileM);
  int bn = 0, resident = 0;
  double best = 0.0;
  for (const int cand : {256, 192, 128}) {
    const int clusters = cand == 256 ? resident_clusters<256>(dev) : cand == 192 ? resident_clusters<192>(dev) : resident_clusters<128>(dev);
    if (clusters == 0) continue;
    const int64_t tiles = tiles_m * ((a.N + cand - 1) / cand);
    const double cost = static_cast<double>((tiles + clusters - 1) / clusters) * (cand + 16);
    if (bn == 0 || cost < best) bn = cand, resident = clusters, best = cost;
  }
  if (bn == 0) return TRDQ_ERR_SHAPE;
  Fp8PairParams p;
  trdq_status st = encode_tmap_u8_sw128(&p.tmap_a, a.codes, a.K, a.M, a.K, kTileK, kTileM);
  if (st == TRDQ_OK) st = encode_tmap_u8_sw128(&p.tmap_b, a.w_codes, a.K, a.N, a.K, kTileK, bn / 2);
  if (st == TRDQ_OK) st = encode_tmap_2d(&p.tmap_out, a.out, 2, a.N, a.M, static_cast<uint64_t>(a.ld) * 2, 64, 32, 128);
  if (st == TRDQ_OK) st = encode_tmap_2d(&p.tmap_out32, a.out, 2, a.N, a.M, static_cast<uint64_t>(a.ld) * 2, 32, 32, 64);
  if (st != TRDQ_OK) return st;
  p.sx = a.scales;
  p.sw = a.w_scales;
  p.bias = static_cast<const __nv_bfloat16*>(a.bias_bf16);
  p.M = a.M;
  p.N = a.N;
  p.num_kb = a.K / kTileK;
  p.tiles_m = static_cast<int32_t>(tiles_m);
  p.tiles_n = (a.N + bn - 1) / bn;
  const int64_t total = tiles_m * p.tiles_n;
  if (total > 0x3FFFFFFF) return TRDQ_ERR_SHAPE;
  p.band = tiles_m >= 32 ? 4 : p.tiles_m;
  p.status = device_status_word();
  if (!p.status) return TRDQ_ERR_CUDA;
  const int clusters = static_cast<int>(total < resident ? total : resident);
  const cudaError_t e = bn == 256   ? (a.act ? launch_pair<256, true>(p, clusters, stream) : launch_pair<256, false>(p, clusters, stream))
                        : bn == 192 ? (a.act ? launch_pair<192, true>(p, clusters, stream) : launch_pair<192, false>(p, clusters, stream))
                                    : (a.act ? launch_pair<128, true>(p, clusters, stream) : launch_pair<128, false>(p, clusters, stream));
  return e == cudaSuccess ? TRDQ_OK : TRDQ_ERR_CUDA;
}

}  // namespace trdq

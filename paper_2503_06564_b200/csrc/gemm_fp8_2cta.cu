// Product of block-scaled e4m3 codes (gemm_fp8.cu has the formula), CTA-PAIR variant for many rows (tcgen05 cta_group::2).
//
// Two CTAs of a cluster compute one 256 x 128 tile of Y: each loads its own 128 rows of the activation codes and half of the weight tile, one
// thread of the leader issues the MMAs of both.  A k-block of the pipeline is one scale block, so every k-block's sums are complete numbers in an
// accumulator of their own, and drain warps add them up in registers, acc = fma(p, fl(sx sw), acc), while the next k-blocks are multiplied:
//   warp 0       TMA of both operands (both CTAs)
//   warp 1       MMAs (leader), four accumulators of 128 columns in turn
//   warp 2       waits for the accumulators' mbarriers and wakes the drain through hardware barriers
//   warps 4-19   drain: two sets of eight warps that take every second tile.  A thread owns one row and 64 columns, its scale is one number a
//                k-block; at the end of a tile bias, activation, bf16, staging tile, TMA store, while the other set adds up the next tile.
// Synchronisation as in gemm_i8_2cta.cu, with the accumulator barriers per k-block.  Every wait for an mbarrier is bounded; the hardware barriers have no limit, but
// the warps that meet at one all come to it equally often, whatever became of the mbarriers.
//
// What bounds it: operand delivery from L2 (24 KB a CTA and k-block, 11 TB/s over the SMs; 9 in a steady load, where the power limit lowers the clocks:
// 32768 x 1152 x 4608 takes 190 us by itself and 225 to 235 back to back), close behind it the drain.  Beside MMAs and copies a
// shared-memory access of another warp is slow, an mbarrier wait that is over takes 70 to 200 clocks, against 256 clocks of MMA and 130 of multiply-adds
// for a k-block.  So one warp waits for all, and hardware barriers (20 clocks) pass it on; and the scales are requested ahead (the row's line fetched
// only a k-block before its use, the round trip set the pace: 32768 x 1152 x 4608 219 us in place of 187, 4096 x 1152 x 4608 32 in place of 28).
// M x N x K, microseconds by itself with one set of drain warps -> two: 4096 x 4608 x 1152 33 -> 28, 2057 x 4624 x 1152 21 -> 18, 16384 x 3456 x 1152 84 -> 73;
// long reductions 32768 x 1152 x 4608 178 -> 187, 8192 x 4096 x 4096 140 -> 139.  Two for every length: one form, which costs the long reductions up to 5 %.
// (Since the waiting warp meets the drain in place of leaving word for it: 16384 x 3456 x 1152 74, 32768 x 1152 x 4608 190, 8192 x 4096 x 4096 138.)
// Measured and not better: tiles of 256 x 256, which need 2/3 of the operand bytes but leave tensor memory two accumulators and a thread 128 sums
// (1040 clocks a k-block in place of 512: the hand-over MMA - commit - wait - loads - release - wait is longer than the MMAs of the other accumulator;
// 32768 x 1152 x 4608 189, 4096 x 1152 x 4608 36, 8192 x 4096 x 4096 131); the same with each 128-column half handed over by itself and sixteen drain
// warps at once (210, 48, 166: four warps a scheduler, each with the loop's own instructions); 256 x 192 (189, 36, 159); scales through shared memory.
#include <cuda_bf16.h>

#include "epilogue.cuh"
#include "internal.h"
#include "pair.cuh"
#include "ptx.cuh"

namespace trdq {
namespace {

constexpr int kTileM = 128;  // rows per CTA; the pair covers 256
constexpr int kTileCh = 128;  // columns: one scale block of the weights
constexpr int kTileK = 128;  // one scale block
constexpr int kUmmaK = 32;
constexpr int kTmemCols = 512;
constexpr int kAccs = kTmemCols / kTileCh;
constexpr int kSets = 2;            // of drain warps
constexpr int kSetWarps = 8;        // 4 lane quarters of tensor memory x 2 column halves
constexpr int kDrainWarps = kSets * kSetWarps;
constexpr int kCols = kTileCh / 2;  // of a drain thread
constexpr int kThreads = 128 + 32 * kDrainWarps;
constexpr int kAhead = 4;  // k-blocks that the row scales are brought into L1 before they are used
// Registers: 640 threads are launched with 96 each; the drain's 64 sums, a tensor-memory load of 16 and its loop need a little more, the others less.
constexpr int kRegsLaunch = 96, kRegsDrain = 104, kRegsOther = 64;
static_assert(32 * kDrainWarps * kRegsDrain + 128 * kRegsOther <= kThreads * kRegsLaunch, "register split exceeds the launch's allocation");
constexpr int kABytes = kTileM * kTileK;
constexpr int kBBytes = (kTileCh / 2) * kTileK;  // this CTA's half of the weight tile
constexpr int kStageBytes = kABytes + kBBytes;
constexpr int kOutBytes = kDrainWarps * 4096;  // a 32 x 64 bf16 tile per drain warp
constexpr int kBiasBytes = kDrainWarps * kCols * 4;
constexpr int kBarrierBytes = 512;
constexpr int kStages = (227 * 1024 - 1024 - kOutBytes - kBiasBytes - kBarrierBytes) / kStageBytes;
constexpr int kOutOff = kStages * kStageBytes;
constexpr int kBiasOff = kOutOff + kOutBytes;
constexpr int kBarOff = kBiasOff + kBiasBytes;
constexpr int kSmemBytes = 1024 + kBarOff + kBarrierBytes;
static_assert(kStageBytes % 1024 == 0, "stage tiles must stay 1024-byte aligned");
static_assert((2 * kStages + 2 * kAccs) * 8 + 4 <= kBarrierBytes, "barriers");

struct alignas(64) Fp8PairParams {
  CUtensorMap tmap_a;    // activation codes, box 128 B x 128 rows
  CUtensorMap tmap_b;    // weight codes, box 128 B x 64 rows
  CUtensorMap tmap_out;  // bf16 output, box 64 x 32, 128-byte swizzle
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
constexpr uint32_t kIdesc = (1u << 4) | (static_cast<uint32_t>(kTileCh >> 3) << 17) | (static_cast<uint32_t>(256 >> 4) << 24);

struct Tile {
  int m0, n0;
};
// Bands of `band` row tiles, column block by column block inside a band: the clusters that run at once cover a rectangle and share panels in L2.
__device__ __forceinline__ Tile tile_at(const Fp8PairParams& p, int tile) {
  const int per_band = p.band * p.tiles_n;
  const int b = tile / per_band;
  const int r = tile - b * per_band;
  const int rows = min(p.band, p.tiles_m - b * p.band);
  const int nt = r / rows;
  return Tile{(b * p.band + (r - nt * rows)) * 2 * kTileM, nt * kTileCh};
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

// Hardware barrier of a set: the warp that waits for the accumulators and the set's warps meet there once a k-block.  All of them wait (bar.sync), so that
// none is ever a k-block ahead of the others and the barrier's count stays right whatever became of the mbarriers: also after a wait that expired, when
// the warp goes through its k-blocks without waiting for them.  (With an arrival that does not wait it would then count several times in one
// passage, which would end without some of the set's warps and leave those waiting for good.)
constexpr int kMeet = 32 + 32 * kSetWarps;
__device__ __forceinline__ void meet(int set) { asm volatile("bar.sync %0, %1;" ::"r"(1 + set), "n"(kMeet) : "memory"); }

// Lane and drain warp, read anew from the hardware: not kept in registers from one use to the next.
struct DrainPlace {
  int lane, dw;
};
__device__ __forceinline__ DrainPlace drain_place() {
  uint32_t tid;
  asm volatile("mov.u32 %0, %%tid.x;" : "=r"(tid));
  return DrainPlace{static_cast<int>(tid & 31), static_cast<int>(tid >> 5) - 4};
}

// MUTE: the self-test's form, whose operands are never copied, so that the waits for them expire.
template <bool ACT, bool MUTE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) gemm_fp8_pair_kernel(const __grid_constant__ Fp8PairParams p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (smem_base - smem_u32(smem_raw));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kBarOff);
  const uint32_t bar_full = smem_u32(bars);            // [kStages] used in the leader: both CTAs' tiles landed
  const uint32_t bar_empty = bar_full + 8 * kStages;   // [kStages] each CTA's own: the MMAs have read the stage
  const uint32_t bar_tfull = bar_empty + 8 * kStages;  // [kAccs]   each CTA's own: the k-block's sums are complete
  const uint32_t bar_tempty = bar_tfull + 8 * kAccs;   // [kAccs]   used in the leader: both CTAs have read them
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * kStages + 2 * kAccs);

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const bool leader = rank == 0;
  const int cluster_id = blockIdx.x >> 1;
  const int num_clusters = gridDim.x >> 1;
  const int total_tiles = p.tiles_m * p.tiles_n;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(bar_full + 8 * s, 2);   // one arrive.expect_tx from each CTA's producer
      mbar_init(bar_empty + 8 * s, 1);  // one multicast commit
    }
    for (int a = 0; a < kAccs; ++a) {
      mbar_init(bar_tfull + 8 * a, 1);
      mbar_init(bar_tempty + 8 * a, 2 * kSetWarps);  // a set's warps of both CTAs
    }
    fence_mbar_init();
    prefetch_tensormap(&p.tmap_a);
    prefetch_tensormap(&p.tmap_b);
    prefetch_tensormap(&p.tmap_out);
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
    const int set = (warp - 4) / kSetWarps;
    // what a tile's beginning and end need is worked out there: kept through the loop it would not fit the registers
    const uint32_t t_lane = tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16) + ((warp - 4) / 4 % 2) * kCols;  // warp % 4: the lane quarter it may read
    const uint32_t leader_tempty = map_to_cta(bar_tempty, 0);
    // Scales of the next k-block, requested while this one is added up: from L1, where the row's was brought kAhead k-blocks before (it is of another line
    // in every k-block; the registers for that many would not fit).  The first of a tile are requested before the end of the set's tile before.
    float qx = 0.0f, qw = 0.0f;
    const float *sxp = nullptr, *swp = nullptr;
    auto scales_of = [&](int tile) {
      const DrainPlace d = drain_place();
      const Tile t = tile_at(p, tile);
      const int row = t.m0 + static_cast<int>(cluster_ctarank()) * kTileM + (d.dw & 3) * 32 + d.lane;
      sxp = p.sx + (row < p.M ? row : 0);
      swp = p.sw + static_cast<int64_t>(t.n0 / kTileCh) * p.num_kb;
    };
    auto request = [&](int kb) {
      if (kb >= p.num_kb) return;
      qx = __ldg(sxp + static_cast<int64_t>(kb) * p.M);
      qw = __ldg(swp + kb);
      if (kb + kAhead < p.num_kb) asm volatile("prefetch.global.L1 [%0];" ::"l"(sxp + static_cast<int64_t>(kb + kAhead) * p.M));
    };
    const int first = cluster_id + set * num_clusters;
    if (first < total_tiles) {
      scales_of(first);
      request(0);
    }
    int acc_idx = set * (p.num_kb % kAccs);                        // accumulator of the next k-block
    const int passed_over = (kSets - 1) * (p.num_kb % kAccs);      // those of the other set's tile between two of this one
    for (int tile = first; tile < total_tiles; tile += kSets * num_clusters) {
      float2 acc[kCols / 2];
#pragma unroll
      for (int j = 0; j < kCols / 2; ++j) acc[j] = make_float2(0.0f, 0.0f);
#pragma unroll 1
      for (int kb = 0; kb < p.num_kb; ++kb) {
        const float scale = __fmul_rn(qx, qw);
        const float2 s2 = make_float2(scale, scale);
        request(kb + 1);
        meet(set);
        tc_fence_after();
        const uint32_t t_row = t_lane + acc_idx * kTileCh;
#pragma unroll
        for (int c = 0; c < kCols / 16; ++c) {
          uint32_t r[16];
          tmem_ld_32x16(t_row + c * 16, r);
          tmem_wait_ld_regs(r);
          if (c + 1 == kCols / 16) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_remote_arrive(leader_tempty + 8 * acc_idx);
            acc_idx = (acc_idx + 1) % kAccs;
          }
#pragma unroll
          for (int j = 0; j < 8; ++j)
            acc[c * 8 + j] = __ffma2_rn(make_float2(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1])), s2, acc[c * 8 + j]);
        }
      }
      acc_idx = (acc_idx + passed_over) % kAccs;
      if (tile + kSets * num_clusters < total_tiles) {
        scales_of(tile + kSets * num_clusters);
        request(0);
      }
      // bias, activation, bf16
      const DrainPlace d = drain_place();
      const Tile t = tile_at(p, tile);
      const int m0 = t.m0 + static_cast<int>(cluster_ctarank()) * kTileM + (d.dw & 3) * 32;
      const int c0 = t.n0 + (d.dw / 4 % 2) * kCols;
      const uint32_t my_stage = smem_base + kOutOff + d.dw * 4096;
      float* const my_bias = reinterpret_cast<float*>(smem + kBiasOff) + d.dw * kCols;
      {
        const int n = c0 + 2 * d.lane;
        const uint32_t b = p.bias && n < p.N ? __ldg(reinterpret_cast<const uint32_t*>(p.bias + n)) : 0u;
        *reinterpret_cast<float2*>(my_bias + 2 * d.lane) = make_float2(__uint_as_float(b << 16), __uint_as_float(b & 0xFFFF0000u));
      }
      if (d.lane == 0) bulk_wait_group_read<0>();  // the previous store has finished reading the staging tile
      __syncwarp();
#pragma unroll
      for (int v = 0; v < 8; ++v) {
        const float4 ba = *reinterpret_cast<const float4*>(my_bias + 8 * v), bb = *reinterpret_cast<const float4*>(my_bias + 8 * v + 4);
        const float2 bias[4] = {make_float2(ba.x, ba.y), make_float2(ba.z, ba.w), make_float2(bb.x, bb.y), make_float2(bb.z, bb.w)};
        uint32_t packed[4];
        float2 y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = __fadd2_rn(acc[4 * v + j], bias[j]);
        if constexpr (ACT) {
          gelu_pack<4>(y, packed);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) packed[j] = pack_bf16(y[j]);
        }
        st_shared_v4(my_stage + d.lane * 128 + ((v ^ (d.lane & 7)) << 4), packed[0], packed[1], packed[2], packed[3]);
      }
      fence_proxy_async_smem();
      __syncwarp();  // (the biases have been read, too)
      if (d.lane == 0 && m0 < p.M && c0 < p.N) {
        tma_store_2d(&p.tmap_out, c0, m0, my_stage);  // rows >= M and columns >= N are clipped
        bulk_commit_group();
      }
    }
    if (lane == 0) bulk_wait_group_read<0>();  // the staging tiles have been read; the stores complete before the grid does
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
    if (warp == 0) {
      // ------------------------------------------------------------------- TMA producer (both CTAs)
      if (!MUTE && elect_one()) {
        BoundedWaiter w(p.status, kStatusTimeoutProducer);
        const uint32_t leader_full = map_to_cta(bar_full, 0);
        Ring st;
        for (int tile = cluster_id; tile < total_tiles; tile += num_clusters) {
          const Tile t = tile_at(p, tile);
          for (int kb = 0; kb < p.num_kb; ++kb) {
            w.wait(bar_empty + 8 * st.idx, st.phase ^ 1);
            const uint32_t a_dst = smem_base + st.idx * kStageBytes, full = leader_full + 8 * st.idx;
            mbar_remote_arrive_expect_tx(full, kStageBytes);
            tma_load_2d_pair(a_dst, &p.tmap_a, kb * kTileK, t.m0 + rank * kTileM, full);
            tma_load_2d_pair(a_dst + kABytes, &p.tmap_b, kb * kTileK, t.n0 + rank * (kTileCh / 2), full);
            st.advance(kStages);
          }
        }
        w.settle();
      }
      __syncwarp();
    } else if (warp == 1) {
      // ------------------------------------------------------------------- MMA issuer (leader only)
      if (leader && elect_one()) {
        BoundedWaiter w(p.status, kStatusTimeoutMma);
        Ring st, acc;
        for (int tile = cluster_id; tile < total_tiles; tile += num_clusters) {
          for (int kb = 0; kb < p.num_kb; ++kb) {
            w.wait(bar_tempty + 8 * acc.idx, acc.phase ^ 1);
            w.wait(bar_full + 8 * st.idx, st.phase);
            tc_fence_after();
            const uint32_t a_addr = smem_base + st.idx * kStageBytes;
            const uint64_t a_desc = umma_desc_k_sw128(a_addr), b_desc = umma_desc_k_sw128(a_addr + kABytes);
#pragma unroll
            for (int k = 0; k < kTileK / kUmmaK; ++k) umma_fp8_pair(tmem_base + acc.idx * kTileCh, a_desc + 2 * k, b_desc + 2 * k, kIdesc, k != 0 ? 1u : 0u);
            umma_commit_pair(bar_empty + 8 * st.idx);
            umma_commit_pair(bar_tfull + 8 * acc.idx);
            st.advance(kStages);
            acc.advance(kAccs);
          }
        }
        w.settle();
      }
      __syncwarp();
    } else if (warp == 2) {
      // ------------------------------------------------------------------- an accumulator is complete: wake the drain (one lane asks; 32 would be 32 accesses)
      BoundedWaiter w(p.status, kStatusTimeoutEpilogue);
      Ring acc;
      int set = 0;
      for (int tile = cluster_id; tile < total_tiles; tile += num_clusters) {
        for (int kb = 0; kb < p.num_kb; ++kb) {
          if (lane == 0) w.wait(bar_tfull + 8 * acc.idx, acc.phase);
          __syncwarp();
          meet(set);
          acc.advance(kAccs);
        }
        set ^= 1;
      }
      w.settle();
      __syncwarp();
    }
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

// The register split draws on what the launch allocates.
bool can_run(void (*kernel)(Fp8PairParams)) {
  cudaFuncAttributes attr;
  return cudaFuncGetAttributes(&attr, kernel) == cudaSuccess && attr.numRegs == kRegsLaunch &&
         cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes) == cudaSuccess;
}

}  // namespace

// Clusters of two CTAs that can be resident at once; 0: the kernel cannot run here.
int fp8_pair_clusters(int dev) {
  static PerDevice<int> cached;
  int known = cached.get(dev);
  if (known != 0) return known > 0 ? known : 0;
  bool ok = can_run(gemm_fp8_pair_kernel<false, false>) && can_run(gemm_fp8_pair_kernel<true, false>);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmemBytes;
  int n = 0;
  ok = ok && cudaOccupancyMaxActiveClusters(&n, gemm_fp8_pair_kernel<false, false>, &cfg) == cudaSuccess && n > 0;
  if (!ok) cudaGetLastError();
  cached.set(dev, ok ? n : -1);
  return ok ? n : 0;
}

trdq_status launch_gemm_fp8_pair(const Fp8Linear& a, cudaStream_t stream, bool mute) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return TRDQ_ERR_CUDA;
  const int resident = fp8_pair_clusters(dev);
  if (resident == 0 || (mute && !can_run(gemm_fp8_pair_kernel<false, true>))) return TRDQ_ERR_SHAPE;
  Fp8PairParams p;
  trdq_status st = encode_tmap_u8_sw128(&p.tmap_a, a.codes, a.K, a.M, a.K, kTileK, kTileM);
  if (st == TRDQ_OK) st = encode_tmap_u8_sw128(&p.tmap_b, a.w_codes, a.K, a.N, a.K, kTileK, kTileCh / 2);
  if (st == TRDQ_OK) st = encode_tmap_2d(&p.tmap_out, a.out, 2, a.N, a.M, static_cast<uint64_t>(a.ld) * 2, kCols, 32, 128);
  if (st != TRDQ_OK) return st;
  p.sx = a.scales;
  p.sw = a.w_scales;
  p.bias = static_cast<const __nv_bfloat16*>(a.bias_bf16);
  p.M = a.M;
  p.N = a.N;
  p.num_kb = a.K / kTileK;
  const int64_t tiles_m = (static_cast<int64_t>(a.M) + 2 * kTileM - 1) / (2 * kTileM);
  p.tiles_m = static_cast<int32_t>(tiles_m);
  p.tiles_n = (a.N + kTileCh - 1) / kTileCh;
  const int64_t total = tiles_m * p.tiles_n;
  if (total > 0x3FFFFFFF) return TRDQ_ERR_SHAPE;
  p.band = tiles_m >= 32 ? 4 : p.tiles_m;
  p.status = device_status_word();
  if (!p.status) return TRDQ_ERR_CUDA;
  const int clusters = static_cast<int>(total < resident ? total : resident);
  const auto kernel = mute ? gemm_fp8_pair_kernel<false, true> : a.act ? gemm_fp8_pair_kernel<true, false> : gemm_fp8_pair_kernel<false, false>;
  const cudaError_t e = launch_overlapped(kernel, dim3(2 * clusters), dim3(kThreads), kSmemBytes, stream, p);
  return e == cudaSuccess ? TRDQ_OK : TRDQ_ERR_CUDA;
}

}  // namespace trdq

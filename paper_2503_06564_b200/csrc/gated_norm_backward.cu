// Gradients of trdq_gated_norm (gated_norm.cu has the forward formulas).  With n = norm(r), m = post(b) (or b), f and fb the factors
// 1 / sqrt(mean square + eps), means over the D channels of a row and sums over the rows of a sample s:
//   dn = dh o (1 + scale_s) o w                    dR = dr + f (dn - n mean(dn o n) - mean(dn))      dx = alpha dR
//   du = dR o gate_s o pw                          db = fb (du - m mean(du o m) - mean(du))          (without post: db = du)
//   A_s = sum dh o n     B_s = sum dh     C_s = sum dR o m
//   dscale_s = w o A_s   dshift_s = B_s   dgate_s = pw o C_s
//   dw = sum_s (1 + scale_s) o A_s        dpw = sum_s gate_s o C_s
// (no mean(dn), mean(du) for the root mean square.)  Three column sums per sample therefore give all five parameter gradients.
//
// A CTA holds one row at a time, CH chunks of eight channels a thread, and walks down a run of rows, so that a thread's columns and their
// running sums stay in its registers.  The runs are of equal length, one for each CTA that the SMs hold, and cross the samples: where a sample ends, and at the
// end of the run, the sums go to the workspace, run c's of sample s to entry c + s (each step along the rows moves to the next run, the
// next sample or both, so no entry is used twice).  A second kernel joins them in a fixed order: equal inputs give equal gradients.  The statistics are taken again from r and b, which are in registers for the gradient itself.
// What bounds it: the latencies of three row sums a row with as many rows in flight as registers allow, beside memory, 12 bytes a channel with a bf16 stream.
// 16384 x 1152 (adaLN) 50 us, 4.5 TB/s of a measured 6.6, 45 without the parameters' gradients; 517 x 4096 (fp32 stream, both norms) 17.5 us.
// Measured and not better: the row sums in two rounds in place of three or four (registers spill: 63 us).
#include <algorithm>

#include "gated_norm.cuh"
#include "pair.cuh"
#include "ptx.cuh"

namespace trdq {
namespace {

constexpr int kJoinWarps = 16;
constexpr int kJoinCtas = 8;
// Entries that a CTA joins by itself.  More in clusters of kJoinCtas: weights from 4096 samples of a row 163 -> 79 us for the whole call, from 592 runs of a sample 63 -> 60;
// 130 entries in a cluster 17.1 -> 19.4, 300 51.3 -> 52.9.
constexpr int64_t kJoinAlone = 384;

template <bool F32>
struct RowInputs {
  StreamChunk<F32> r, dr;
  uint4 b, dh;
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// What a thread keeps between rows besides its sums: its columns' two parameters, and the inputs of the next row, which are on their way while this row is
// computed.  In registers (LOCAL false), or in 16-byte pieces of shared memory that no other thread touches, `step` threads apart (LOCAL true): with one chunk a
// thread 96 registers instead of 128, so five warps a scheduler and not four; with two, most of what would spill (2048 x 8192 113 -> 72 us; 152 bytes of a thread still
// do, 176 with an fp32 stream, which takes 113).
template <bool F32, bool LOCAL>
struct Kept;
template <bool F32>
struct Kept<F32, false> {
  Chunk gain, gate;
  RowInputs<F32> next;
  __device__ __forceinline__ void clear(float4*, int) {
    next.r.clear();
    next.dr.clear();
    next.b = next.dh = zero4();
  }
  __device__ __forceinline__ void set_params(const Chunk& a, const Chunk& b) { gain = a, gate = b; }
  __device__ __forceinline__ Chunk get_gain() const { return gain; }
  __device__ __forceinline__ Chunk get_gate() const { return gate; }
  __device__ __forceinline__ void request(const char* r, const char* dr, const char* b, const char* dh) {
    next.r.load(r);
    if (dr) next.dr.load(dr);
    if (b) next.b = *reinterpret_cast<const uint4*>(b);
    next.dh = *reinterpret_cast<const uint4*>(dh);
  }
  __device__ __forceinline__ RowInputs<F32> get() const { return next; }
};
template <bool F32>
struct Kept<F32, true> {
  static constexpr int kHalves = F32 ? 2 : 1;            // pieces of a chunk of the stream
  static constexpr int kGain = 2 * kHalves + 2, kGate = kGain + 2, kPieces = kGate + 2;  // behind r, dr, b, dh
  float4* mine;
  int step;
  __device__ __forceinline__ void clear(float4* at, int threads) {
    mine = at;
    step = threads;
#pragma unroll
    for (int k = 0; k < kGain; ++k) mine[k * step] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  }
  __device__ __forceinline__ void put(int piece, const Chunk& c) {
    mine[piece * step] = make_float4(c.p[0].x, c.p[0].y, c.p[1].x, c.p[1].y);
    mine[(piece + 1) * step] = make_float4(c.p[2].x, c.p[2].y, c.p[3].x, c.p[3].y);
  }
  __device__ __forceinline__ Chunk chunk(int piece) const {
    const float4 a = mine[piece * step], b = mine[(piece + 1) * step];
    return Chunk{{make_float2(a.x, a.y), make_float2(a.z, a.w), make_float2(b.x, b.y), make_float2(b.z, b.w)}};
  }
  __device__ __forceinline__ void set_params(const Chunk& a, const Chunk& b) {
    put(kGain, a);
    put(kGate, b);
  }
  __device__ __forceinline__ Chunk get_gain() const { return chunk(kGain); }
  __device__ __forceinline__ Chunk get_gate() const { return chunk(kGate); }
  // (the pieces of the row before are in registers by now)
  __device__ __forceinline__ void request(const char* r, const char* dr, const char* b, const char* dh) {
    const uint32_t at = smem_u32(mine), by = static_cast<uint32_t>(step) * 16;
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      cp_async16(at + h * by, r + 16 * h);
      if (dr) cp_async16(at + (kHalves + h) * by, dr + 16 * h);
    }
    if (b) cp_async16(at + 2 * kHalves * by, b);
    cp_async16(at + (2 * kHalves + 1) * by, dh);
  }
  __device__ __forceinline__ RowInputs<F32> get() const {
    RowInputs<F32> v;
    v.r.load_pieces(mine, step);
    v.dr.load_pieces(mine + kHalves * step, step);
    v.b = *reinterpret_cast<const uint4*>(mine + 2 * kHalves * step);
    v.dh = *reinterpret_cast<const uint4*>(mine + (2 * kHalves + 1) * step);
    return v;
  }
};

constexpr int kLocalThreads = 640;  // of an SM, with LOCAL and one chunk a thread
template <bool F32>
constexpr int kLocalPieces = Kept<F32, true>::kPieces;

template <int CH, bool F32, bool LOCAL>
__global__ void __launch_bounds__(LOCAL && CH == 1 ? kLocalThreads : 32 * kRowWarps, 1) gated_norm_backward_kernel(const GatedNormBackward p) {
  extern __shared__ float4 local[];
  __shared__ float4 slots[RowSum::kSlots];
  RowSum sums(slots);
  const float inv_d = __fdiv_rn(1.0f, static_cast<float>(p.D));
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * p.rows_per_run;
  const int rows = static_cast<int>(min(static_cast<int64_t>(p.rows_per_run), p.M - row0));
  griddep_launch_dependents();
  griddep_wait();

  constexpr int kBytes = F32 ? 4 : 2;
  bool in[CH];
  int at[CH];
  const char *r_at[CH], *dr_at[CH], *b_at[CH], *dh_at[CH];
  char *dx_at[CH], *db_at[CH];
  Chunk A[CH], B[CH], C[CH];
  const Chunk none{{make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)}};
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    at[j] = static_cast<int>(threadIdx.x + j * blockDim.x);
    in[j] = at[j] < p.D / 8;
    r_at[j] = stream_at(p.r, row0, p.ldr, at[j], F32);
    dr_at[j] = stream_at(p.dr, row0, p.lddr, at[j], F32);
    b_at[j] = stream_at(p.b, row0, p.ldb, at[j], false);
    dh_at[j] = stream_at(p.dh, row0, p.lddh, at[j], false);
    dx_at[j] = stream_at(p.dx, row0, p.lddx, at[j], F32);
    db_at[j] = stream_at(p.db, row0, p.lddb, at[j], false);
    A[j] = B[j] = C[j] = none;
  }

  Kept<F32, LOCAL> kept[CH];
#pragma unroll
  for (int j = 0; j < CH; ++j) kept[j].clear(local + j * kLocalPieces<F32> * blockDim.x + threadIdx.x, blockDim.x);  // what is not loaded (lanes outside the row, inputs that are not there) stays zero
  auto fetch = [&](bool valid) {
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      if (valid && in[j]) kept[j].request(r_at[j], p.dr ? dr_at[j] : nullptr, p.b ? b_at[j] : nullptr, dh_at[j]);
      r_at[j] += p.ldr * kBytes;
      dr_at[j] += p.lddr * kBytes;
      b_at[j] += p.ldb * 2;
      dh_at[j] += p.lddh * 2;
    }
  };
  fetch(rows > 0);
  int64_t s = row0 / p.rows_per_sample;                                                               // the sample of the row at hand
  int until = static_cast<int>(min((s + 1) * p.rows_per_sample - row0, static_cast<int64_t>(rows)));  // the run's row it ends at
  auto begin = [&]() {
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      Chunk gain = chunk_shift(none, 1.0f), gate = gain;  // (1 + scale) o w and gate o pw of this thread's columns
      if (in[j]) {
        if (p.scale) gain = chunk_shift(widen(load_param(p.scale + s * p.ld_scale, at[j])), 1.0f);
        if (p.weight) gain = chunk_mul(gain, widen(load_param(p.weight, at[j])));
        if (p.gate) gate = widen(load_param(p.gate + s * p.ld_gate, at[j]));
        if (p.post_weight) gate = chunk_mul(gate, widen(load_param(p.post_weight, at[j])));
      }
      kept[j].set_params(gain, gate);
    }
  };
  auto flush = [&]() {
    const int64_t plane = static_cast<int64_t>(p.entries) * p.D;
    auto put = [](float* to, const Chunk& v) {
      reinterpret_cast<float4*>(to)[0] = make_float4(v.p[0].x, v.p[0].y, v.p[1].x, v.p[1].y);
      reinterpret_cast<float4*>(to)[1] = make_float4(v.p[2].x, v.p[2].y, v.p[3].x, v.p[3].y);
    };
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      if (in[j]) {
        float* const to = p.workspace + (blockIdx.x + s) * p.D + 8 * at[j];
        if (p.dscale || p.dweight) put(to, A[j]);
        if (p.dshift) put(to + plane, B[j]);
        if (p.dgate || p.dpost_weight) put(to + 2 * plane, C[j]);
      }
      A[j] = B[j] = C[j] = none;
    }
  };
  auto prefetch = [&](const uint16_t* param, int64_t ld) {
    if (!param) return;
#pragma unroll
    for (int j = 0; j < CH; ++j)
      if (in[j]) prefetch_l1(param + (s + 1) * ld + 8 * at[j]);
  };
  begin();
  const float2 alpha2 = make_float2(p.alpha, p.alpha);
  for (int row = 0; row < rows; ++row) {
    if (row == until) {
      flush();
      ++s;
      until = static_cast<int>(min(static_cast<int64_t>(until) + p.rows_per_sample, static_cast<int64_t>(rows)));
      begin();
    }
    if (row + 2 == until && until < rows) {  // soon the next sample's parameters
      prefetch(p.scale, p.ld_scale);
      prefetch(p.gate, p.ld_gate);
    }
    Chunk n[CH], m[CH], dh[CH], dR[CH];
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      if (LOCAL && j == 0) cp_async_wait_all();
      const RowInputs<F32> now = kept[j].get();
      n[j] = now.r.value();
      m[j] = widen(now.b);
      dh[j] = widen(now.dh);
      dR[j] = now.dr.value();
    }
    fetch(row + 1 < rows);

    const float f = row_centre(n, in, p.norm, inv_d, p.eps, sums);
    float fb = 1.0f;
    if (p.post != TRDQ_NORM_NONE) {
      fb = row_centre(m, in, p.post, inv_d, p.eps, sums);
#pragma unroll
      for (int j = 0; j < CH; ++j) m[j] = chunk_scale(m[j], fb);
    }
    float2 t = make_float2(0.0f, 0.0f);
    Chunk dn[CH];
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      n[j] = chunk_scale(n[j], f);
#pragma unroll
      for (int i = 0; i < 4; ++i) B[j].p[i] = __fadd2_rn(B[j].p[i], dh[j].p[i]);
      A[j] = chunk_fma(dh[j], n[j], A[j]);
      dn[j] = chunk_mul(dh[j], kept[j].get_gain());
      t = __fadd2_rn(t, make_float2(chunk_dot(dn[j], n[j]), chunk_sum(dn[j])));
    }
    t = sums.two(t);
    const float along = -__fmul_rn(t.x, inv_d), mean = p.norm == TRDQ_NORM_LAYER ? -__fmul_rn(t.y, inv_d) : 0.0f;
    const float2 f2 = make_float2(f, f), along2 = make_float2(along, along), mean2 = make_float2(mean, mean);
    Chunk du[CH];
#pragma unroll
    for (int j = 0; j < CH; ++j) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        dR[j].p[i] = __ffma2_rn(__ffma2_rn(n[j].p[i], along2, __fadd2_rn(dn[j].p[i], mean2)), f2, dR[j].p[i]);
      C[j] = chunk_fma(dR[j], m[j], C[j]);
      du[j] = chunk_mul(dR[j], kept[j].get_gate());
      if (p.dx && in[j]) {
        StreamChunk<F32> o;
        Chunk v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v.p[i] = __fmul2_rn(dR[j].p[i], alpha2);
        o.set(v);
        o.store(dx_at[j]);
      }
      dx_at[j] += p.lddx * kBytes;
    }
    if (!p.db) continue;  // the same for every thread
    if (p.post != TRDQ_NORM_NONE) {
      float2 e = make_float2(0.0f, 0.0f);
#pragma unroll
      for (int j = 0; j < CH; ++j)
        if (in[j]) e = __fadd2_rn(e, make_float2(chunk_dot(du[j], m[j]), chunk_sum(du[j])));
      e = sums.two(e);
      const float2 fb2 = make_float2(fb, fb), a2 = make_float2(-__fmul_rn(e.x, inv_d), -__fmul_rn(e.x, inv_d));
      const float me = p.post == TRDQ_NORM_LAYER ? -__fmul_rn(e.y, inv_d) : 0.0f;
#pragma unroll
      for (int j = 0; j < CH; ++j) {
#pragma unroll
        for (int i = 0; i < 4; ++i) du[j].p[i] = __fmul2_rn(__ffma2_rn(m[j].p[i], a2, __fadd2_rn(du[j].p[i], make_float2(me, me))), fb2);
      }
    }
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      if (in[j]) *reinterpret_cast<uint4*>(db_at[j]) = narrow(du[j]);
      db_at[j] += p.lddb * 2;
    }
  }

  flush();
}

__device__ __forceinline__ float4 widen4(const uint16_t* v) {
  const uint2 w = *reinterpret_cast<const uint2*>(v);
  const float2 a = widen_bf16x2(w.x), b = widen_bf16x2(w.y);
  return make_float4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ float4 fma4(const float4& a, const float4& b, const float4& c) {
  return make_float4(__fmaf_rn(a.x, b.x, c.x), __fmaf_rn(a.y, b.y, c.y), __fmaf_rn(a.z, b.z, c.z), __fmaf_rn(a.w, b.w, c.w));
}
// (the outputs are only known to be floats)
__device__ __forceinline__ void put4(float* to, const float4& v) { to[0] = v.x, to[1] = v.y, to[2] = v.z, to[3] = v.w; }
__device__ __forceinline__ float4 ones4() { return make_float4(1.0f, 1.0f, 1.0f, 1.0f); }
__device__ __forceinline__ float4 zeros4() { return make_float4(0.0f, 0.0f, 0.0f, 0.0f); }

// What a plane's sums become: a sample's gradient, and the parameter that multiplies it.
__device__ __forceinline__ float* sample_output(const GatedNormBackward& p, int plane) { return plane == 0 ? p.dscale : plane == 1 ? p.dshift : p.dgate; }
__device__ __forceinline__ const uint16_t* sample_factor(const GatedNormBackward& p, int plane) { return plane == 0 ? p.weight : plane == 1 ? nullptr : p.post_weight; }

// The first and last entry of a sample, one for each run that it has rows of.
__device__ __forceinline__ void sample_entries(const GatedNormBackward& p, int64_t sample, int64_t* first, int64_t* last) {
  const int64_t end = min((sample + 1) * p.rows_per_sample, static_cast<int64_t>(p.M));
  *first = sample * p.rows_per_sample / p.rows_per_run + sample;
  *last = (end - 1) / p.rows_per_run + sample;
}

// Joins many entries of a plane, 32 columns a CTA, four a thread.  WEIGHTS: the weights' gradients, from all entries; else those of a sample.  The groups of eight threads take every `groups`-th entry; their sums are added in order.  Bound by latency: with 128 columns
// and all three planes in one CTA the sums of 130 runs of 4096 took 7 us instead of 5.
// SHARED: the entries are cut among the kJoinCtas CTAs of a cluster, whose sums are added in their order.
template <bool WEIGHTS, bool SHARED>
__device__ __forceinline__ void join_columns(const GatedNormBackward& p, int plane, int columns, int64_t sample) {
  __shared__ float4 part[kJoinWarps][8];
  const int quad = threadIdx.x & 7, group = threadIdx.x >> 3, groups = blockDim.x >> 3;
  const int col = (columns * 8 + quad) * 4;
  const bool in = col < p.D;
  float* const to = !WEIGHTS ? sample_output(p, plane) : plane == 0 ? p.dweight : plane == 1 ? nullptr : p.dpost_weight;
  if (!to) return;
  const int64_t rps = p.rows_per_sample, rpr = p.rows_per_run;
  int64_t first = 0, last = p.entries - 1;
  if (!WEIGHTS) sample_entries(p, sample, &first, &last);
  const uint32_t rank = SHARED ? cluster_ctarank() : 0;
  if (SHARED) {
    const int64_t n = last + 1 - first, from = first + n * rank / kJoinCtas;
    last = first + n * (rank + 1) / kJoinCtas - 1;
    first = from;
  }
  const uint16_t* const factor = !WEIGHTS ? nullptr : plane == 0 ? p.scale : p.gate;
  const int64_t ld_factor = plane == 0 ? p.ld_scale : p.ld_gate;
  const float* const from = p.workspace + plane * p.entries * p.D + col;
  const uint16_t* const by = WEIGHTS ? nullptr : sample_factor(p, plane);
  griddep_wait();
  const float4 after = by && in ? widen4(by + col) : ones4();
  float4 sum = zeros4();
  if (in && (!WEIGHTS || rps >= p.M)) {
    float4 k = ones4();
    if (factor) k = plane == 0 ? RowSum::add(k, widen4(factor + col)) : widen4(factor + col);
#pragma unroll 4
    for (int64_t i = first + group; i <= last; i += groups) sum = fma4(*reinterpret_cast<const float4*>(from + i * p.D), k, sum);
  } else if (in) {
#pragma unroll 2
    for (int64_t i = first + group; i <= last; i += groups) {
      // Sample s begins with entry floor(s rps / rpr) + s = floor(s (rps + rpr) / rpr).  The last entry before a sample that begins with a run is nobody's.
      const int64_t s = ((i + 1) * rpr - 1) / (rps + rpr);
      if ((i - s) * rpr >= min((s + 1) * rps, static_cast<int64_t>(p.M))) continue;
      float4 k = ones4();
      if (factor) k = plane == 0 ? RowSum::add(k, widen4(factor + s * ld_factor + col)) : widen4(factor + s * ld_factor + col);
      sum = fma4(*reinterpret_cast<const float4*>(from + i * p.D), k, sum);
    }
  }
#pragma unroll
  for (int d = 8; d <= 16; d <<= 1)
    sum = RowSum::add(sum, make_float4(__shfl_xor_sync(0xffffffffu, sum.x, d), __shfl_xor_sync(0xffffffffu, sum.y, d), __shfl_xor_sync(0xffffffffu, sum.z, d),
                                       __shfl_xor_sync(0xffffffffu, sum.w, d)));
  const int warps = blockDim.x >> 5;
  if (warps > 1) {
    if ((threadIdx.x & 31) < 8) part[threadIdx.x >> 5][quad] = sum;
    __syncthreads();
    sum = part[0][quad];
    for (int w = 1; w < warps; ++w) sum = RowSum::add(sum, part[w][quad]);
  }
  if constexpr (SHARED) {
    __shared__ float4 whole[8];
    if (group == 0) whole[quad] = sum;
    cluster_sync_all();
    if (rank == 0 && group == 0) {
#pragma unroll
      for (int k = 1; k < kJoinCtas; ++k) sum = RowSum::add(sum, ld_cluster_v4(map_to_cta(smem_u32(&whole[quad]), k)));
    }
    cluster_sync_all();  // no CTA leaves while its sums are read
    if (rank != 0) return;
  }
  if (!in || group != 0) return;
  put4(to + (WEIGHTS ? 0 : sample * p.D) + col, by ? fma4(sum, after, zeros4()) : sum);
}

template <bool WEIGHTS>
__global__ void __launch_bounds__(32 * kJoinWarps) gated_norm_join_kernel(const GatedNormBackward p) {
  join_columns<WEIGHTS, false>(p, blockIdx.z, blockIdx.y, blockIdx.x);
}
template <bool WEIGHTS>
__global__ void __cluster_dims__(kJoinCtas, 1, 1) __launch_bounds__(32 * kJoinWarps) gated_norm_join_shared_kernel(const GatedNormBackward p) {
  join_columns<WEIGHTS, true>(p, blockIdx.z, blockIdx.y, blockIdx.x / kJoinCtas);
}

// Joins samples of few entries: a thread takes four columns of a plane of a sample and adds its entries in order.  CTAs from sample_ctas on: the weights, which
// saves a launch (five rows 6.4 -> 5.0 us).  The whole
// call with this join and with the one above, us: 16384 x 1152 in samples of 256 rows, ten entries each, 50, 52; 18846 x 680 in samples of 16 45, 79; 4096 x 1152 in samples of one 60, 258.
__global__ void __launch_bounds__(256) gated_norm_join_samples_kernel(const GatedNormBackward p, unsigned sample_ctas) {
  if (blockIdx.x >= sample_ctas) return join_columns<true, false>(p, blockIdx.y, static_cast<int>(blockIdx.x - sample_ctas), 0);
  const int quads = p.D / 4;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, of = item / quads;
  const int col = static_cast<int>(item - of * quads) * 4, plane = blockIdx.y;
  float* const to = sample_output(p, plane);
  if (!to || of > (p.M - 1) / p.rows_per_sample) return;
  int64_t first, last;
  sample_entries(p, of, &first, &last);
  const float* const from = p.workspace + plane * p.entries * p.D + col;
  const uint16_t* const by = sample_factor(p, plane);
  griddep_wait();
  const float4 after = by ? widen4(by + col) : ones4();
  float4 sum = zeros4();
#pragma unroll 4
  for (int64_t i = first; i <= last; ++i) sum = RowSum::add(sum, *reinterpret_cast<const float4*>(from + i * p.D));
  put4(to + of * p.D + col, by ? fma4(sum, after, zeros4()) : sum);
}

// Two chunks a thread.  What the kernel may ask for is state of the function on its device, which calls of other widths share, from other threads too: it
// is set once, to what the widest rows take.
template <bool F32>
cudaError_t launch_wide(const GatedNormBackward& p, dim3 grid, dim3 threads, cudaStream_t stream) {
  constexpr size_t kThreadBytes = sizeof(float4) * 2 * kLocalPieces<F32>;
  static PerDeviceFlag configured;
  const auto kernel = gated_norm_backward_kernel<2, F32, true>;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && !configured.get(dev)) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kThreadBytes * 32 * kRowWarps));
    if (e == cudaSuccess) configured.set(dev, true);
  }
  return e != cudaSuccess ? e : launch_overlapped(kernel, grid, threads, kThreadBytes * threads.x, stream, p);
}

}  // namespace

// Whether the kernel with less in registers holds more CTAs of the width.  us, without and with it: 16384 x 1152 56.2, 52.3; 16384 x 2560 148.5, 107.6;
// 16384 x 1024 46.1, 44.7.  With an fp32 stream, which is nearer to the memory's bound (5.0 TB/s) and has half as much again to keep, it lost: 68.1, 82.1.
static bool keeps_local(int threads, bool f32) { return !f32 && kLocalThreads / threads > 512 / threads; }

// The rows in runs of equal length, one for each of the CTAs that the SMs hold at once, and the entries of the workspace.  Runs cut at the samples' ends
// instead left SMs idle: 16384 x 1152 in samples of 256 took 61 us, 56 without.
void gated_norm_backward_runs(int32_t M, int32_t D, bool f32, int32_t rows_per_sample, int32_t* rows_per_run, int64_t* entries) {
  constexpr int kSms = 148;
  const int threads = row_threads(D), per_sm = (row_chunks(D) == 1 && keeps_local(threads, f32) ? kLocalThreads : 512) / threads;
  const int64_t slots = static_cast<int64_t>(kSms) * per_sm, rows = M;
  *rows_per_run = static_cast<int32_t>((rows + slots - 1) / slots);
  *entries = (rows + *rows_per_run - 1) / *rows_per_run + (rows - 1) / rows_per_sample;
}

trdq_status launch_gated_norm_backward(const GatedNormBackward& args, cudaStream_t stream) {
  GatedNormBackward p = args;
  const int64_t grid = (static_cast<int64_t>(p.M) + p.rows_per_run - 1) / p.rows_per_run, samples = (static_cast<int64_t>(p.M) - 1) / p.rows_per_sample + 1;
  if (samples > 0x7FFFFFFE || row_threads(p.D) > 32 * kRowWarps) return TRDQ_ERR_SHAPE;
  const int threads = row_threads(p.D);
  const dim3 g(static_cast<unsigned>(grid)), t(threads);
  cudaError_t e;
  if (row_chunks(p.D) == 2) {
    e = p.f32 ? launch_wide<true>(p, g, t, stream) : launch_wide<false>(p, g, t, stream);
  } else if (keeps_local(threads, p.f32)) {
    e = launch_overlapped(gated_norm_backward_kernel<1, false, true>, g, t, sizeof(float4) * kLocalPieces<false> * threads, stream, p);
  } else {
    e = launch_overlapped(p.f32 ? gated_norm_backward_kernel<1, true, false> : gated_norm_backward_kernel<1, false, false>, g, t, 0, stream, p);
  }
  if (e != cudaSuccess) return TRDQ_ERR_CUDA;
  auto warps_for = [](int64_t entries) { return static_cast<unsigned>(std::min<int64_t>(kJoinWarps, std::max<int64_t>(1, entries / 16))); };  // four a group
  const unsigned blocks32 = (p.D / 4 + 7) / 8;
  bool weights = p.dweight || p.dpost_weight;
  if (p.dscale || p.dshift || p.dgate) {
    const int64_t most = (std::min<int64_t>(p.rows_per_sample, p.M) - 1) / p.rows_per_run + 2;  // entries of a sample
    if (most <= 16) {
      const int64_t ctas = (samples * (p.D / 4) + 255) / 256;
      if (ctas > 0x7FFFFFFF - blocks32) return TRDQ_ERR_SHAPE;
      const unsigned sample_ctas = static_cast<unsigned>(ctas);
      const bool both = weights && p.entries <= kJoinAlone;
      e = launch_overlapped(gated_norm_join_samples_kernel, dim3(sample_ctas + (both ? blocks32 : 0), 3), dim3(256), 0, stream, p, sample_ctas);
      weights = weights && !both;
    } else if (most <= kJoinAlone) {
      e = launch_overlapped(gated_norm_join_kernel<false>, dim3(static_cast<unsigned>(samples), blocks32, 3), dim3(32 * warps_for(most)), 0, stream, p);
    } else {
      if (samples > 0x7FFFFFFF / kJoinCtas) return TRDQ_ERR_SHAPE;
      e = launch_overlapped(gated_norm_join_shared_kernel<false>, dim3(static_cast<unsigned>(samples * kJoinCtas), blocks32, 3), dim3(32 * warps_for(most / kJoinCtas)), 0,
                            stream, p);
    }
    if (e != cudaSuccess) return TRDQ_ERR_CUDA;
  }
  if (weights && p.entries <= kJoinAlone) {
    e = launch_overlapped(gated_norm_join_kernel<true>, dim3(1, blocks32, 3), dim3(32 * warps_for(p.entries)), 0, stream, p);
  } else if (weights) {
    e = launch_overlapped(gated_norm_join_shared_kernel<true>, dim3(kJoinCtas, blocks32, 3), dim3(32 * warps_for(p.entries / kJoinCtas)), 0, stream, p);
  }
  return e == cudaSuccess ? TRDQ_OK : TRDQ_ERR_CUDA;
}

}  // namespace trdq

// Gradients of trdq_gated_norm (gated_norm.cu has the forward formulas).  With n = norm(r), m = post(b) (or b), f and fb the factors
// 1 / sqrt(mean square + eps), means over the D channels of a row and sums over the rows of a sample s:
//   dn = dh o (1 + scale_s) o w                    dR = dr + f (dn - n mean(dn o n) - mean(dn))      dx = alpha dR
//   du = dR o gate_s o pw                          db = fb (du - m mean(du o m) - mean(du))          (without post: db = du)
//   A_s = sum dh o n     B_s = sum dh     C_s = sum dR o m
//   dscale_s = w o A_s   dshift_s = B_s   dgate_s = pw o C_s
//   dw = sum_s (1 + scale_s) o A_s        dpw = sum_s gate_s o C_s
// (no mean(dn), mean(du) for the root mean square.)  Three column sums per sample therefore give all five parameter gradients.
//
// A CTA holds one row at a time, CH chunks of eight channels a thread, and walks down a run of rows of one sample, so that a thread's
// columns and their running sums stay in its registers.  The runs' sums go to the workspace and are joined by a second kernel in a
// fixed order: equal inputs give equal gradients.  The statistics are taken again from r and b, which are in registers for the gradient itself.
// What bounds it: memory, 12 bytes a channel with a bf16 stream.
#include <algorithm>

#include "gated_norm.cuh"
#include "ptx.cuh"

namespace trdq {
namespace {

constexpr int kMostWarps = 16;

// Sums over all warps of the CTA, as TeamSum.
struct CtaSum {
  float* slots;  // [2][2][kMostWarps]
  int warps;
  int turn = 0;
  __device__ __forceinline__ CtaSum(float* s, int w) : slots(s), warps(w) {}
  __device__ __forceinline__ float2 sum(float2 v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      v.x = __fadd_rn(v.x, __shfl_xor_sync(0xffffffffu, v.x, d));
      v.y = __fadd_rn(v.y, __shfl_xor_sync(0xffffffffu, v.y, d));
    }
    if (warps == 1) return v;
    float2* const here = reinterpret_cast<float2*>(slots) + turn * kMostWarps;
    turn ^= 1;
    if ((threadIdx.x & 31) == 0) here[threadIdx.x >> 5] = v;
    __syncthreads();
    float2 s = here[0];
    for (int k = 1; k < warps; ++k) s = __fadd2_rn(s, here[k]);
    return s;
  }
};

template <bool F32>
struct RowInputs {
  StreamChunk<F32> r, dr;
  uint4 b, dh;
};

template <int CH, bool F32>
__global__ void __launch_bounds__(32 * kMostWarps) gated_norm_backward_kernel(const GatedNormBackward p) {
  __shared__ float2 slots[2 * kMostWarps];
  CtaSum cta(reinterpret_cast<float*>(slots), blockDim.x >> 5);
  const int chunks = p.D / 8;
  const float inv_d = __fdiv_rn(1.0f, static_cast<float>(p.D));
  const int64_t s = blockIdx.x / p.runs;
  const int64_t run = blockIdx.x - s * p.runs;
  const int64_t sample0 = s * p.rows_per_sample;
  const int64_t row0 = sample0 + run * p.rows_per_run;
  const int64_t row1 = min(min(row0 + p.rows_per_run, sample0 + p.rows_per_sample), static_cast<int64_t>(p.M));
  griddep_launch_dependents();
  griddep_wait();

  bool in[CH];
  Chunk gain[CH], gate[CH];  // (1 + scale) o w and gate o pw of this thread's columns
  Chunk A[CH], B[CH], C[CH];
  const Chunk none{{make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)}};
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const int c = threadIdx.x + j * blockDim.x;
    in[j] = c < chunks;
    A[j] = B[j] = C[j] = none;
    gain[j] = gate[j] = chunk_shift(none, 1.0f);
    if (!in[j]) continue;
    if (p.scale) gain[j] = chunk_shift(widen(load_param(p.scale + s * p.ld_scale, c)), 1.0f);
    if (p.weight) gain[j] = chunk_mul(gain[j], widen(load_param(p.weight, c)));
    if (p.gate) gate[j] = widen(load_param(p.gate + s * p.ld_gate, c));
    if (p.post_weight) gate[j] = chunk_mul(gate[j], widen(load_param(p.post_weight, c)));
  }

  RowInputs<F32> next[CH];
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const int c = threadIdx.x + j * blockDim.x;
      next[j].r.clear();
      next[j].dr.clear();
      next[j].b = next[j].dh = zero4();
      if (!in[j] || row >= row1) continue;
      next[j].r.load(stream_row(p.r, row, p.ldr, F32), c);
      if (p.dr) next[j].dr.load(stream_row(p.dr, row, p.lddr, F32), c);
      if (p.b) next[j].b = *(reinterpret_cast<const uint4*>(p.b + row * p.ldb) + c);
      next[j].dh = *(reinterpret_cast<const uint4*>(p.dh + row * p.lddh) + c);
    }
  };
  fetch(row0);
  for (int64_t row = row0; row < row1; ++row) {
    Chunk n[CH], m[CH], dh[CH], dR[CH];
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      n[j] = next[j].r.value();
      m[j] = widen(next[j].b);
      dh[j] = widen(next[j].dh);
      dR[j] = next[j].dr.value();
    }
    fetch(row + 1);

    // statistics of r and of b together
    if (p.norm == TRDQ_NORM_LAYER || p.post == TRDQ_NORM_LAYER) {
      float2 t = make_float2(0.0f, 0.0f);
#pragma unroll
      for (int j = 0; j < CH; ++j) t = __fadd2_rn(t, make_float2(chunk_sum(n[j]), chunk_sum(m[j])));
      t = cta.sum(t);
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        if (!in[j]) continue;
        if (p.norm == TRDQ_NORM_LAYER) n[j] = chunk_shift(n[j], -__fmul_rn(t.x, inv_d));
        if (p.post == TRDQ_NORM_LAYER) m[j] = chunk_shift(m[j], -__fmul_rn(t.y, inv_d));
      }
    }
    float2 q = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int j = 0; j < CH; ++j) q = __fadd2_rn(q, make_float2(chunk_dot(n[j], n[j]), chunk_dot(m[j], m[j])));
    q = cta.sum(q);
    const float f = __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(__fmul_rn(q.x, inv_d), p.eps)));
    const float fb = p.post == TRDQ_NORM_NONE ? 1.0f : __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(__fmul_rn(q.y, inv_d), p.eps)));

    float2 t = make_float2(0.0f, 0.0f);
    Chunk dn[CH];
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      n[j] = chunk_scale(n[j], f);
      m[j] = chunk_scale(m[j], fb);
#pragma unroll
      for (int i = 0; i < 4; ++i) B[j].p[i] = __fadd2_rn(B[j].p[i], dh[j].p[i]);
      A[j] = chunk_fma(dh[j], n[j], A[j]);
      dn[j] = chunk_mul(dh[j], gain[j]);
      t = __fadd2_rn(t, make_float2(chunk_dot(dn[j], n[j]), chunk_sum(dn[j])));
    }
    t = cta.sum(t);
    const float along = -__fmul_rn(t.x, inv_d), mean = p.norm == TRDQ_NORM_LAYER ? -__fmul_rn(t.y, inv_d) : 0.0f;
    const float2 f2 = make_float2(f, f), along2 = make_float2(along, along), mean2 = make_float2(mean, mean);
    const float2 alpha2 = make_float2(p.alpha, p.alpha);
    Chunk du[CH];
#pragma unroll
    for (int j = 0; j < CH; ++j) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        dR[j].p[i] = __ffma2_rn(__ffma2_rn(n[j].p[i], along2, __fadd2_rn(dn[j].p[i], mean2)), f2, dR[j].p[i]);
      C[j] = chunk_fma(dR[j], m[j], C[j]);
      du[j] = chunk_mul(dR[j], gate[j]);
      if (p.dx && in[j]) {
        StreamChunk<F32> o;
        Chunk v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v.p[i] = __fmul2_rn(dR[j].p[i], alpha2);
        o.set(v);
        o.store(stream_row(p.dx, row, p.lddx, F32), threadIdx.x + j * blockDim.x);
      }
    }
    if (!p.db) continue;  // the same for every thread
    if (p.post != TRDQ_NORM_NONE) {
      float2 e = make_float2(0.0f, 0.0f);
#pragma unroll
      for (int j = 0; j < CH; ++j)
        if (in[j]) e = __fadd2_rn(e, make_float2(chunk_dot(du[j], m[j]), chunk_sum(du[j])));
      e = cta.sum(e);
      const float2 fb2 = make_float2(fb, fb), a2 = make_float2(-__fmul_rn(e.x, inv_d), -__fmul_rn(e.x, inv_d));
      const float me = p.post == TRDQ_NORM_LAYER ? -__fmul_rn(e.y, inv_d) : 0.0f;
#pragma unroll
      for (int j = 0; j < CH; ++j) {
#pragma unroll
        for (int i = 0; i < 4; ++i) du[j].p[i] = __fmul2_rn(__ffma2_rn(m[j].p[i], a2, __fadd2_rn(du[j].p[i], make_float2(me, me))), fb2);
      }
    }
#pragma unroll
    for (int j = 0; j < CH; ++j)
      if (in[j]) *(reinterpret_cast<uint4*>(p.db + row * p.lddb) + threadIdx.x + j * blockDim.x) = narrow(du[j]);
  }

  // this run's column sums
  const int64_t plane = static_cast<int64_t>(gridDim.x) * p.D;
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const int c = threadIdx.x + j * blockDim.x;
    if (!in[j]) continue;
    float* const at = p.workspace + static_cast<int64_t>(blockIdx.x) * p.D + 8 * c;
    auto put = [](float* to, const Chunk& v) {
      reinterpret_cast<float4*>(to)[0] = make_float4(v.p[0].x, v.p[0].y, v.p[1].x, v.p[1].y);
      reinterpret_cast<float4*>(to)[1] = make_float4(v.p[2].x, v.p[2].y, v.p[3].x, v.p[3].y);
    };
    if (p.dscale || p.dweight) put(at, A[j]);
    if (p.dshift) put(at + plane, B[j]);
    if (p.dgate || p.dpost_weight) put(at + 2 * plane, C[j]);
  }
}

// Joins the runs.  blockIdx.x < sample_blocks: the gradients of a sample's parameters, 32 columns; the CTAs behind them: those of the weights.
__global__ void __launch_bounds__(1024) gated_norm_join_kernel(const GatedNormBackward p) {
  __shared__ float part[3][32][33];
  const int lane = threadIdx.x, group = threadIdx.y, groups = blockDim.y;
  const int col = blockIdx.y * 32 + lane;
  const bool in = col < p.D;
  const int64_t count = static_cast<int64_t>(p.samples) * p.runs;
  const int64_t plane = count * p.D;
  const bool weights = blockIdx.x >= static_cast<unsigned>(p.sample_blocks);
  const int64_t first = weights ? 0 : static_cast<int64_t>(blockIdx.x) * p.runs;
  const int64_t runs = weights ? count : p.runs;
  griddep_wait();
  float a = 0.0f, b = 0.0f, c = 0.0f;
  if (in) {
    for (int64_t i = group; i < runs; i += groups) {
      const float* const at = p.workspace + (first + i) * p.D + col;
      if (weights) {
        const int64_t s = i / p.runs;
        if (p.dweight) a = __fmaf_rn(at[0], p.scale ? __fadd_rn(1.0f, __uint_as_float(static_cast<uint32_t>(p.scale[s * p.ld_scale + col]) << 16)) : 1.0f, a);
        if (p.dpost_weight) c = __fmaf_rn(at[2 * plane], p.gate ? __uint_as_float(static_cast<uint32_t>(p.gate[s * p.ld_gate + col]) << 16) : 1.0f, c);
      } else {
        if (p.dscale) a = __fadd_rn(a, at[0]);
        if (p.dshift) b = __fadd_rn(b, at[plane]);
        if (p.dgate) c = __fadd_rn(c, at[2 * plane]);
      }
    }
  }
  part[0][group][lane] = a;
  part[1][group][lane] = b;
  part[2][group][lane] = c;
  __syncthreads();
  if (group != 0 || !in) return;
  for (int g = 1; g < groups; ++g) {
    a = __fadd_rn(a, part[0][g][lane]);
    b = __fadd_rn(b, part[1][g][lane]);
    c = __fadd_rn(c, part[2][g][lane]);
  }
  auto bf = [](const uint16_t* v, int64_t i) { return v ? __uint_as_float(static_cast<uint32_t>(v[i]) << 16) : 1.0f; };
  if (weights) {
    if (p.dweight) p.dweight[col] = a;
    if (p.dpost_weight) p.dpost_weight[col] = c;
  } else {
    const int64_t at = static_cast<int64_t>(blockIdx.x) * p.D + col;
    if (p.dscale) p.dscale[at] = __fmul_rn(a, bf(p.weight, col));
    if (p.dshift) p.dshift[at] = b;
    if (p.dgate) p.dgate[at] = __fmul_rn(c, bf(p.post_weight, col));
  }
}

}  // namespace

// Runs a sample's rows are cut into: enough for every SM to hold several CTAs, none across two samples.
void gated_norm_backward_runs(int32_t M, int32_t rows_per_sample, int32_t* samples, int32_t* runs, int32_t* rows_per_run) {
  constexpr int kRuns = 148 * 6;
  const int64_t rps = std::min<int64_t>(rows_per_sample, M);
  const int64_t per = std::min<int64_t>(rps, (static_cast<int64_t>(M) + kRuns - 1) / kRuns);
  *samples = static_cast<int32_t>((M + rps - 1) / rps);
  *rows_per_run = static_cast<int32_t>(per);
  *runs = static_cast<int32_t>((rps + per - 1) / per);
}

trdq_status launch_gated_norm_backward(const GatedNormBackward& args, cudaStream_t stream) {
  GatedNormBackward p = args;
  const int64_t grid = static_cast<int64_t>(p.samples) * p.runs;
  if (grid > 0x7FFFFFFE || p.D > 2 * 8 * 32 * kMostWarps) return TRDQ_ERR_SHAPE;
  const int chunks = p.D / 8;
  const int ch = chunks > 32 * kMostWarps ? 2 : 1;
  const int threads = ((chunks + ch - 1) / ch + 31) / 32 * 32;
  const auto kernel = ch == 1 ? (p.f32 ? gated_norm_backward_kernel<1, true> : gated_norm_backward_kernel<1, false>)
                              : (p.f32 ? gated_norm_backward_kernel<2, true> : gated_norm_backward_kernel<2, false>);
  if (launch_overlapped(kernel, dim3(static_cast<unsigned>(grid)), dim3(threads), 0, stream, p) != cudaSuccess) return TRDQ_ERR_CUDA;
  const bool weights = p.dweight || p.dpost_weight, per_sample = p.dscale || p.dshift || p.dgate;
  if (!weights && !per_sample) return TRDQ_OK;
  const int groups = weights || p.runs > 8 ? 32 : std::max(1, p.runs);
  p.sample_blocks = per_sample ? p.samples : 0;
  const dim3 jgrid(static_cast<unsigned>(p.sample_blocks + (weights ? 1 : 0)), (p.D + 31) / 32);
  return launch_overlapped(gated_norm_join_kernel, jgrid, dim3(32, groups), 0, stream, p) == cudaSuccess ? TRDQ_OK : TRDQ_ERR_CUDA;
}

}  // namespace trdq

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

template <bool F32>
struct RowInputs {
  StreamChunk<F32> r, dr;
  uint4 b, dh;
};

template <int CH, bool F32>
__global__ void __launch_bounds__(32 * kRowWarps) gated_norm_backward_kernel(const GatedNormBackward p) {
  __shared__ float4 slots[RowSum::kSlots];
  RowSum sums(slots);
  const float inv_d = __fdiv_rn(1.0f, static_cast<float>(p.D));
  const int64_t s = blockIdx.x / p.runs;
  const int64_t run = blockIdx.x - s * p.runs;
  const int64_t sample0 = s * p.rows_per_sample;
  const int64_t row0 = sample0 + run * p.rows_per_run;
  const int64_t row1 = min(min(row0 + p.rows_per_run, sample0 + p.rows_per_sample), static_cast<int64_t>(p.M));
  const int rows = static_cast<int>(row1 > row0 ? row1 - row0 : 0);
  griddep_launch_dependents();
  griddep_wait();

  constexpr int kBytes = F32 ? 4 : 2;
  bool in[CH];
  int at[CH];
  const char *r_at[CH], *dr_at[CH], *b_at[CH], *dh_at[CH];
  char *dx_at[CH], *db_at[CH];
  Chunk gain[CH], gate[CH];  // (1 + scale) o w and gate o pw of this thread's columns
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
    gain[j] = gate[j] = chunk_shift(none, 1.0f);
    if (!in[j]) continue;
    if (p.scale) gain[j] = chunk_shift(widen(load_param(p.scale + s * p.ld_scale, at[j])), 1.0f);
    if (p.weight) gain[j] = chunk_mul(gain[j], widen(load_param(p.weight, at[j])));
    if (p.gate) gate[j] = widen(load_param(p.gate + s * p.ld_gate, at[j]));
    if (p.post_weight) gate[j] = chunk_mul(gate[j], widen(load_param(p.post_weight, at[j])));
  }

  RowInputs<F32> next[CH];
#pragma unroll
  for (int j = 0; j < CH; ++j) {  // what is not loaded (lanes outside the row, inputs that are not there) stays zero
    next[j].r.clear();
    next[j].dr.clear();
    next[j].b = next[j].dh = zero4();
  }
  auto fetch = [&](bool valid) {
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      if (valid && in[j]) {
        next[j].r.load(r_at[j]);
        if (p.dr) next[j].dr.load(dr_at[j]);
        if (p.b) next[j].b = *reinterpret_cast<const uint4*>(b_at[j]);
        next[j].dh = *reinterpret_cast<const uint4*>(dh_at[j]);
      }
      r_at[j] += p.ldr * kBytes;
      dr_at[j] += p.lddr * kBytes;
      b_at[j] += p.ldb * 2;
      dh_at[j] += p.lddh * 2;
    }
  };
  fetch(rows > 0);
  const float2 alpha2 = make_float2(p.alpha, p.alpha);
  for (int row = 0; row < rows; ++row) {
    Chunk n[CH], m[CH], dh[CH], dR[CH];
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      n[j] = next[j].r.value();
      m[j] = widen(next[j].b);
      dh[j] = widen(next[j].dh);
      dR[j] = next[j].dr.value();
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
      dn[j] = chunk_mul(dh[j], gain[j]);
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
      du[j] = chunk_mul(dR[j], gate[j]);
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

  // this run's column sums
  const int64_t plane = static_cast<int64_t>(gridDim.x) * p.D;
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    if (!in[j]) continue;
    float* const to = p.workspace + static_cast<int64_t>(blockIdx.x) * p.D + 8 * at[j];
    auto put = [](float* to, const Chunk& v) {
      reinterpret_cast<float4*>(to)[0] = make_float4(v.p[0].x, v.p[0].y, v.p[1].x, v.p[1].y);
      reinterpret_cast<float4*>(to)[1] = make_float4(v.p[2].x, v.p[2].y, v.p[3].x, v.p[3].y);
    };
    if (p.dscale || p.dweight) put(to, A[j]);
    if (p.dshift) put(to + plane, B[j]);
    if (p.dgate || p.dpost_weight) put(to + 2 * plane, C[j]);
  }
}

// Joins the runs, four columns a thread.  blockIdx.x < sample_blocks: the gradients of a sample's parameters; the CTAs behind them: those of the
// weights.  The blockDim.y groups of a CTA take every blockDim.y-th run, and their sums are added in order.
__global__ void __launch_bounds__(1024) gated_norm_join_kernel(const GatedNormBackward p) {
  __shared__ float4 part[3][32][32];
  const int lane = threadIdx.x, group = threadIdx.y, groups = blockDim.y;
  const int col = (blockIdx.y * 32 + lane) * 4;
  const bool in = col < p.D;
  const int64_t count = static_cast<int64_t>(p.samples) * p.runs;
  const int64_t plane = count * p.D;
  const bool weights = blockIdx.x >= static_cast<unsigned>(p.sample_blocks);
  const int64_t first = weights ? 0 : static_cast<int64_t>(blockIdx.x) * p.runs;
  const int64_t runs = weights ? count : p.runs;
  const bool want_a = weights ? p.dweight != nullptr : p.dscale != nullptr, want_b = !weights && p.dshift;
  const bool want_c = weights ? p.dpost_weight != nullptr : p.dgate != nullptr;
  griddep_wait();
  auto four = [](const uint16_t* v) {
    const uint2 w = *reinterpret_cast<const uint2*>(v);
    const float2 a = widen_bf16x2(w.x), b = widen_bf16x2(w.y);
    return make_float4(a.x, a.y, b.x, b.y);
  };
  auto fma4 = [](const float4& a, const float4& b, const float4& c) {
    return make_float4(__fmaf_rn(a.x, b.x, c.x), __fmaf_rn(a.y, b.y, c.y), __fmaf_rn(a.z, b.z, c.z), __fmaf_rn(a.w, b.w, c.w));
  };
  const float4 one = make_float4(1.0f, 1.0f, 1.0f, 1.0f);
  float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f), b = a, c = a;
  if (in) {
#pragma unroll 4
    for (int64_t i = group; i < runs; i += groups) {
      const float* const at = p.workspace + (first + i) * p.D + col;
      float4 ka = one, kc = one;
      if (weights) {
        const int64_t s = i / p.runs;
        if (p.scale) ka = RowSum::add(one, four(p.scale + s * p.ld_scale + col));
        if (p.gate) kc = four(p.gate + s * p.ld_gate + col);
      }
      if (want_a) a = fma4(*reinterpret_cast<const float4*>(at), ka, a);
      if (want_b) b = RowSum::add(b, *reinterpret_cast<const float4*>(at + plane));
      if (want_c) c = fma4(*reinterpret_cast<const float4*>(at + 2 * plane), kc, c);
    }
  }
  if (groups > 1) {
    part[0][group][lane] = a;
    part[1][group][lane] = b;
    part[2][group][lane] = c;
    __syncthreads();
    if (group != 0) return;
    for (int g = 1; g < groups; ++g) {
      a = RowSum::add(a, part[0][g][lane]);
      b = RowSum::add(b, part[1][g][lane]);
      c = RowSum::add(c, part[2][g][lane]);
    }
  }
  if (!in) return;
  auto put = [](float* to, const float4& v) { to[0] = v.x, to[1] = v.y, to[2] = v.z, to[3] = v.w; };  // (the outputs are only known to be floats)
  const float4 none = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (weights) {
    if (want_a) put(p.dweight + col, a);
    if (want_c) put(p.dpost_weight + col, c);
  } else {
    const int64_t at = static_cast<int64_t>(blockIdx.x) * p.D + col;
    if (want_a) put(p.dscale + at, p.weight ? fma4(a, four(p.weight + col), none) : a);
    if (want_b) put(p.dshift + at, b);
    if (want_c) put(p.dgate + at, p.post_weight ? fma4(c, four(p.post_weight + col), none) : c);
  }
}

}  // namespace

// Runs a sample's rows are cut into, none across two samples.  The SMs hold `slots` CTAs at once (128 registers a thread); a run costs
// its rows and about four more for its parameters and its sums, and the CTAs work through the runs in rounds.
void gated_norm_backward_runs(int32_t M, int32_t D, int32_t rows_per_sample, int32_t* samples, int32_t* runs, int32_t* rows_per_run) {
  constexpr int kSms = 148, kRunCost = 4;
  const int64_t slots = static_cast<int64_t>(kSms) * std::max(1, 512 / row_threads(D));
  const int64_t rps = std::min<int64_t>(rows_per_sample, M);
  const int64_t count = (M + rps - 1) / rps;
  int64_t best_rows = rps, best_cost = -1;
  for (int64_t rounds = 1; rounds <= 4; ++rounds) {
    const int64_t wanted = std::max<int64_t>(1, rounds * slots / count);
    const int64_t rows = (rps + wanted - 1) / wanted;
    const int64_t total = count * ((rps + rows - 1) / rows);
    const int64_t cost = (total + slots - 1) / slots * (rows + kRunCost);
    if (best_cost < 0 || cost < best_cost) {
      best_cost = cost;
      best_rows = rows;
    }
  }
  *samples = static_cast<int32_t>(count);
  *rows_per_run = static_cast<int32_t>(best_rows);
  *runs = static_cast<int32_t>((rps + best_rows - 1) / best_rows);
}

trdq_status launch_gated_norm_backward(const GatedNormBackward& args, cudaStream_t stream) {
  GatedNormBackward p = args;
  const int64_t grid = static_cast<int64_t>(p.samples) * p.runs;
  if (grid > 0x7FFFFFFE || row_threads(p.D) > 32 * kRowWarps) return TRDQ_ERR_SHAPE;
  const int ch = row_chunks(p.D), threads = row_threads(p.D);
  const auto kernel = ch == 1 ? (p.f32 ? gated_norm_backward_kernel<1, true> : gated_norm_backward_kernel<1, false>)
                              : (p.f32 ? gated_norm_backward_kernel<2, true> : gated_norm_backward_kernel<2, false>);
  if (launch_overlapped(kernel, dim3(static_cast<unsigned>(grid)), dim3(threads), 0, stream, p) != cudaSuccess) return TRDQ_ERR_CUDA;
  const bool weights = p.dweight || p.dpost_weight, per_sample = p.dscale || p.dshift || p.dgate;
  if (!weights && !per_sample) return TRDQ_OK;
  p.sample_blocks = per_sample ? p.samples : 0;
  const int64_t most = weights ? grid : p.runs;
  const int groups = most > 64 ? 32 : most > 8 ? 8 : most > 2 ? 2 : 1;
  const dim3 jgrid(static_cast<unsigned>(p.sample_blocks + (weights ? 1 : 0)), (p.D / 4 + 31) / 32);
  return launch_overlapped(gated_norm_join_kernel, jgrid, dim3(32, groups), 0, stream, p) == cudaSuccess ? TRDQ_OK : TRDQ_ERR_CUDA;
}

}  // namespace trdq

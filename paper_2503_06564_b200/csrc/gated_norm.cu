// What lies between the linears of two neighbouring sub-blocks, in one pass (trdq_gated_norm, trdq_gated_norm_fp8):
//   u = post(b) o pw,   r = stream(alpha x + gate_s o u),   n = norm(r) o w,   h = n o (1 + scale_s) + shift_s
// post and norm: LayerNorm or root mean square without parameters of their own, post also none; s = the sample of the row.  r is
// rounded to the stream's type before its statistics are taken, so h is the norm of what is stored: a program that reads r back, the
// backward pass first of all, sees the function that was computed.  h goes out in bf16, or, never stored, through the rotation of Eq. 10
// and the block quantizer of fp8.cuh.
//
// A CTA holds one row in registers, eight channels a thread (sixteen above 4096), so that each input is read once and the variance is
// a mean of squared deviations, not a difference of two large sums.  It walks down a run of neighbouring rows: the next row's inputs are
// requested before this one's are used, and the sample's parameters stay in registers until the sample changes.  Sixteen lanes hold a
// 128-block of the rotation: three butterfly stages in a thread, four by shuffle, in the order h = 1, 2, ..., 64 of the other kernels.
// What bounds it: memory, 8 bytes a channel with a bf16 stream, 7 with codes, and close behind it instruction issue.  32768 x 1152 (adaLN, bf16) 55 us, 5.5 TB/s of
// a measured 6.6; 8190 x 1152 to codes 22 us, issue alone (0.63 a clock and scheduler beside packed operations of two; without rotation and quantizer 15 us).
// More than 4096 channels, 4096 x 8192: bf16 52 us, fp32 stream 75, bf16 to codes 69, fp32 to codes 125; with an fp32 stream the 128 registers do not hold two chunks (40 bytes of
// a thread spill, 96 with codes).
// Measured and not better: two rows a step with one barrier (122 registers, 61 us); two rows that meet inside a warp where D is an odd multiple of 128 (65 us); groups
// of rows in a CTA with barriers of their own; 16 channels a thread (61 us); the inputs of two or three rows ahead in shared memory (55 us, codes 24 us).
#include <algorithm>

#include "fp8.cuh"
#include "gated_norm.cuh"
#include "ptx.cuh"

namespace trdq {
namespace {

__device__ __forceinline__ Chunk load_vec(const float* vec, int chunk) {
  const float4 a = __ldg(reinterpret_cast<const float4*>(vec) + 2 * chunk), b = __ldg(reinterpret_cast<const float4*>(vec) + 2 * chunk + 1);
  return Chunk{{make_float2(a.x, a.y), make_float2(a.z, a.w), make_float2(b.x, b.y), make_float2(b.z, b.w)}};
}

// 128-point transform of a block held by sixteen lanes, eight consecutive channels each.
__device__ __forceinline__ void wht128_lanes16(Chunk& c, int lane) {
#pragma unroll
  for (int i = 0; i < 4; ++i) c.p[i] = make_float2(__fadd_rn(c.p[i].x, c.p[i].y), __fsub_rn(c.p[i].x, c.p[i].y));
#pragma unroll
  for (int hb = 1; hb <= 2; hb <<= 1) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if ((i & hb) == 0) {
        const float2 a = c.p[i], d = c.p[i + hb];
        c.p[i] = __fadd2_rn(a, d);
        c.p[i + hb] = __ffma2_rn(d, make_float2(-1.0f, -1.0f), a);  // a - d, one rounding
      }
    }
  }
#pragma unroll
  for (int mask = 1; mask <= 8; mask <<= 1) {
    const float sgn = (lane & mask) ? -1.0f : 1.0f;  // upper lane: other - own, lower lane: own + other
    const float2 s2 = make_float2(sgn, sgn);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 other = make_float2(__shfl_xor_sync(0xffffffffu, c.p[i].x, mask), __shfl_xor_sync(0xffffffffu, c.p[i].y, mask));
      c.p[i] = __ffma2_rn(c.p[i], s2, other);
    }
  }
}

__device__ __forceinline__ float chunk_absmax(const Chunk& c) {
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) m = fmaxf(m, fmaxf(fabsf(c.p[i].x), fabsf(c.p[i].y)));
  return m;
}

template <int CH, bool F32, bool FP8>
__global__ void __launch_bounds__(32 * kRowWarps) gated_norm_kernel(const GatedNorm p, int32_t rows_per_cta) {
  __shared__ float4 slots[RowSum::kSlots];
  RowSum sums(slots);
  const int lane = threadIdx.x & 31;
  const float inv_d = __fdiv_rn(1.0f, static_cast<float>(p.D));
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * rows_per_cta;
  const int rows = static_cast<int>(min(static_cast<int64_t>(rows_per_cta), p.M - row0));
  griddep_launch_dependents();
  griddep_wait();

  // Addresses of this thread's chunks, moved on row by row.
  constexpr int kBytes = F32 ? 4 : 2;
  bool in[CH];
  int at[CH];
  const char *x_at[CH], *b_at[CH];
  char *r_at[CH], *out_at[CH];
  float* scale_at[CH];
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    at[j] = static_cast<int>(threadIdx.x + j * blockDim.x);
    in[j] = at[j] < p.D / 8;
    x_at[j] = stream_at(p.x, row0, p.ldx, at[j], F32);
    b_at[j] = stream_at(p.b, row0, p.ldb, at[j], false);
    r_at[j] = stream_at(p.r, row0, p.ldr, at[j], F32);
    out_at[j] = static_cast<char*>(p.out) + (row0 * p.ldo + 8 * at[j]) * (FP8 ? 1 : 2);
    if constexpr (FP8) scale_at[j] = p.scales + static_cast<int64_t>(at[j] / 16) * p.M + row0;
  }
  const Chunk none{{make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)}};

  StreamChunk<F32> next_x[CH];
  uint4 next_b[CH];
#pragma unroll
  for (int j = 0; j < CH; ++j) {  // what is not loaded (lanes outside the row, no branch) stays zero
    next_x[j].clear();
    next_b[j] = zero4();
  }
  auto fetch = [&](bool valid) {
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      if (valid && in[j]) {
        next_x[j].load(x_at[j]);
        if (p.b) next_b[j] = *reinterpret_cast<const uint4*>(b_at[j]);
      }
      x_at[j] += p.ldx * kBytes;
      b_at[j] += p.ldb * 2;
    }
  };
  fetch(rows > 0);

  Chunk gate[CH], gain[CH], shift[CH];  // gate o pw, (1 + scale) o w, shift of this thread's columns; with the rotation the last two times its vector
  int until = 0;                        // rows from row0 on that these hold for
  const float2 alpha2 = make_float2(p.alpha, p.alpha);
  for (int i = 0; i < rows; ++i) {
    if (i >= until) {
      const int64_t s = (row0 + i) / p.rows_per_sample;
      until = static_cast<int>(min((s + 1) * p.rows_per_sample - row0, static_cast<int64_t>(rows)));
      uint4 g[CH], sc[CH], sh[CH], w[CH], pw[CH];  // all requested before the first is used
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        const int c = in[j] ? at[j] : 0;
        g[j] = p.gate ? load_param(p.gate + s * p.ld_gate, c) : zero4();
        sc[j] = p.scale ? load_param(p.scale + s * p.ld_scale, c) : zero4();
        sh[j] = p.shift ? load_param(p.shift + s * p.ld_shift, c) : zero4();
        w[j] = p.weight ? load_param(p.weight, c) : zero4();
        pw[j] = p.post_weight ? load_param(p.post_weight, c) : zero4();
      }
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        gate[j] = p.gate ? widen(g[j]) : chunk_shift(none, 1.0f);
        if (p.post_weight) gate[j] = chunk_mul(gate[j], widen(pw[j]));
        gain[j] = chunk_shift(widen(sc[j]), 1.0f);
        if (p.weight) gain[j] = chunk_mul(gain[j], widen(w[j]));
        shift[j] = widen(sh[j]);
        if (!in[j]) shift[j] = none;
        if constexpr (FP8) {
          if (p.vec && in[j]) {
            const Chunk vec = load_vec(p.vec, at[j]);
            gain[j] = chunk_mul(gain[j], vec);
            shift[j] = chunk_mul(shift[j], vec);
          }
        }
      }
    }
    if (FP8 && i + 2 == until && until < rows) {  // soon the next sample's parameters (with bf16 out its registers cost a CTA an SM: 15.5 -> 19.3 us)
      const int64_t s = (row0 + until) / p.rows_per_sample;
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        if (p.gate && in[j]) prefetch_l1(p.gate + s * p.ld_gate + 8 * at[j]);
        if (p.scale && in[j]) prefetch_l1(p.scale + s * p.ld_scale + 8 * at[j]);
        if (p.shift && in[j]) prefetch_l1(p.shift + s * p.ld_shift + 8 * at[j]);
      }
    }
    StreamChunk<F32> x[CH];
    Chunk v[CH];
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      x[j] = next_x[j];
      v[j] = widen(next_b[j]);
    }
    fetch(i + 1 < rows);

    if (p.post != TRDQ_NORM_NONE) {
      const float f = row_centre(v, in, p.post, inv_d, p.eps, sums);
#pragma unroll
      for (int j = 0; j < CH; ++j) v[j] = chunk_scale(v[j], f);
    }
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const Chunk xv = x[j].value();
#pragma unroll
      for (int k = 0; k < 4; ++k) v[j].p[k] = __ffma2_rn(v[j].p[k], gate[j].p[k], __fmul2_rn(xv.p[k], alpha2));
      x[j].set(v[j]);
      v[j] = x[j].value();
      if (p.r && in[j]) x[j].store(r_at[j]);
      r_at[j] += p.ldr * kBytes;
    }
    const float f = row_centre(v, in, p.norm, inv_d, p.eps, sums);
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      v[j] = chunk_fma(chunk_scale(v[j], f), gain[j], shift[j]);
      if constexpr (FP8) {
        if (p.vec) wht128_lanes16(v[j], lane);
        float m = chunk_absmax(v[j]);
#pragma unroll
        for (int k = 1; k < 16; k <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, k));
        const Fp8Factor q = fp8_factor(m);
        if (in[j]) {
          const Chunk o = chunk_scale(v[j], q.mul);
          *reinterpret_cast<uint2*>(out_at[j]) = make_uint2(fp8_pack4(o.p[0], o.p[1]), fp8_pack4(o.p[2], o.p[3]));
          if ((lane & 15) == 0) *scale_at[j] = q.scale;
        }
        ++scale_at[j];
      } else {
        if (in[j]) *reinterpret_cast<uint4*>(out_at[j]) = narrow(v[j]);
      }
      out_at[j] += p.ldo * (FP8 ? 1 : 2);
    }
  }
}

template <int CH, bool F32, bool FP8>
cudaError_t launch(const GatedNorm& p, int dev, int sms, cudaStream_t stream) {
  // CTAs of this width that an SM holds at once
  static PerDevice<int> resident[kRowWarps];
  const int threads = row_threads(p.D);
  int per_sm = resident[threads / 32 - 1].get(dev);
  if (per_sm == 0) {
    const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, gated_norm_kernel<CH, F32, FP8>, threads, 0);
    if (e != cudaSuccess) return e;
    per_sm = std::max(1, per_sm);
    resident[threads / 32 - 1].set(dev, per_sm);
  }
  const int64_t ctas = std::min<int64_t>(p.M, static_cast<int64_t>(per_sm) * sms);
  const int32_t rows = static_cast<int32_t>((p.M + ctas - 1) / ctas);
  const unsigned grid = static_cast<unsigned>((static_cast<int64_t>(p.M) + rows - 1) / rows);
  return launch_overlapped(gated_norm_kernel<CH, F32, FP8>, dim3(grid), dim3(threads), 0, stream, p, rows);
}

template <int CH>
cudaError_t launch_chunks(const GatedNorm& p, int dev, int sms, cudaStream_t stream) {
  const bool fp8 = p.scales != nullptr;
  return p.f32 ? (fp8 ? launch<CH, true, true>(p, dev, sms, stream) : launch<CH, true, false>(p, dev, sms, stream))
               : (fp8 ? launch<CH, false, true>(p, dev, sms, stream) : launch<CH, false, false>(p, dev, sms, stream));
}

}  // namespace

trdq_status launch_gated_norm(const GatedNorm& p, cudaStream_t stream) {
  int dev = 0, sms = 148;
  if (cudaGetDevice(&dev) != cudaSuccess) return TRDQ_ERR_CUDA;
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (row_threads(p.D) > 32 * kRowWarps) return TRDQ_ERR_SHAPE;
  const cudaError_t e = row_chunks(p.D) == 1 ? launch_chunks<1>(p, dev, sms, stream) : launch_chunks<2>(p, dev, sms, stream);
  return e == cudaSuccess ? TRDQ_OK : TRDQ_ERR_CUDA;
}

}  // namespace trdq

// What lies between the linears of two neighbouring sub-blocks, in one pass (trdq_gated_norm, trdq_gated_norm_fp8):
//   u = post(b) o pw,   r = stream(alpha x + gate_s o u),   n = norm(r) o w,   h = n o (1 + scale_s) + shift_s
// post and norm: LayerNorm or root mean square without parameters of their own, post also none; s = the sample of the row.  r is
// rounded to the stream's type before its statistics are taken, so h is the norm of what is stored: a program that reads r back, the
// backward pass first of all, sees the function that was computed.  h goes out in bf16, or, never stored, through the rotation of Eq. 10
// and the block quantizer of fp8.cuh.
//
// A team of W warps holds a row in registers, CH chunks of eight channels a lane, so that each input is read once and the variance is the mean of
// squared deviations, not a difference of two large sums.  Sixteen lanes hold a 128-block: three butterfly stages in a thread, four
// by shuffle, in the order h = 1, 2, ..., 64 of the other kernels.
// What bounds it: memory.  8 bytes a channel with a bf16 stream, 7 with codes.
#include <algorithm>
#include <type_traits>

#include "fp8.cuh"
#include "gated_norm.cuh"
#include "ptx.cuh"

namespace trdq {
namespace {

constexpr int kWarps = 8;

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

// v -> (v - mean) or v, and 1 / sqrt(mean square + eps) of the result; chunks outside the row stay zero.
template <int W, int CH>
__device__ __forceinline__ float centre(Chunk (&v)[CH], const bool (&in)[CH], int kind, float d, float eps, TeamSum<W>& team) {
  if (kind == TRDQ_NORM_LAYER) {
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < CH; ++j) s = __fadd_rn(s, chunk_sum(v[j]));
    const float mean = __fdiv_rn(team.sum(s), d);
#pragma unroll
    for (int j = 0; j < CH; ++j)
      if (in[j]) v[j] = chunk_shift(v[j], -mean);
  }
  float q = 0.0f;
#pragma unroll
  for (int j = 0; j < CH; ++j) q = __fadd_rn(q, chunk_dot(v[j], v[j]));
  return __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(__fdiv_rn(team.sum(q), d), eps)));
}

template <int W, int CH, bool F32, bool FP8>
__global__ void __launch_bounds__(32 * kWarps) gated_norm_kernel(const GatedNorm p) {
  constexpr int kTeams = kWarps / W;
  __shared__ float slots[kTeams][TeamSum<W>::kFloats];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int team_id = warp / W;
  TeamSum<W> team(slots[team_id], team_id, warp % W);
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kTeams + team_id;
  griddep_launch_dependents();
  griddep_wait();
  if (row >= p.M) return;  // whole teams
  const int64_t s = row / p.rows_per_sample;
  const int chunks = p.D / 8;
  const int first = (warp % W) * 32 + lane;
  const float d = static_cast<float>(p.D);

  bool in[CH];
  StreamChunk<F32> x[CH];
  uint4 b[CH];
  const void* const xrow = stream_row(p.x, row, p.ldx, F32);
  const uint16_t* const brow = p.b ? p.b + row * p.ldb : nullptr;
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const int c = first + j * 32 * W;
    in[j] = c < chunks;
    x[j].clear();
    b[j] = zero4();
    if (in[j]) {
      x[j].load(xrow, c);
      if (brow) b[j] = *(reinterpret_cast<const uint4*>(brow) + c);
    }
  }
  Chunk v[CH];
  if (brow) {
#pragma unroll
    for (int j = 0; j < CH; ++j) v[j] = widen(b[j]);
    if (p.post != TRDQ_NORM_NONE) {
      const float f = centre<W, CH>(v, in, p.post, d, p.eps, team);
#pragma unroll
      for (int j = 0; j < CH; ++j) v[j] = chunk_scale(v[j], f);
    }
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const int c = first + j * 32 * W;
      if (!in[j]) continue;
      if (p.post_weight) v[j] = chunk_mul(v[j], widen(load_param(p.post_weight, c)));
      if (p.gate) v[j] = chunk_mul(v[j], widen(load_param(p.gate + s * p.ld_gate, c)));
    }
  } else {
#pragma unroll
    for (int j = 0; j < CH; ++j) v[j] = Chunk{{make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)}};
  }
  const float2 alpha2 = make_float2(p.alpha, p.alpha);
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const Chunk xv = x[j].value();
#pragma unroll
    for (int i = 0; i < 4; ++i) v[j].p[i] = brow ? __fadd2_rn(__fmul2_rn(xv.p[i], alpha2), v[j].p[i]) : __fmul2_rn(xv.p[i], alpha2);
    x[j].set(v[j]);
    v[j] = x[j].value();
  }
  if (p.r) {
    void* const rrow = stream_row(p.r, row, p.ldr, F32);
#pragma unroll
    for (int j = 0; j < CH; ++j)
      if (in[j]) x[j].store(rrow, first + j * 32 * W);
  }

  const float f = centre<W, CH>(v, in, p.norm, d, p.eps, team);
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const int c = first + j * 32 * W;
    v[j] = chunk_scale(v[j], f);
    if (in[j]) {
      if (p.weight) v[j] = chunk_mul(v[j], widen(load_param(p.weight, c)));
      if (p.scale) v[j] = chunk_mul(v[j], chunk_shift(widen(load_param(p.scale + s * p.ld_scale, c)), 1.0f));
      if (p.shift) {
        const Chunk sh = widen(load_param(p.shift + s * p.ld_shift, c));
#pragma unroll
        for (int i = 0; i < 4; ++i) v[j].p[i] = __fadd2_rn(v[j].p[i], sh.p[i]);
      }
    }
    if constexpr (FP8) {
      if (p.vec) {
        if (in[j]) v[j] = chunk_mul(v[j], load_vec(p.vec, c));
        wht128_lanes16(v[j], lane);
      }
      float m = chunk_absmax(v[j]);
#pragma unroll
      for (int k = 1; k < 16; k <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, k));
      const Fp8Factor q = fp8_factor(m);
      if (in[j]) {
        const Chunk o = chunk_scale(v[j], q.mul);
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.out) + row * p.D + 8 * c) = make_uint2(fp8_pack4(o.p[0], o.p[1]), fp8_pack4(o.p[2], o.p[3]));
        if ((lane & 15) == 0) p.scales[static_cast<int64_t>(c / 16) * p.M + row] = q.scale;
      }
    } else {
      if (in[j]) *(reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.out) + row * p.ldo) + c) = narrow(v[j]);
    }
  }
}

template <int W, int CH>
cudaError_t launch_shape(const GatedNorm& p, cudaStream_t stream) {
  constexpr int kTeams = kWarps / W;
  const unsigned grid = static_cast<unsigned>((static_cast<int64_t>(p.M) + kTeams - 1) / kTeams);
  const bool fp8 = p.scales != nullptr;
  const auto kernel = p.f32 ? (fp8 ? gated_norm_kernel<W, CH, true, true> : gated_norm_kernel<W, CH, true, false>)
                            : (fp8 ? gated_norm_kernel<W, CH, false, true> : gated_norm_kernel<W, CH, false, false>);
  return launch_overlapped(kernel, dim3(grid), dim3(32 * kWarps), 0, stream, p);
}

template <int W>
cudaError_t launch_warps(const GatedNorm& p, int ch, cudaStream_t stream) {
  switch (ch) {
    case 1: return launch_shape<W, 1>(p, stream);
    case 2: return launch_shape<W, 2>(p, stream);
    case 3: return launch_shape<W, 3>(p, stream);
    case 4: return launch_shape<W, 4>(p, stream);
    default: return launch_shape<W, 5>(p, stream);
  }
}

}  // namespace

trdq_status launch_gated_norm(const GatedNorm& p, cudaStream_t stream) {
  const int chunks = p.D / 8;
  int W = 1;
  while (W < kWarps && (chunks + 32 * W - 1) / (32 * W) > 5) W *= 2;
  const int ch = (chunks + 32 * W - 1) / (32 * W);
  if (ch > 5) return TRDQ_ERR_SHAPE;
  const cudaError_t e = W == 1 ? launch_warps<1>(p, ch, stream) : W == 2 ? launch_warps<2>(p, ch, stream) : W == 4 ? launch_warps<4>(p, ch, stream) : launch_warps<8>(p, ch, stream);
  return e == cudaSuccess ? TRDQ_OK : TRDQ_ERR_CUDA;
}

}  // namespace trdq

// Entry points of the block-scaled 8-bit float path and of the fused norms between a block's linears: argument validation on the
// host, before anything is launched.
#include <cmath>
#include <initializer_list>

#include "internal.h"

namespace trdq {
namespace {

bool aligned(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// Fused vector of t's group for K channels; rot == nullptr: none.
trdq_status rotation_vector(const trdq_rotation* rot, int32_t t, int32_t K, bool weight, const float** vec) {
  *vec = nullptr;
  if (!rot) return TRDQ_OK;
  if (rot->dense || rot->perm || rot->K != K) return TRDQ_ERR_MISMATCH;
  const int g = find_group(rot->t_bounds, t);
  if (g < 0) return TRDQ_ERR_TIMESTEP;
  if (!on_current_device(rot->device)) return TRDQ_ERR_MISMATCH;
  *vec = (weight ? rot->weight_vec : rot->act_vec) + static_cast<size_t>(g) * K;
  return TRDQ_OK;
}

bool blocks_of_128(int32_t K) { return K > 0 && K % TRDQ_BLOCK == 0 && K <= TRDQ_MAX_K; }

// A matrix of D columns in rows of ld elements of `bytes` each.
trdq_status check_matrix(const void* p, int64_t ld, int32_t D, int bytes) {
  if (ld < D) return TRDQ_ERR_SHAPE;
  return aligned(p, 16) && ld * bytes % 16 == 0 ? TRDQ_OK : TRDQ_ERR_ALIGN;
}

constexpr int32_t kMostChannels = 8192;

trdq_status check_op(const trdq_gated_norm_op* op) {
  if (!op) return TRDQ_ERR_NULL;
  if (op->M < 0 || op->D <= 0 || op->D % 8 != 0 || op->D > kMostChannels || op->rows_per_sample < 1) return TRDQ_ERR_SHAPE;
  if (op->norm != TRDQ_NORM_LAYER && op->norm != TRDQ_NORM_RMS) return TRDQ_ERR_SHAPE;
  if (op->post_norm != TRDQ_NORM_NONE && op->post_norm != TRDQ_NORM_LAYER && op->post_norm != TRDQ_NORM_RMS) return TRDQ_ERR_SHAPE;
  if (!(op->eps >= 0.0f) || !std::isfinite(op->eps) || !std::isfinite(op->res_scale)) return TRDQ_ERR_SHAPE;
  if (op->M == 0) return TRDQ_OK;
  if (!op->X) return TRDQ_ERR_NULL;
  if (!op->branch_bf16 && (op->gate_bf16 || op->post_weight_bf16 || op->post_norm != TRDQ_NORM_NONE)) return TRDQ_ERR_NULL;
  trdq_status st = check_matrix(op->X, op->ldx, op->D, op->stream_f32 ? 4 : 2);
  if (st == TRDQ_OK && op->branch_bf16) st = check_matrix(op->branch_bf16, op->ldb, op->D, 2);
  if (st == TRDQ_OK && op->gate_bf16) st = check_matrix(op->gate_bf16, op->ld_gate, op->D, 2);
  if (st == TRDQ_OK && op->shift_bf16) st = check_matrix(op->shift_bf16, op->ld_shift, op->D, 2);
  if (st == TRDQ_OK && op->scale_bf16) st = check_matrix(op->scale_bf16, op->ld_scale, op->D, 2);
  if (st == TRDQ_OK && !(aligned(op->weight_bf16, 16) && aligned(op->post_weight_bf16, 16))) st = TRDQ_ERR_ALIGN;
  return st;
}

trdq_status run_fp8_linear(const Fp8Linear& p, bool mute, void* stream) {
  if (p.M < 0 || p.N <= 0 || p.N % 16 != 0 || !blocks_of_128(p.K)) return TRDQ_ERR_SHAPE;
  if (p.act != TRDQ_ACT_NONE && p.act != TRDQ_ACT_GELU_TANH) return TRDQ_ERR_SHAPE;
  if (p.M == 0) return TRDQ_OK;
  if (!p.codes || !p.scales || !p.w_codes || !p.w_scales || !p.out) return TRDQ_ERR_NULL;
  if (p.ld < p.N) return TRDQ_ERR_SHAPE;
  if (p.ld % 8 != 0 || !aligned(p.out, 16) || !aligned(p.codes, 16) || !aligned(p.w_codes, 16) || !aligned(p.scales, 4) || !aligned(p.w_scales, 4) ||
      !aligned(p.bias_bf16, 8))
    return TRDQ_ERR_ALIGN;
  cudaStream_t const cs = static_cast<cudaStream_t>(stream);
  return finish(mute ? launch_gemm_fp8_pair(p, cs, true) : launch_gemm_fp8(p, cs), stream);
}

trdq_status run_gated_norm(const trdq_gated_norm_op* op, void* R, int64_t ldr, void* out, int64_t ldo, float* scales, const float* vec,
                           void* stream) {
  if (R) {
    const trdq_status st = check_matrix(R, ldr, op->D, op->stream_f32 ? 4 : 2);
    if (st != TRDQ_OK) return st;
    if (R == op->X && ldr != op->ldx && op->M > 1) return TRDQ_ERR_SHAPE;  // rows would be overwritten before they are read
  }
  GatedNorm p;
  p.x = op->X;
  p.b = static_cast<const uint16_t*>(op->branch_bf16);
  p.gate = static_cast<const uint16_t*>(op->gate_bf16);
  p.shift = static_cast<const uint16_t*>(op->shift_bf16);
  p.scale = static_cast<const uint16_t*>(op->scale_bf16);
  p.weight = static_cast<const uint16_t*>(op->weight_bf16);
  p.post_weight = static_cast<const uint16_t*>(op->post_weight_bf16);
  p.ldx = op->ldx;
  p.ldb = op->ldb;
  p.ld_gate = op->ld_gate;
  p.ld_shift = op->ld_shift;
  p.ld_scale = op->ld_scale;
  p.r = R;
  p.ldr = ldr;
  p.out = out;
  p.ldo = ldo;
  p.scales = scales;
  p.vec = vec;
  p.M = op->M;
  p.D = op->D;
  p.rows_per_sample = op->rows_per_sample;
  p.norm = op->norm;
  p.post = op->post_norm;
  p.eps = op->eps;
  p.alpha = op->res_scale;
  p.f32 = op->stream_f32 != 0;
  return finish(launch_gated_norm(p, static_cast<cudaStream_t>(stream)), stream);
}

}  // namespace
}  // namespace trdq

using namespace trdq;

extern "C" {

trdq_status trdq_fp8_quantize(const trdq_rotation* rot, int32_t t, const void* X_bf16, int64_t ldx, int32_t M, int32_t K, uint8_t* codes,
                              float* scales, void* stream) {
  if (M < 0 || !blocks_of_128(K)) return TRDQ_ERR_SHAPE;
  const float* vec;
  const trdq_status st = rotation_vector(rot, t, K, false, &vec);
  if (st != TRDQ_OK || M == 0) return st;
  if (!X_bf16 || !codes || !scales) return TRDQ_ERR_NULL;
  if (ldx < K) return TRDQ_ERR_SHAPE;
  if (ldx % 8 != 0 || !aligned(X_bf16, 16) || !aligned(codes, 16) || !aligned(scales, 4)) return TRDQ_ERR_ALIGN;
  return finish(launch_fp8_quantize(X_bf16, ldx, M, K, vec, codes, scales, static_cast<cudaStream_t>(stream)), stream);
}

trdq_status trdq_fp8_quantize_weights(const trdq_rotation* rot, int32_t t, const void* W_bf16, int32_t N, int32_t K, uint8_t* codes,
                                      float* scales, void* stream) {
  if (N <= 0 || N % 16 != 0 || !blocks_of_128(K)) return TRDQ_ERR_SHAPE;
  const float* vec;
  const trdq_status st = rotation_vector(rot, t, K, true, &vec);
  if (st != TRDQ_OK) return st;
  if (!W_bf16 || !codes || !scales) return TRDQ_ERR_NULL;
  if (!aligned(W_bf16, 16) || !aligned(codes, 16) || !aligned(scales, 4)) return TRDQ_ERR_ALIGN;
  return finish(launch_fp8_quantize_weights(W_bf16, N, K, vec, codes, scales, static_cast<cudaStream_t>(stream)), stream);
}

trdq_status trdq_fp8_linear(const uint8_t* codes, const float* scales, int32_t M, int32_t K, const uint8_t* w_codes, const float* w_scales,
                            int32_t N, const void* bias_bf16, void* Y_bf16, int64_t ldy, int32_t act, void* stream) {
  return run_fp8_linear(Fp8Linear{codes, scales, w_codes, w_scales, bias_bf16, Y_bf16, ldy, M, N, K, act}, false, stream);
}

trdq_status trdq_selftest_fp8_linear_expiry(const uint8_t* codes, const float* scales, int32_t M, int32_t K, const uint8_t* w_codes,
                                            const float* w_scales, int32_t N, void* Y_bf16, int64_t ldy, void* stream) {
  return run_fp8_linear(Fp8Linear{codes, scales, w_codes, w_scales, nullptr, Y_bf16, ldy, M, N, K, TRDQ_ACT_NONE}, true, stream);
}

trdq_status trdq_gated_norm(const trdq_gated_norm_op* op, void* R, int64_t ldr, void* H_bf16, int64_t ldh, void* stream) {
  trdq_status st = check_op(op);
  if (st != TRDQ_OK || op->M == 0) return st;
  if (!H_bf16) return TRDQ_ERR_NULL;
  st = check_matrix(H_bf16, ldh, op->D, 2);
  if (st != TRDQ_OK) return st;
  return run_gated_norm(op, R, ldr, H_bf16, ldh, nullptr, nullptr, stream);
}

trdq_status trdq_gated_norm_fp8(const trdq_gated_norm_op* op, const trdq_rotation* rot, int32_t t, void* R, int64_t ldr, uint8_t* codes,
                                float* scales, void* stream) {
  trdq_status st = check_op(op);
  if (st != TRDQ_OK) return st;
  if (op->D % TRDQ_BLOCK != 0) return TRDQ_ERR_SHAPE;
  const float* vec;
  st = rotation_vector(rot, t, op->D, false, &vec);
  if (st != TRDQ_OK || op->M == 0) return st;
  if (!codes || !scales) return TRDQ_ERR_NULL;
  if (!aligned(codes, 16) || !aligned(scales, 4)) return TRDQ_ERR_ALIGN;
  return run_gated_norm(op, R, ldr, codes, op->D, scales, vec, stream);
}

trdq_status trdq_gated_norm_backward_workspace(const trdq_gated_norm_op* op, uint64_t* bytes) {
  if (!op || !bytes) return TRDQ_ERR_NULL;
  if (op->M < 0 || op->D <= 0 || op->D % 8 != 0 || op->D > kMostChannels || op->rows_per_sample < 1) return TRDQ_ERR_SHAPE;
  *bytes = 0;
  if (op->M == 0) return TRDQ_OK;
  int32_t rows;
  int64_t entries;
  gated_norm_backward_runs(op->M, op->D, op->stream_f32 != 0, op->rows_per_sample, &rows, &entries);
  *bytes = 3ull * static_cast<uint64_t>(entries) * static_cast<uint64_t>(op->D) * sizeof(float);
  return TRDQ_OK;
}

trdq_status trdq_gated_norm_backward(const trdq_gated_norm_op* op, const void* dH_bf16, int64_t lddh, const void* dR, int64_t lddr, void* dX,
                                     int64_t lddx, void* dB_bf16, int64_t lddb, float* dgate, float* dshift, float* dscale, float* dweight,
                                     float* dpost_weight, void* workspace, uint64_t workspace_bytes, void* stream) {
  trdq_status st = check_op(op);
  if (st != TRDQ_OK) return st;
  for (const float* g : std::initializer_list<const float*>{dgate, dshift, dscale, dweight, dpost_weight})
    if (!aligned(g, 4)) return TRDQ_ERR_ALIGN;
  if (op->M == 0) {  // sums over no rows
    cudaStream_t const cs = static_cast<cudaStream_t>(stream);
    for (float* g : std::initializer_list<float*>{dweight, dpost_weight})
      if (g && cudaMemsetAsync(g, 0, static_cast<size_t>(op->D) * sizeof(float), cs) != cudaSuccess) return TRDQ_ERR_CUDA;
    return finish(TRDQ_OK, stream);
  }
  if (!dH_bf16 || (dgate && !op->gate_bf16) || (dshift && !op->shift_bf16) || (dscale && !op->scale_bf16) || (dweight && !op->weight_bf16) ||
      (dpost_weight && !op->post_weight_bf16) || (dB_bf16 && !op->branch_bf16))
    return TRDQ_ERR_NULL;
  const int stream_bytes = op->stream_f32 ? 4 : 2;
  st = check_matrix(dH_bf16, lddh, op->D, 2);
  if (st == TRDQ_OK && dR) st = check_matrix(dR, lddr, op->D, stream_bytes);
  if (st == TRDQ_OK && dX) st = check_matrix(dX, lddx, op->D, stream_bytes);
  if (st == TRDQ_OK && dB_bf16) st = check_matrix(dB_bf16, lddb, op->D, 2);
  if (st != TRDQ_OK) return st;
  if (dX && dX == dR && lddx != lddr && op->M > 1) return TRDQ_ERR_SHAPE;
  GatedNormBackward p;
  // without modulation the rows are one sample, which joins faster and needs no more workspace
  p.rows_per_sample = op->gate_bf16 || op->shift_bf16 || op->scale_bf16 ? op->rows_per_sample : op->M;
  gated_norm_backward_runs(op->M, op->D, op->stream_f32 != 0, p.rows_per_sample, &p.rows_per_run, &p.entries);
  if (dgate || dshift || dscale || dweight || dpost_weight) {
    uint64_t need = 0;
    trdq_gated_norm_backward_workspace(op, &need);
    if (!workspace) return TRDQ_ERR_NULL;
    if (!aligned(workspace, 16)) return TRDQ_ERR_ALIGN;
    if (workspace_bytes < need) return TRDQ_ERR_NOMEM;
  }
  p.r = op->X;
  p.dr = dR;
  p.b = static_cast<const uint16_t*>(op->branch_bf16);
  p.dh = static_cast<const uint16_t*>(dH_bf16);
  p.gate = static_cast<const uint16_t*>(op->gate_bf16);
  p.scale = static_cast<const uint16_t*>(op->scale_bf16);
  p.weight = static_cast<const uint16_t*>(op->weight_bf16);
  p.post_weight = static_cast<const uint16_t*>(op->post_weight_bf16);
  p.ldr = op->ldx;
  p.lddr = lddr;
  p.ldb = op->ldb;
  p.lddh = lddh;
  p.ld_gate = op->ld_gate;
  p.ld_scale = op->ld_scale;
  p.dx = dX;
  p.db = static_cast<uint16_t*>(dB_bf16);
  p.lddx = lddx;
  p.lddb = lddb;
  p.dgate = dgate;
  p.dshift = dshift;
  p.dscale = dscale;
  p.dweight = dweight;
  p.dpost_weight = dpost_weight;
  p.workspace = static_cast<float*>(workspace);
  p.M = op->M;
  p.D = op->D;
  p.norm = op->norm;
  p.post = op->post_norm;
  p.eps = op->eps;
  p.alpha = op->res_scale;
  p.f32 = op->stream_f32 != 0;
  return finish(launch_gated_norm_backward(p, static_cast<cudaStream_t>(stream)), stream);
}

}  // extern "C"

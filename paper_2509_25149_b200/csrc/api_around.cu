// C-ABI entry points around the linear layers: argument validation of the norm, the activation's gradient and the copies in 8 bits.
#include <cmath>

#include "around.h"
#include "common.cuh"

using namespace nvfp4;

namespace nvfp4 {

nvfp4_status check_copy8(const nvfp4_tensor* t, int64_t rows, int64_t cols) {
  if (!t || !t->codes || !t->scales) return NVFP4_ERR_NULL;
  if (t->format != NVFP4_FORMAT_MXFP8 || t->sf_layout != NVFP4_SF_LINEAR) return NVFP4_ERR_ARG;
  if (t->rows != rows || t->cols != cols || rows <= 0 || cols <= 0 || rows > (int64_t)1 << 30 || cols > (int64_t)1 << 30 || cols % 8 != 0)
    return NVFP4_ERR_SHAPE;
  if (!aligned(t->codes, 16) || !aligned(t->scales, 16)) return NVFP4_ERR_ALIGN;
  return NVFP4_OK;
}

}  // namespace nvfp4

namespace {

bool sizes_ok(int64_t rows, int64_t cols) {
  return rows > 0 && cols > 0 && rows <= (int64_t)1 << 30 && cols <= (int64_t)1 << 30 && cols % 8 == 0;
}
// a matrix that is there: its leading dimension and alignment
nvfp4_status check_matrix(const void* p, int64_t ld, int64_t cols, bool fp32) {
  if (!p) return NVFP4_OK;
  if (ld < cols) return NVFP4_ERR_SHAPE;
  if (ld % (fp32 ? 4 : 8) != 0 || !aligned(p, 16)) return NVFP4_ERR_ALIGN;
  return NVFP4_OK;
}
nvfp4_status status_of(cudaError_t e) { return e == cudaSuccess ? NVFP4_OK : NVFP4_ERR_CUDA; }
size_t bytes_of(int64_t floats) { return ((size_t)floats * 4 + 255) / 256 * 256; }

}  // namespace

extern "C" {

nvfp4_status nvfp4_dequantize_bf16(const nvfp4_tensor* t, void* out_bf16, int64_t ld, void* cuda_stream) {
  if (!t || !out_bf16) return NVFP4_ERR_NULL;
  nvfp4_status st = check_copy8(t, t->rows, t->cols);
  if (st != NVFP4_OK) return st;
  if ((st = check_matrix(out_bf16, ld, t->cols, false)) != NVFP4_OK) return st;
  return status_of(launch_dequantize8(*t, out_bf16, false, ld, static_cast<cudaStream_t>(cuda_stream)));
}

nvfp4_status nvfp4_rmsnorm_fwd(const void* x_bf16, int64_t ldx, const void* residual, int64_t ldr, int32_t residual_is_fp32,
                               const float* gain, int64_t rows, int64_t cols, float eps, void* h, int64_t ldh, void* y_bf16,
                               int64_t ldy, const nvfp4_tensor* y8, const nvfp4_tensor* h8, float* rstd, void* cuda_stream) {
  if (!x_bf16 || (!h && !y_bf16 && !y8 && !h8 && !rstd)) return NVFP4_ERR_NULL;
  if (!sizes_ok(rows, cols)) return NVFP4_ERR_SHAPE;
  if (!(eps > 0.f) || !std::isfinite(eps) || (h && !residual)) return NVFP4_ERR_ARG;
  const bool fp32 = residual_is_fp32 != 0;
  nvfp4_status st;
  if ((st = check_matrix(x_bf16, ldx, cols, false)) != NVFP4_OK || (st = check_matrix(residual, ldr, cols, fp32)) != NVFP4_OK ||
      (st = check_matrix(h, ldh, cols, fp32)) != NVFP4_OK || (st = check_matrix(y_bf16, ldy, cols, false)) != NVFP4_OK)
    return st;
  if (!aligned(gain, 16) || !aligned(rstd, 4)) return NVFP4_ERR_ALIGN;
  if ((y8 && (st = check_copy8(y8, rows, cols)) != NVFP4_OK) || (h8 && (st = check_copy8(h8, rows, cols)) != NVFP4_OK)) return st;
  NormFwd a{};
  a.x = x_bf16; a.residual = residual; a.gain = gain;
  a.h = h; a.y = y_bf16; a.rstd = rstd;
  a.y8 = y8; a.h8 = h8;
  a.rows = rows; a.cols = cols;
  a.ldx = ldx; a.ldr = ldr; a.ldh = ldh; a.ldy = ldy;
  a.eps = eps;
  a.fp32 = fp32;
  return status_of(launch_rmsnorm_fwd(a, static_cast<cudaStream_t>(cuda_stream)));
}

size_t nvfp4_rmsnorm_bwd_workspace_bytes(int64_t rows, int64_t cols) {
  return rows > 0 && cols > 0 ? bytes_of(rmsnorm_bwd_workspace_floats(rows, cols)) : 0;
}

nvfp4_status nvfp4_rmsnorm_bwd(const void* dy_bf16, int64_t lddy, const void* h, int64_t ldh, int32_t h_is_fp32,
                               const nvfp4_tensor* h8, const float* gain, const float* rstd, int64_t rows, int64_t cols,
                               const void* residual_grad, int64_t ldrg, void* dh, int64_t lddh, int32_t dh_is_fp32, float* dgain,
                               int32_t accumulate_dgain, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (!dy_bf16 || !rstd || !dh || (!h && !h8)) return NVFP4_ERR_NULL;
  if (h && h8) return NVFP4_ERR_ARG;
  if (!sizes_ok(rows, cols)) return NVFP4_ERR_SHAPE;
  const bool fp32 = dh_is_fp32 != 0;
  nvfp4_status st;
  if ((st = check_matrix(dy_bf16, lddy, cols, false)) != NVFP4_OK || (st = check_matrix(h, ldh, cols, h_is_fp32 != 0)) != NVFP4_OK ||
      (st = check_matrix(residual_grad, ldrg, cols, fp32)) != NVFP4_OK || (st = check_matrix(dh, lddh, cols, fp32)) != NVFP4_OK)
    return st;
  if (!aligned(gain, 16) || !aligned(rstd, 4) || !aligned(dgain, 4)) return NVFP4_ERR_ALIGN;
  if (h8 && (st = check_copy8(h8, rows, cols)) != NVFP4_OK) return st;
  if (dgain || rmsnorm_bwd_needs_workspace(cols)) {
    if (!workspace || workspace_bytes < nvfp4_rmsnorm_bwd_workspace_bytes(rows, cols)) return NVFP4_ERR_WORKSPACE;
    if (!aligned(workspace, 256)) return NVFP4_ERR_ALIGN;
  }
  NormBwd a{};
  a.dy = dy_bf16; a.h = h; a.h8 = h8;
  a.gain = gain; a.rstd = rstd;
  a.residual_grad = residual_grad;
  a.dh = dh; a.dgain = dgain;
  a.workspace = static_cast<float*>(workspace);
  a.rows = rows; a.cols = cols;
  a.lddy = lddy; a.ldh = ldh; a.ldrg = ldrg; a.lddh = lddh;
  a.h_fp32 = h_is_fp32 != 0; a.dh_fp32 = fp32; a.accumulate = accumulate_dgain != 0;
  return status_of(launch_rmsnorm_bwd(a, static_cast<cudaStream_t>(cuda_stream)));
}

size_t nvfp4_act_bwd_workspace_bytes(int64_t rows, int64_t cols) {
  return rows > 0 && cols > 0 ? bytes_of(act_bwd_workspace_floats(rows, cols)) : 0;
}

nvfp4_status nvfp4_act_bwd(const void* da_bf16, int64_t ldda, const void* z_bf16, int64_t ldz, const nvfp4_tensor* z8, int32_t act,
                           int64_t rows, int64_t cols, void* dz_bf16, int64_t lddz, void* a_bf16, int64_t lda, float* dbias,
                           int32_t accumulate_dbias, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (!da_bf16 || (!dz_bf16 && !a_bf16 && !dbias)) return NVFP4_ERR_NULL;
  if (act < NVFP4_ACT_NONE || act > NVFP4_ACT_GELU || (z_bf16 && z8)) return NVFP4_ERR_ARG;
  if (!z_bf16 && !z8 && (act != NVFP4_ACT_NONE || a_bf16)) return NVFP4_ERR_NULL;
  if (!sizes_ok(rows, cols)) return NVFP4_ERR_SHAPE;
  nvfp4_status st;
  if ((st = check_matrix(da_bf16, ldda, cols, false)) != NVFP4_OK || (st = check_matrix(z_bf16, ldz, cols, false)) != NVFP4_OK ||
      (st = check_matrix(dz_bf16, lddz, cols, false)) != NVFP4_OK || (st = check_matrix(a_bf16, lda, cols, false)) != NVFP4_OK)
    return st;
  if (!aligned(dbias, 4)) return NVFP4_ERR_ALIGN;
  if (z8 && (st = check_copy8(z8, rows, cols)) != NVFP4_OK) return st;
  if (dbias) {
    if (!workspace || workspace_bytes < nvfp4_act_bwd_workspace_bytes(rows, cols)) return NVFP4_ERR_WORKSPACE;
    if (!aligned(workspace, 256)) return NVFP4_ERR_ALIGN;
  }
  ActBwd a{};
  a.da = da_bf16; a.z = z_bf16; a.z8 = z8;
  a.dz = dz_bf16; a.a = a_bf16; a.dbias = dbias;
  a.workspace = static_cast<float*>(workspace);
  a.rows = rows; a.cols = cols;
  a.ldda = ldda; a.ldz = ldz; a.lddz = lddz; a.lda = lda;
  a.act = act;
  a.accumulate = accumulate_dbias != 0;
  return status_of(launch_act_bwd(a, static_cast<cudaStream_t>(cuda_stream)));
}

}  // extern "C"

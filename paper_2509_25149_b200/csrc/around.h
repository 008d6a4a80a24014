// Internal launch interface of the operators around the linear layers: copies in 8 bits, the norm, the activation's gradient.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "nvfp4.h"

namespace nvfp4 {

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
// argument check of a copy in 8 bits (api_around.cu)
nvfp4_status check_copy8(const nvfp4_tensor* t, int64_t rows, int64_t cols);

// copy8.cu
cudaError_t launch_quantize8(const void* x, bool fp32, int64_t rows, int64_t cols, int64_t ld, const nvfp4_tensor& q, cudaStream_t s);
cudaError_t launch_dequantize8(const nvfp4_tensor& q, void* out, bool out_fp32, int64_t ld, cudaStream_t s);

// norm.cu
struct NormFwd {
  const void* x;         // bf16
  const void* residual;  // NULL, bf16 or binary32
  const float* gain;     // NULL: ones
  void* h;               // NULL, or x + residual in the residual's type
  void* y;               // NULL or bf16
  float* rstd;           // NULL or one per row
  const nvfp4_tensor* y8;
  const nvfp4_tensor* h8;
  int64_t rows, cols, ldx, ldr, ldh, ldy;
  float eps;
  bool fp32;  // residual and h
};
cudaError_t launch_rmsnorm_fwd(const NormFwd& a, cudaStream_t s);
struct NormBwd {
  const void* dy;  // bf16
  const void* h;   // bf16 or binary32, or NULL
  const nvfp4_tensor* h8;
  const float* gain;  // NULL: ones
  const float* rstd;
  const void* residual_grad;  // NULL, or in dh's type
  void* dh;
  float* dgain;  // NULL: not wanted
  float* workspace;
  int64_t rows, cols, lddy, ldh, ldrg, lddh;
  bool h_fp32, dh_fp32, accumulate;
};
int64_t rmsnorm_bwd_workspace_floats(int64_t rows, int64_t cols);
bool rmsnorm_bwd_needs_workspace(int64_t cols);  // without dgain
cudaError_t launch_rmsnorm_bwd(const NormBwd& a, cudaStream_t s);

// act_bwd.cu
struct ActBwd {
  const void* da;  // bf16
  const void* z;   // bf16, or NULL
  const nvfp4_tensor* z8;
  void* dz;  // NULL or bf16
  void* a;   // NULL or bf16
  float* dbias;  // NULL: not wanted
  float* workspace;
  int64_t rows, cols, ldda, ldz, lddz, lda;
  int act;
  bool accumulate;
};
int64_t act_bwd_workspace_floats(int64_t rows, int64_t cols);
cudaError_t launch_act_bwd(const ActBwd& a, cudaStream_t s);

// out[c] = (accumulate ? out[c] : 0) + sum of `parts` rows of partial sums [parts x cols], in a fixed order (act_bwd.cu); where
// split > 0 the columns from there on go to out2, and out or out2 may be NULL
cudaError_t launch_column_sums(const float* partial, int64_t parts, int64_t cols, float* out, bool accumulate, cudaStream_t s,
                               float* out2 = nullptr, int64_t split = 0);

}  // namespace nvfp4

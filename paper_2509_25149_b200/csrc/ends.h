// Internal launch interface of the operators at the ends of a training step: head norms with rotation, embedding, log probabilities,
// gradient norm and clipping.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "nvfp4.h"

namespace nvfp4 {

// tokens, targets or positions
struct Indices {
  const void* p;
  bool wide;  // int64
#ifdef __CUDACC__
  __device__ __forceinline__ int64_t operator[](int64_t i) const {
    return wide ? static_cast<const int64_t*>(p)[i] : static_cast<const int32_t*>(p)[i];
  }
#endif
};

// heads.cu
struct Heads {
  const void* x;   // bf16
  const void* dy;  // gradient only
  void* y;         // y or dx
  const float* gain_q;
  const float* gain_k;
  const float* inv_freq;
  Indices positions;  // p == NULL: the row
  float* dgain_q;
  float* dgain_k;
  float* workspace;
  int64_t rows, ldx, lddy, ldy;
  int heads_q, heads_k, dim, rotary;
  float eps;
  bool interleaved, accumulate;
};
cudaError_t launch_headnorm_fwd(const Heads& a, cudaStream_t s);
int64_t headnorm_bwd_workspace_floats(int64_t rows, int heads_q, int heads_k, int dim);
cudaError_t launch_headnorm_bwd(const Heads& a, cudaStream_t s);

// embed.cu
struct Embed {
  Indices tokens;
  const void* table;  // or dout
  void* out;          // or dtable
  void* workspace;
  int64_t n, vocab, cols, ldt, ldo;  // ldt: of table or dtable, ldo: of out or dout
  float scale;
  bool in_fp32, out_fp32, accumulate;
};
cudaError_t launch_embedding_fwd(const Embed& a, cudaStream_t s);
size_t embedding_bwd_workspace(int64_t n, int64_t cols);
cudaError_t launch_embedding_bwd(const Embed& a, cudaStream_t s);

// logprob.cu
struct Logprob {
  const void* logits;
  Indices targets;  // p == NULL: none
  float* logprob;
  float* lse;
  float* stats;    // written by the forward pass, read by the gradient
  float* entropy;  // likewise
  int* top_ids;
  float* top_logprobs;
  const float* dlogprob;
  const float* dentropy;
  void* dlogits;
  int64_t rows, vocab, ld, lddl, dcols;
  float scale;
  int top;
  bool fp32, out_fp32;
};
cudaError_t launch_logprob_fwd(const Logprob& a, cudaStream_t s);
cudaError_t launch_logprob_bwd(const Logprob& a, cudaStream_t s);

// clip.cu
size_t grad_sq_norm_workspace();
cudaError_t launch_grad_sq_norm(const nvfp4_grad* grads, int n, double* sum, bool accumulate, double* workspace, cudaStream_t s);
cudaError_t launch_grad_clip(const nvfp4_grad* grads, int n, const double* sum, float max_norm, float* stats, cudaStream_t s);

}  // namespace nvfp4

// C-ABI entry points at the ends of a training step: argument validation of the head norms, the embedding, the log probabilities and clipping.
#include <cmath>

#include "around.h"
#include "common.cuh"
#include "ends.h"

using namespace nvfp4;

namespace {

constexpr int64_t kMost = (int64_t)1 << 30;  // rows, columns, tokens
nvfp4_status status_of(cudaError_t e) { return e == cudaSuccess ? NVFP4_OK : NVFP4_ERR_CUDA; }
size_t padded(size_t bytes) { return (bytes + 255) / 256 * 256; }

// a matrix: its leading dimension and alignment
nvfp4_status check_matrix(const void* p, int64_t ld, int64_t cols, bool fp32) {
  if (ld < cols) return NVFP4_ERR_SHAPE;
  if (ld % (fp32 ? 4 : 8) != 0 || !aligned(p, 16)) return NVFP4_ERR_ALIGN;
  return NVFP4_OK;
}
nvfp4_status check_indices(const void* p, int32_t wide) { return aligned(p, wide ? 8 : 4) ? NVFP4_OK : NVFP4_ERR_ALIGN; }
nvfp4_status check_workspace(const void* p, size_t bytes, size_t wanted) {
  if (!p || bytes < wanted) return NVFP4_ERR_WORKSPACE;
  return aligned(p, 256) ? NVFP4_OK : NVFP4_ERR_ALIGN;
}

bool head_sizes_ok(int64_t rows, int32_t heads_q, int32_t heads_k, int32_t dim) {
  return rows > 0 && rows <= kMost && heads_q >= 0 && heads_k >= 0 && (int64_t)heads_q + heads_k > 0 && dim > 0 && dim <= 256 && dim % 8 == 0 &&
         ((int64_t)heads_q + heads_k) * dim <= kMost;
}
nvfp4_status check_heads(const Heads& h, const void* positions) {
  if (!h.x || !h.y || (h.rotary != 0 && !h.inv_freq)) return NVFP4_ERR_NULL;
  if (!head_sizes_ok(h.rows, h.heads_q, h.heads_k, h.dim) || h.rotary < 0 || h.rotary > h.dim || h.rotary % 16 != 0) return NVFP4_ERR_SHAPE;
  if (!(h.eps >= 0x1p-126f) || !std::isfinite(h.eps)) return NVFP4_ERR_ARG;
  const int64_t cols = (int64_t)(h.heads_q + h.heads_k) * h.dim;
  nvfp4_status st;
  if ((st = check_matrix(h.x, h.ldx, cols, false)) != NVFP4_OK || (st = check_matrix(h.y, h.ldy, cols, false)) != NVFP4_OK) return st;
  if (!aligned(h.gain_q, 16) || !aligned(h.gain_k, 16) || !aligned(h.inv_freq, 4)) return NVFP4_ERR_ALIGN;
  return check_indices(positions, h.positions.wide);
}

nvfp4_status check_embed(const Embed& e) {
  if (!e.tokens.p || !e.table || !e.out) return NVFP4_ERR_NULL;
  if (e.n <= 0 || e.n > kMost || e.vocab <= 0 || e.vocab > kMost || e.cols <= 0 || e.cols > kMost || e.cols % 8 != 0) return NVFP4_ERR_SHAPE;
  if (!std::isfinite(e.scale)) return NVFP4_ERR_ARG;
  return check_indices(e.tokens.p, e.tokens.wide);
}

nvfp4_status check_logits(const Logprob& l) {
  if (l.rows <= 0 || l.rows > kMost || l.vocab <= 0 || l.vocab > kMost) return NVFP4_ERR_SHAPE;
  if (!(l.scale >= 0x1p-60f && l.scale <= 0x1p27f)) return NVFP4_ERR_ARG;
  nvfp4_status st;
  if ((st = check_matrix(l.logits, l.ld, l.vocab, l.fp32)) != NVFP4_OK) return st;
  if (!aligned(l.stats, 8) || !aligned(l.entropy, 4)) return NVFP4_ERR_ALIGN;
  return check_indices(l.targets.p, l.targets.wide);
}

nvfp4_status check_grads(const nvfp4_grad* grads, int32_t n, bool out) {
  if (!grads) return NVFP4_ERR_NULL;
  if (n <= 0) return NVFP4_ERR_SHAPE;
  for (int32_t i = 0; i < n; ++i) {
    const nvfp4_grad& g = grads[i];
    if (g.count < 0 || g.count > (int64_t)1 << 40) return NVFP4_ERR_SHAPE;
    if (g.count > 0 && !g.data) return NVFP4_ERR_NULL;
    if (!aligned(g.data, g.is_fp32 ? 4 : 2)) return NVFP4_ERR_ALIGN;
    if (!out || !g.out) continue;
    if (!aligned(g.out, g.out_is_fp32 ? 4 : 2)) return NVFP4_ERR_ALIGN;
    if (g.out == g.data && (g.out_is_fp32 != 0) != (g.is_fp32 != 0)) return NVFP4_ERR_ARG;
  }
  return NVFP4_OK;
}

}  // namespace

extern "C" {

nvfp4_status nvfp4_headnorm_fwd(const void* x_bf16, int64_t ldx, int64_t rows, int32_t heads_q, int32_t heads_k, int32_t head_dim,
                                const float* gain_q, const float* gain_k, float eps, const float* inv_freq, int32_t rotary_dim,
                                int32_t interleaved, const void* positions, int32_t positions_are_int64, void* y_bf16, int64_t ldy,
                                void* cuda_stream) {
  Heads h{};
  h.x = x_bf16; h.y = y_bf16;
  h.gain_q = gain_q; h.gain_k = gain_k;
  h.inv_freq = inv_freq;
  h.positions = Indices{positions, positions_are_int64 != 0};
  h.rows = rows; h.ldx = ldx; h.ldy = ldy;
  h.heads_q = heads_q; h.heads_k = heads_k;
  h.dim = head_dim; h.rotary = rotary_dim;
  h.eps = eps;
  h.interleaved = interleaved != 0;
  const nvfp4_status st = check_heads(h, positions);
  if (st != NVFP4_OK) return st;
  if (y_bf16 == x_bf16 && ldx != ldy) return NVFP4_ERR_ARG;
  return status_of(launch_headnorm_fwd(h, static_cast<cudaStream_t>(cuda_stream)));
}

size_t nvfp4_headnorm_bwd_workspace_bytes(int64_t rows, int32_t heads_q, int32_t heads_k, int32_t head_dim) {
  return head_sizes_ok(rows, heads_q, heads_k, head_dim) ? padded((size_t)headnorm_bwd_workspace_floats(rows, heads_q, heads_k, head_dim) * 4) : 0;
}

nvfp4_status nvfp4_headnorm_bwd(const void* dy_bf16, int64_t lddy, const void* x_bf16, int64_t ldx, int64_t rows, int32_t heads_q,
                                int32_t heads_k, int32_t head_dim, const float* gain_q, const float* gain_k, float eps,
                                const float* inv_freq, int32_t rotary_dim, int32_t interleaved, const void* positions,
                                int32_t positions_are_int64, void* dx_bf16, int64_t lddx, float* dgain_q, float* dgain_k,
                                int32_t accumulate_dgain, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (!dy_bf16) return NVFP4_ERR_NULL;
  Heads h{};
  h.x = x_bf16; h.dy = dy_bf16; h.y = dx_bf16;
  h.gain_q = gain_q; h.gain_k = gain_k;
  h.inv_freq = inv_freq;
  h.positions = Indices{positions, positions_are_int64 != 0};
  h.dgain_q = dgain_q; h.dgain_k = dgain_k;
  h.workspace = static_cast<float*>(workspace);
  h.rows = rows; h.ldx = ldx; h.lddy = lddy; h.ldy = lddx;
  h.heads_q = heads_q; h.heads_k = heads_k;
  h.dim = head_dim; h.rotary = rotary_dim;
  h.eps = eps;
  h.interleaved = interleaved != 0; h.accumulate = accumulate_dgain != 0;
  nvfp4_status st = check_heads(h, positions);
  if (st != NVFP4_OK || (st = check_matrix(dy_bf16, lddy, (int64_t)(heads_q + heads_k) * head_dim, false)) != NVFP4_OK) return st;
  if (!aligned(dgain_q, 4) || !aligned(dgain_k, 4)) return NVFP4_ERR_ALIGN;
  if ((dx_bf16 == dy_bf16 && lddx != lddy) || (dx_bf16 == x_bf16 && lddx != ldx)) return NVFP4_ERR_ARG;
  if ((dgain_q || dgain_k) &&
      (st = check_workspace(workspace, workspace_bytes, nvfp4_headnorm_bwd_workspace_bytes(rows, heads_q, heads_k, head_dim))) != NVFP4_OK)
    return st;
  return status_of(launch_headnorm_bwd(h, static_cast<cudaStream_t>(cuda_stream)));
}

nvfp4_status nvfp4_embedding_fwd(const void* tokens, int32_t tokens_are_int64, int64_t n, const void* table, int32_t table_is_fp32,
                                 int64_t ldt, int64_t vocab, int64_t cols, float scale, void* out, int32_t out_is_fp32, int64_t ldo,
                                 void* cuda_stream) {
  Embed e{};
  e.tokens = Indices{tokens, tokens_are_int64 != 0};
  e.table = table; e.out = out;
  e.n = n; e.vocab = vocab; e.cols = cols;
  e.ldt = ldt; e.ldo = ldo;
  e.scale = scale;
  e.in_fp32 = table_is_fp32 != 0; e.out_fp32 = out_is_fp32 != 0;
  nvfp4_status st = check_embed(e);
  if (st != NVFP4_OK || (st = check_matrix(table, ldt, cols, e.in_fp32)) != NVFP4_OK || (st = check_matrix(out, ldo, cols, e.out_fp32)) != NVFP4_OK)
    return st;
  return status_of(launch_embedding_fwd(e, static_cast<cudaStream_t>(cuda_stream)));
}

size_t nvfp4_embedding_bwd_workspace_bytes(int64_t n, int64_t vocab, int64_t cols) {
  return n > 0 && n <= kMost && vocab > 0 && vocab <= kMost && cols > 0 && cols <= kMost ? padded(embedding_bwd_workspace(n, cols)) : 0;
}

nvfp4_status nvfp4_embedding_bwd(const void* tokens, int32_t tokens_are_int64, int64_t n, const void* dout, int32_t dout_is_fp32, int64_t lddo,
                                 int64_t vocab, int64_t cols, float scale, float* dtable, int64_t lddt, int32_t accumulate, void* workspace,
                                 size_t workspace_bytes, void* cuda_stream) {
  Embed e{};
  e.tokens = Indices{tokens, tokens_are_int64 != 0};
  e.table = dout; e.out = dtable;
  e.workspace = workspace;
  e.n = n; e.vocab = vocab; e.cols = cols;
  e.ldt = lddt; e.ldo = lddo;
  e.scale = scale;
  e.in_fp32 = dout_is_fp32 != 0; e.out_fp32 = true; e.accumulate = accumulate != 0;
  nvfp4_status st = check_embed(e);
  if (st != NVFP4_OK || (st = check_matrix(dout, lddo, cols, e.in_fp32)) != NVFP4_OK || (st = check_matrix(dtable, lddt, cols, true)) != NVFP4_OK ||
      (st = check_workspace(workspace, workspace_bytes, nvfp4_embedding_bwd_workspace_bytes(n, vocab, cols))) != NVFP4_OK)
    return st;
  return status_of(launch_embedding_bwd(e, static_cast<cudaStream_t>(cuda_stream)));
}

nvfp4_status nvfp4_logprob_fwd(const void* logits, int32_t logits_are_fp32, int64_t ld, int64_t rows, int64_t vocab, const void* targets,
                               int32_t targets_are_int64, float scale, float* logprob, float* lse, float* stats, float* entropy, int32_t top,
                               int32_t* top_ids, float* top_logprobs, void* cuda_stream) {
  if (!logits || (!logprob && !lse && !stats && !entropy && !top_ids && !top_logprobs) || (logprob && !targets)) return NVFP4_ERR_NULL;
  Logprob l{};
  l.logits = logits;
  l.targets = Indices{targets, targets_are_int64 != 0};
  l.logprob = logprob; l.lse = lse; l.stats = stats; l.entropy = entropy;
  l.top_ids = top_ids; l.top_logprobs = top_logprobs;
  l.rows = rows; l.vocab = vocab; l.ld = ld;
  l.scale = scale;
  l.top = top;
  l.fp32 = logits_are_fp32 != 0;
  const nvfp4_status st = check_logits(l);
  if (st != NVFP4_OK) return st;
  if ((top_ids || top_logprobs) && (top < 1 || top > NVFP4_TOP_MAX || top > vocab)) return NVFP4_ERR_SHAPE;
  if (!aligned(logprob, 4) || !aligned(lse, 4) || !aligned(top_ids, 4) || !aligned(top_logprobs, 4)) return NVFP4_ERR_ALIGN;
  return status_of(launch_logprob_fwd(l, static_cast<cudaStream_t>(cuda_stream)));
}

nvfp4_status nvfp4_logprob_bwd(const void* logits, int32_t logits_are_fp32, int64_t ld, int64_t rows, int64_t vocab, const void* targets,
                               int32_t targets_are_int64, float scale, const float* stats, const float* entropy, const float* dlogprob,
                               const float* dentropy, void* dlogits, int32_t dlogits_are_fp32, int64_t lddl, int64_t dcols, void* cuda_stream) {
  if (!logits || !stats || !dlogits || (!dlogprob && !dentropy) || (dlogprob && !targets) || (dentropy && !entropy)) return NVFP4_ERR_NULL;
  Logprob l{};
  l.logits = logits;
  l.targets = Indices{dlogprob ? targets : nullptr, targets_are_int64 != 0};
  l.stats = const_cast<float*>(stats); l.entropy = const_cast<float*>(entropy);
  l.dlogprob = dlogprob; l.dentropy = dentropy;
  l.dlogits = dlogits;
  l.rows = rows; l.vocab = vocab; l.ld = ld; l.lddl = lddl; l.dcols = dcols;
  l.scale = scale;
  l.fp32 = logits_are_fp32 != 0; l.out_fp32 = dlogits_are_fp32 != 0;
  nvfp4_status st = check_logits(l);
  if (st != NVFP4_OK) return st;
  if (dcols < vocab || dcols > kMost + 8) return NVFP4_ERR_SHAPE;
  if ((st = check_matrix(dlogits, lddl, dcols, l.out_fp32)) != NVFP4_OK) return st;
  if (!aligned(dlogprob, 4) || !aligned(dentropy, 4)) return NVFP4_ERR_ALIGN;
  if (dlogits == logits && (l.fp32 != l.out_fp32 || (rows > 1 && ld != lddl))) return NVFP4_ERR_ARG;  // (a single row has no next one)
  return status_of(launch_logprob_bwd(l, static_cast<cudaStream_t>(cuda_stream)));
}

size_t nvfp4_grad_sq_norm_workspace_bytes(void) { return padded(grad_sq_norm_workspace()); }

nvfp4_status nvfp4_grad_sq_norm(const nvfp4_grad* grads, int32_t n, double* sum, int32_t accumulate, void* workspace, size_t workspace_bytes,
                                void* cuda_stream) {
  if (!sum) return NVFP4_ERR_NULL;
  nvfp4_status st = check_grads(grads, n, false);
  if (st != NVFP4_OK) return st;
  if (!aligned(sum, 8)) return NVFP4_ERR_ALIGN;
  if ((st = check_workspace(workspace, workspace_bytes, nvfp4_grad_sq_norm_workspace_bytes())) != NVFP4_OK) return st;
  return status_of(launch_grad_sq_norm(grads, n, sum, accumulate != 0, static_cast<double*>(workspace), static_cast<cudaStream_t>(cuda_stream)));
}

nvfp4_status nvfp4_grad_clip(const nvfp4_grad* grads, int32_t n, const double* sum, float max_norm, float* stats, void* cuda_stream) {
  if (!sum) return NVFP4_ERR_NULL;
  const nvfp4_status st = check_grads(grads, n, true);
  if (st != NVFP4_OK) return st;
  if (!(max_norm > 0.f) || !std::isfinite(max_norm)) return NVFP4_ERR_ARG;
  if (!aligned(sum, 8) || !aligned(stats, 4)) return NVFP4_ERR_ALIGN;
  return status_of(launch_grad_clip(grads, n, sum, max_norm, stats, static_cast<cudaStream_t>(cuda_stream)));
}

}  // extern "C"

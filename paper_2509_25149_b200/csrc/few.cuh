// Products of few rows and their epilogue, z = A B^T + bias, D = act(z) + residual: what gemm_few.cu and gemm_tokens.cuh share.  A lane has a column of
// D there, a warp a block of 32 of them, so that a row's block of the copy in 8 bits is a warp's.
#pragma once
#include "act.cuh"
#include "around.h"
#include "copy8.cuh"
#include "gemm.h"

namespace nvfp4 {

struct FewArgs {
  const uint16_t* a;
  const uint16_t* b;
  uint16_t* d;
  const float* bias;
  const uint16_t* residual;
  uint16_t* z;
  Copy8 z8;
  int64_t lda, ldb, ldd, ldr, ldz;
  int M, N, K, act, shares;  // shares: CTAs of a cluster
  int chain;                 // tokens_kernel with z in 8 bits: k-blocks of an accumulator
};

inline FewArgs few_args(const DenseGemmArgs& g, const EpilogueArgs& e) {
  FewArgs a{};
  a.a = static_cast<const uint16_t*>(g.a);
  a.b = static_cast<const uint16_t*>(g.b);
  a.d = static_cast<uint16_t*>(g.d);
  a.bias = e.bias;
  a.residual = static_cast<const uint16_t*>(e.residual);
  a.z = static_cast<uint16_t*>(e.z);
  a.z8 = Copy8{e.z8_codes, e.z8_scales, blocks8(g.N)};
  a.lda = g.lda; a.ldb = g.ldb; a.ldd = g.ldd; a.ldr = e.ldr; a.ldz = e.ldz;
  a.M = g.M; a.N = g.N; a.K = g.K;
  a.act = e.act;
  return a;
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
template <int ACT, int OWN>
__device__ __forceinline__ void activate_all(float (&v)[OWN]) {
#pragma unroll
  for (int j = 0; j < OWN; ++j) v[j] = act_value<ACT>(v[j]);
}

// What follows the sums v: rows first, first + stride, ... (OWN of them) of the 32 columns from n0 on, a lane to a column.  What it reads is asked
// for before the sums are there: the bias once (0.3 us where each call loaded it), the residual by residual_rows.  Each question is asked once for all
// rows: asked for row after row they were 0.14 us a row, of jumps over code that did not apply.
__device__ __forceinline__ float bias_of(const FewArgs& g, int n) { return g.bias && n < g.N ? g.bias[n] : 0.f; }
template <int OWN>
__device__ __forceinline__ void residual_rows(const FewArgs& g, float (&res)[OWN], int n, int first, int stride) {
  if (!g.residual || n >= g.N) return;
#pragma unroll
  for (int j = 0; j < OWN; ++j) {
    const int64_t m = first + j * stride;
    res[j] = m < g.M ? bf16_lo(g.residual[m * g.ldr + n]) : 0.f;
  }
}
template <int OWN>
__device__ __forceinline__ void finish_rows(const FewArgs& g, float (&v)[OWN], const float (&res)[OWN], float bias, int n0, int first, int stride,
                                            int lane) {
  const int n = n0 + lane;
  const bool live = n < g.N;
#pragma unroll
  for (int j = 0; j < OWN; ++j) v[j] += bias;
  if (g.z8.codes) {
#pragma unroll
    for (int j = 0; j < OWN; ++j) {
      const int64_t m = first + j * stride;
      if (m >= g.M) break;  // (the same for the whole warp)
      float top = live ? fabsf(v[j]) : 0.f;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      const uint32_t byte = scale_byte8(top);
      if (live) g.z8.codes[m * g.N + n] = (uint8_t)e4m3x4(v[j] * encode_scale8(byte), 0.f, 0.f, 0.f);
      if (lane == 0) g.z8.scales[m * g.z8.blocks + (n0 >> 5)] = (uint8_t)byte;
    }
  }
  if (!live) return;
  if (g.z) {
#pragma unroll
    for (int j = 0; j < OWN; ++j) {
      const int64_t m = first + j * stride;
      if (m < g.M) g.z[m * g.ldz + n] = (uint16_t)pack2(v[j], 0.f);
    }
  }
  switch (g.act) {
    case NVFP4_ACT_RELU2: activate_all<NVFP4_ACT_RELU2>(v); break;
    case NVFP4_ACT_SILU: activate_all<NVFP4_ACT_SILU>(v); break;
    case NVFP4_ACT_GELU: activate_all<NVFP4_ACT_GELU>(v); break;
    default: break;
  }
  if (g.residual) {
#pragma unroll
    for (int j = 0; j < OWN; ++j) v[j] += res[j];
  }
#pragma unroll
  for (int j = 0; j < OWN; ++j) {
    const int64_t m = first + j * stride;
    if (m < g.M) g.d[m * g.ldd + n] = (uint16_t)pack2(v[j], 0.f);
  }
}

}  // namespace nvfp4

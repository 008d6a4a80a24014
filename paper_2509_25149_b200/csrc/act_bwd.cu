// The gradient through an activation, dz = da act'(z), with the bias gradient (the column sums of dz) and, where asked, act(z) made
// again for the weight gradient of the layer behind: from the z that the product's epilogue kept, in bf16 or in 8 bits.
// Bound by HBM (da 2, z 1 + 1/32 or 2, dz 2, a 2 bytes per element), so everything is one pass: a CTA takes 256 columns and a run
// of rows, a lane eight neighbouring columns, and their sums stay in its registers.  The sums of a CTA leave as a row of partial
// sums, which a second kernel adds in a fixed order: no atomics, the same bits in every run.
#include "act.cuh"
#include "around.h"
#include "copy8.cuh"

namespace nvfp4 {

namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps, kCols = 256, kDepth = 4;

// Rows of a CTA: about eight rounds of four CTAs on each of 148 SMs, so that the last round is a small part of the whole, but
// 64 rows at least where there are so many
int64_t chunk_rows(int64_t rows, int64_t cols) {
  const int64_t strips = (cols + kCols - 1) / kCols, chunks = (4736 + strips - 1) / strips;
  int64_t n = (rows + chunks - 1) / chunks;
  n = n < 64 ? 64 : n;
  return (n + kWarps * kDepth - 1) / (kWarps * kDepth) * (kWarps * kDepth);
}
int64_t chunk_count(int64_t rows, int64_t cols) {
  const int64_t n = chunk_rows(rows, cols);
  return (rows + n - 1) / n;
}

struct Args {
  const uint16_t* da;
  const uint16_t* z;
  Copy8 z8;
  uint16_t* dz;
  uint16_t* a;
  float* partial;  // NULL: no bias gradient
  int64_t rows, cols, ldda, ldz, lddz, lda, chunk_rows;
};

template <int ACT, bool Z8>
__global__ void __launch_bounds__(kThreads) act_bwd_kernel(const Args g) {
  griddep_wait();
  griddep_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t col = (int64_t)blockIdx.x * kCols + lane * 8;
  const bool live = col < g.cols, have_z = ACT != NVFP4_ACT_NONE || g.a != nullptr;
  const int64_t r0 = (int64_t)blockIdx.y * g.chunk_rows, r1 = min(r0 + g.chunk_rows, g.rows);
  float sum[8] = {};
  for (int64_t r = r0 + warp; live && r < r1; r += kWarps * kDepth) {
    uint4 da[kDepth], z[kDepth];
    uint2 codes[kDepth];
    uint32_t byte[kDepth];
#pragma unroll
    for (int u = 0; u < kDepth; ++u) {
      const int64_t row = r + u * kWarps;
      if (row >= r1) break;
      da[u] = ldg128_stream(g.da + row * g.ldda + col);
      if (have_z) {
        if (Z8) {
          codes[u] = ldg64_stream(g.z8.codes + row * g.cols + col);
          byte[u] = ldg8(g.z8.scales + row * g.z8.blocks + (col >> 5));
        } else {
          z[u] = ldg128_stream(g.z + row * g.ldz + col);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kDepth; ++u) {
      const int64_t row = r + u * kWarps;
      if (row >= r1) break;
      float d[8], v[8] = {}, out[8], a[8];
      unpack8(da[u], d);
      if (have_z) {
        if (Z8)
          decode8(codes[u], decode_scale8(byte[u]), v);
        else
          unpack8(z[u], v);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        out[i] = d[i] * act_slope<ACT>(v[i], a[i]);
        sum[i] += out[i];
      }
      if (g.dz) store8<false>(g.dz, row * g.lddz + col, out);
      if (g.a) store8<false>(g.a, row * g.lda + col, a);
    }
  }
  if (!g.partial) return;
  __shared__ float part[kWarps][kCols];
#pragma unroll
  for (int i = 0; i < 8; ++i) part[warp][lane * 8 + i] = sum[i];
  __syncthreads();
  const int64_t c = (int64_t)blockIdx.x * kCols + threadIdx.x;
  if (c >= g.cols) return;
  float total = 0.f;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) total += part[w][threadIdx.x];
  g.partial[(int64_t)blockIdx.y * g.cols + c] = total;
}

constexpr int kShares = 8;

// 32 columns to a CTA; every warp sums a share of the rows, one thread a column's eight shares
__global__ void __launch_bounds__(32 * kShares) column_sums_kernel(const float* partial, int64_t parts, int64_t cols, float* out,
                                                                   int accumulate) {
  griddep_wait();
  griddep_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t c = (int64_t)blockIdx.x * 32 + lane;
  const int64_t p0 = parts * warp / kShares, p1 = parts * (warp + 1) / kShares;
  float s = 0.f;
  if (c < cols) {
    const float* p = partial + p0 * cols + c;
#pragma unroll 8
    for (int64_t k = p0; k < p1; ++k, p += cols) s += *p;
  }
  __shared__ float share[kShares][32];
  share[warp][lane] = s;
  __syncthreads();
  if (warp != 0 || c >= cols) return;
  float total = 0.f;
#pragma unroll
  for (int k = 0; k < kShares; ++k) total += share[k][lane];
  out[c] = accumulate ? out[c] + total : total;
}

template <int ACT>
cudaError_t launch_act(const Args& k, bool z8, dim3 grid, cudaStream_t s) {
  return launch_divided(kStreamingCarveout, z8 ? act_bwd_kernel<ACT, true> : act_bwd_kernel<ACT, false>, grid, dim3(kThreads), 0, s, k);
}

}  // namespace

int64_t act_bwd_workspace_floats(int64_t rows, int64_t cols) { return chunk_count(rows, cols) * cols; }

cudaError_t launch_column_sums(const float* partial, int64_t parts, int64_t cols, float* out, bool accumulate, cudaStream_t s) {
  const cudaError_t e = launch_divided(kStreamingCarveout, column_sums_kernel, dim3((unsigned)((cols + 31) / 32)),
                                       dim3(32 * kShares), 0, s, partial, parts, cols, out, (int)accumulate);
  count_launch();
  return e;
}

cudaError_t launch_act_bwd(const ActBwd& a, cudaStream_t s) {
  Args k{};
  k.da = static_cast<const uint16_t*>(a.da);
  k.z = static_cast<const uint16_t*>(a.z);
  if (a.z8) k.z8 = Copy8{a.z8->codes, a.z8->scales, blocks8(a.cols)};
  k.dz = static_cast<uint16_t*>(a.dz);
  k.a = static_cast<uint16_t*>(a.a);
  k.partial = a.dbias ? a.workspace : nullptr;
  k.rows = a.rows; k.cols = a.cols;
  k.ldda = a.ldda; k.ldz = a.ldz; k.lddz = a.lddz; k.lda = a.lda;
  k.chunk_rows = chunk_rows(a.rows, a.cols);
  const int64_t chunks = chunk_count(a.rows, a.cols);
  const dim3 grid((unsigned)((a.cols + kCols - 1) / kCols), (unsigned)chunks);
  const bool z8 = a.z8 != nullptr;
  cudaError_t e;
  switch (a.act) {
    case NVFP4_ACT_RELU2: e = launch_act<NVFP4_ACT_RELU2>(k, z8, grid, s); break;
    case NVFP4_ACT_SILU: e = launch_act<NVFP4_ACT_SILU>(k, z8, grid, s); break;
    case NVFP4_ACT_GELU: e = launch_act<NVFP4_ACT_GELU>(k, z8, grid, s); break;
    default: e = launch_act<NVFP4_ACT_NONE>(k, z8, grid, s); break;
  }
  count_launch();
  if (e != cudaSuccess || !a.dbias) return e;
  return launch_column_sums(a.workspace, chunks, a.cols, a.dbias, a.accumulate, s);
}

}  // namespace nvfp4

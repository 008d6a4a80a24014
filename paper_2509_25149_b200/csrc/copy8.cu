// Copies in 8 bits of a bf16 or binary32 tensor, and their values: what a layer keeps of an activation for its backward pass.
// Both kernels are bound by HBM: 2 (4) + 1 + 1/32 bytes per element one way, 1 + 1/32 + 2 the other.  A thread has chunks of
// eight neighbouring elements, kDepth of them in flight; four lanes share a block, whose maximum two shuffles find.  A row is
// padded to whole blocks in the count of chunks, so that a block never straddles a row's end.
#include "around.h"
#include "copy8.cuh"

namespace nvfp4 {

namespace {

constexpr int kThreads = 256, kDepth = 4;

// Walks a thread through chunks first, first + step, ... of rows of n chunks (coordinates move by additions)
struct Chunks {
  int64_t r, c, dr, dc, n;
  __device__ __forceinline__ Chunks(int64_t n_) : n(n_) {
    const int64_t first = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, step = (int64_t)gridDim.x * blockDim.x;
    r = first / n;
    c = first - r * n;
    dr = step / n;
    dc = step - dr * n;
  }
  __device__ __forceinline__ void next() {
    r += dr;
    c += dc;
    if (c >= n) {
      c -= n;
      ++r;
    }
  }
};

template <bool F32>
__global__ void __launch_bounds__(kThreads) quantize8_kernel(const void* x, int64_t rows, int64_t cols, int64_t ld, Copy8 q) {
  griddep_wait();
  griddep_launch_dependents();
  const int64_t n = q.blocks * 4, total = rows * n, step = (int64_t)gridDim.x * kThreads;
  Chunks w(n);
  // (turns are counted for the block: every lane takes part in the shuffles)
  for (int64_t done = (int64_t)blockIdx.x * kThreads; done < total; done += step * kDepth) {
    Raw8<F32> raw[kDepth];
    int64_t r[kDepth], c[kDepth];
    bool live[kDepth];
#pragma unroll
    for (int u = 0; u < kDepth; ++u) {
      r[u] = w.r;
      c[u] = w.c;
      live[u] = w.r < rows && w.c * 8 < cols;
      if (live[u])
        raw[u].load(x, w.r * ld + w.c * 8);
      else
        raw[u].zero();
      w.next();
    }
#pragma unroll
    for (int u = 0; u < kDepth; ++u) {
      float v[8];
      raw[u].values(v);
      store_chunk8(q, v, r[u], c[u], cols, live[u]);
    }
  }
}

template <bool F32>
__global__ void __launch_bounds__(kThreads) dequantize8_kernel(Copy8 q, int64_t rows, int64_t cols, void* out, int64_t ld) {
  griddep_wait();
  griddep_launch_dependents();
  const int64_t n = cols >> 3, total = rows * n, step = (int64_t)gridDim.x * kThreads;
  Chunks w(n);
  for (int64_t done = (int64_t)blockIdx.x * kThreads; done < total; done += step * kDepth) {
    uint2 codes[kDepth] = {};
    uint32_t byte[kDepth] = {};
    int64_t at[kDepth];
    bool live[kDepth];
#pragma unroll
    for (int u = 0; u < kDepth; ++u) {
      live[u] = w.r < rows;
      at[u] = w.r * ld + w.c * 8;
      if (live[u]) {
        codes[u] = ldg64_stream(q.codes + w.r * cols + w.c * 8);
        byte[u] = ldg8(q.scales + w.r * q.blocks + (w.c >> 2));
      }
      w.next();
    }
#pragma unroll
    for (int u = 0; u < kDepth; ++u) {
      float v[8];
      decode8(codes[u], decode_scale8(byte[u]), v);
      if (live[u]) store8<F32>(out, at[u], v);
    }
  }
}

cudaError_t grid_for(int64_t chunks, unsigned* grid) {
  int sms = 0;
  const cudaError_t e = sm_count(&sms);
  if (e != cudaSuccess) return e;
  const int64_t want = (chunks + kThreads * kDepth - 1) / (kThreads * kDepth), cap = (int64_t)sms * 32;
  *grid = (unsigned)(want < cap ? want : cap);
  return cudaSuccess;
}

}  // namespace

cudaError_t launch_quantize8(const void* x, bool fp32, int64_t rows, int64_t cols, int64_t ld, const nvfp4_tensor& q, cudaStream_t s) {
  const Copy8 c{q.codes, q.scales, blocks8(cols)};
  unsigned grid;
  cudaError_t e = grid_for(rows * c.blocks * 4, &grid);
  if (e != cudaSuccess) return e;
  e = launch_divided(kStreamingCarveout, fp32 ? quantize8_kernel<true> : quantize8_kernel<false>, dim3(grid), dim3(kThreads), 0, s, x,
                     rows, cols, ld, c);
  count_launch();
  return e;
}

cudaError_t launch_dequantize8(const nvfp4_tensor& q, void* out, bool out_fp32, int64_t ld, cudaStream_t s) {
  const Copy8 c{q.codes, q.scales, blocks8(q.cols)};
  unsigned grid;
  cudaError_t e = grid_for(q.rows * (q.cols >> 3), &grid);
  if (e != cudaSuccess) return e;
  e = launch_divided(kStreamingCarveout, out_fp32 ? dequantize8_kernel<true> : dequantize8_kernel<false>, dim3(grid), dim3(kThreads), 0,
                     s, c, q.rows, q.cols, out, ld);
  count_launch();
  return e;
}

}  // namespace nvfp4

// Copies in 8 bits of a bf16 or binary32 tensor, and their values: what a layer keeps of an activation for its backward pass.
// Both kernels are bound by HBM: 2 (4) + 1 + 1/32 bytes per element one way, 1 + 1/32 + 2 the other.  A thread has chunks of
// eight (sixteen) neighbouring elements, some of them in flight; four (two) lanes share a block, whose maximum shuffles find.  A row is
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

// Rows of whole 16 elements that begin on 32 bytes: chunks of sixteen, of which two lanes share a block (half the instructions per element:
// 8192 x 20480 89.4 -> 76.5 us, 8192 x 5120 27.1 -> 21.7, binary32 34.8 -> 32.3)
template <bool F32>
__global__ void __launch_bounds__(kThreads) quantize8_wide_kernel(const void* x, int64_t rows, int64_t cols, int64_t ld, Copy8 q) {
  griddep_wait();
  griddep_launch_dependents();
  constexpr int kDepthWide = 2;
  const int64_t n = q.blocks * 2, total = rows * n, step = (int64_t)gridDim.x * kThreads;
  Chunks w(n);
  for (int64_t done = (int64_t)blockIdx.x * kThreads; done < total; done += step * kDepthWide) {
    uint32_t raw[kDepthWide][F32 ? 16 : 8];
    int64_t r[kDepthWide], c[kDepthWide];
    bool live[kDepthWide];
#pragma unroll
    for (int u = 0; u < kDepthWide; ++u) {
      r[u] = w.r;
      c[u] = w.c;
      live[u] = w.r < rows && w.c * 16 < cols;
      if (live[u]) {
        const uint8_t* const src = static_cast<const uint8_t*>(x) + (w.r * ld + w.c * 16) * (F32 ? 4 : 2);
        ldg256_stream(src, *reinterpret_cast<uint32_t(*)[8]>(&raw[u][0]));
        if (F32) ldg256_stream(src + 32, *reinterpret_cast<uint32_t(*)[8]>(&raw[u][F32 ? 8 : 0]));
      } else {
#pragma unroll
        for (int k = 0; k < (F32 ? 16 : 8); ++k) raw[u][k] = 0u;
      }
      w.next();
    }
#pragma unroll
    for (int u = 0; u < kDepthWide; ++u) {
      float v[16];
#pragma unroll
      for (int k = 0; k < 16; ++k)
        v[k] = F32 ? __uint_as_float(raw[u][F32 ? k : 0]) : (k & 1) ? bf16_hi(raw[u][k >> 1]) : bf16_lo(raw[u][k >> 1]);
      float m;
      if (F32) {
        m = amax16_3(v);
      } else {
        uint32_t acc = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) acc = absmax_bf16x2(acc, raw[u][k]);
        m = amax_of_pair(acc);
      }
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
      const uint32_t byte = scale_byte8(m);
      const float scale = encode_scale8(byte);
      const uint2 lo = encode8(*reinterpret_cast<const float(*)[8]>(&v[0]), scale), hi = encode8(*reinterpret_cast<const float(*)[8]>(&v[8]), scale);
      if (!live[u]) continue;
      *reinterpret_cast<uint4*>(q.codes + r[u] * cols + c[u] * 16) = make_uint4(lo.x, lo.y, hi.x, hi.y);
      if ((c[u] & 1) == 0) q.scales[r[u] * q.blocks + (c[u] >> 1)] = (uint8_t)byte;
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

// The same the other way, into bf16, with stores of 32 bytes (8192 x 20480 83.3 -> 79.3 us; two of 16 bytes each 86.9)
__global__ void __launch_bounds__(kThreads) dequantize8_wide_kernel(Copy8 q, int64_t rows, int64_t cols, uint16_t* out, int64_t ld) {
  griddep_wait();
  griddep_launch_dependents();
  const int64_t n = cols >> 4, total = rows * n, step = (int64_t)gridDim.x * kThreads;
  Chunks w(n);
  for (int64_t done = (int64_t)blockIdx.x * kThreads; done < total; done += step * kDepth) {
    uint4 codes[kDepth] = {};
    uint32_t byte[kDepth] = {};
    int64_t at[kDepth];
    bool live[kDepth];
#pragma unroll
    for (int u = 0; u < kDepth; ++u) {
      live[u] = w.r < rows;
      at[u] = w.r * ld + w.c * 16;
      if (live[u]) {
        codes[u] = ldg128_stream(q.codes + w.r * cols + w.c * 16);
        byte[u] = ldg8(q.scales + w.r * q.blocks + (w.c >> 1));
      }
      w.next();
    }
#pragma unroll
    for (int u = 0; u < kDepth; ++u) {
      if (!live[u]) continue;
      float2 a[4], b[4];
      const float scale = decode_scale8(byte[u]);
      decode8(make_uint2(codes[u].x, codes[u].y), scale, a);
      decode8(make_uint2(codes[u].z, codes[u].w), scale, b);
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(out + at[u]), "r"(pack2(a[0].x, a[0].y)),
                   "r"(pack2(a[1].x, a[1].y)), "r"(pack2(a[2].x, a[2].y)), "r"(pack2(a[3].x, a[3].y)), "r"(pack2(b[0].x, b[0].y)),
                   "r"(pack2(b[1].x, b[1].y)), "r"(pack2(b[2].x, b[2].y)), "r"(pack2(b[3].x, b[3].y))
                   : "memory");
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
  if (cols % 16 == 0 && ld % 16 == 0 && aligned(x, 32)) {
    if ((e = grid_for(rows * c.blocks * 2, &grid)) != cudaSuccess) return e;
    e = launch_divided(kStreamingCarveout, fp32 ? quantize8_wide_kernel<true> : quantize8_wide_kernel<false>, dim3(grid), dim3(kThreads), 0, s,
                       x, rows, cols, ld, c);
  } else {
    e = launch_divided(kStreamingCarveout, fp32 ? quantize8_kernel<true> : quantize8_kernel<false>, dim3(grid), dim3(kThreads), 0, s, x,
                       rows, cols, ld, c);
  }
  count_launch();
  return e;
}

cudaError_t launch_dequantize8(const nvfp4_tensor& q, void* out, bool out_fp32, int64_t ld, cudaStream_t s) {
  const Copy8 c{q.codes, q.scales, blocks8(q.cols)};
  unsigned grid;
  cudaError_t e = grid_for(q.rows * (q.cols >> 3), &grid);
  if (e != cudaSuccess) return e;
  if (!out_fp32 && q.cols % 16 == 0 && ld % 16 == 0 && aligned(out, 32)) {
    if ((e = grid_for(q.rows * (q.cols >> 4), &grid)) != cudaSuccess) return e;
    e = launch_divided(kStreamingCarveout, dequantize8_wide_kernel, dim3(grid), dim3(kThreads), 0, s, c, q.rows, q.cols,
                       static_cast<uint16_t*>(out), ld);
    count_launch();
    return e;
  }
  e = launch_divided(kStreamingCarveout, out_fp32 ? dequantize8_kernel<true> : dequantize8_kernel<false>, dim3(grid), dim3(kThreads), 0,
                     s, c, q.rows, q.cols, out, ld);
  count_launch();
  return e;
}

}  // namespace nvfp4

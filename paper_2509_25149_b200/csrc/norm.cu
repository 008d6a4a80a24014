// Root-mean-square norm with the residual's addition, and its gradient.
//   forward   h = x + residual (one binary32 addition);  rstd = 1 / sqrt(mean(h^2) + eps);  y = h rstd gain
//   gradient  n = h rstd;  g = dy gain;  c = mean(g n);  dh = rstd (g - n c) + residual_grad;  dgain = sum over rows of dy n
// y and the copies in 8 bits are taken of the binary32 h, before it is rounded to the residual's type: y is as exact as it can be,
// and what the backward pass reads (the stored h) is off by that one rounding.
//
// Both are bound by HBM, so a row is read once: it stays in the registers of one to sixteen warps (up to five chunks of eight
// elements a lane) between the statistic and its use, and warps of a row exchange partial sums through shared memory.
#include "around.h"
#include "copy8.cuh"

namespace nvfp4 {

namespace {

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float dot8(const float (&a)[8], const float (&b)[8], float s) {
#pragma unroll
  for (int i = 0; i < 8; ++i) s = fmaf(a[i], b[i], s);
  return s;
}

struct Fwd {
  const uint16_t* x;
  const void* residual;
  const float* gain;
  void* h;
  uint16_t* y;
  float* rstd;
  Copy8 y8, h8;
  int64_t rows, cols, ldx, ldr, ldh, ldy;
  float eps;
};

__device__ __forceinline__ float rstd_of(float sum, int64_t cols, float eps) {
  return __frcp_rn(__fsqrt_rn(__fdiv_rn(sum, (float)cols) + eps));
}

// RES: 0 = no residual, 1 = bf16, 2 = binary32.  What follows the statistic, for one chunk.
template <int RES>
__device__ __forceinline__ void finish_chunk(const Fwd& a, const float (&v)[8], float rstd, int64_t row, int64_t chunk, bool live) {
  if (RES && a.h && live) store8<RES == 2>(a.h, row * a.ldh + chunk * 8, v);
  if (a.h8.codes) store_chunk8(a.h8, v, row, chunk, a.cols, live);
  if (!a.y && !a.y8.codes) return;
  float g[8], y[8] = {};
  if (live) {
    load_gain(a.gain, chunk * 8, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = v[i] * rstd * g[i];
    if (a.y) store8<false>(a.y, row * a.ldy + chunk * 8, y);
  }
  if (a.y8.codes) store_chunk8(a.y8, y, row, chunk, a.cols, live);
}

template <int RES>
struct Loaded {
  Raw8<false> x;
  Raw8<RES == 2> r;
  __device__ __forceinline__ void load(const Fwd& a, int64_t row, int64_t chunk, bool live) {
    if (live) {
      x.load(a.x, row * a.ldx + chunk * 8);
      if (RES) r.load(a.residual, row * a.ldr + chunk * 8);
    } else {
      x.zero();
      if (RES) r.zero();
    }
  }
  __device__ __forceinline__ void sum(float (&v)[8]) const {
    x.values(v);
    if (RES) {
      float w[8];
      r.values(w);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += w[i];
    }
  }
};

template <int WPR>
constexpr int kWarpsOf = WPR < 4 ? 4 : WPR;  // warps of a CTA

// WPR warps to a row, whose lanes take every WPR-th group of 32 chunks
template <int RES, int WPR, int KEEP>
__global__ void __launch_bounds__(32 * kWarpsOf<WPR>) rmsnorm_fwd_kernel(const Fwd a) {
  constexpr int kWarps = kWarpsOf<WPR>, kRows = kWarps / WPR;
  __shared__ float part[2][kWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, seg = warp % WPR, sub = warp / WPR;
  const int64_t n = a.cols >> 3;
  griddep_wait();
  griddep_launch_dependents();
  int it = 0;
  // every warp of a CTA takes the same number of turns, so the barrier and the shuffles are met by all
  for (int64_t base = (int64_t)blockIdx.x * kRows; base < a.rows; base += (int64_t)gridDim.x * kRows, ++it) {
    const int64_t row = base + sub;
    Loaded<RES> raw[KEEP];
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
      const int64_t chunk = lane + 32 * (seg + WPR * i);
      raw[i].load(a, row, chunk, row < a.rows && chunk < n);
    }
    float v[KEEP][8], sum = 0.f;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
      raw[i].sum(v[i]);
      sum = dot8(v[i], v[i], sum);
    }
    sum = warp_sum(sum);
    if (WPR > 1) {
      if (lane == 0) part[it & 1][warp] = sum;
      __syncthreads();
      sum = 0.f;
#pragma unroll
      for (int w = 0; w < WPR; ++w) sum += part[it & 1][sub * WPR + w];
    }
    const float rstd = rstd_of(sum, a.cols, a.eps);
    if (a.rstd && seg == 0 && lane == 0 && row < a.rows) a.rstd[row] = rstd;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
      const int64_t chunk = lane + 32 * (seg + WPR * i);
      finish_chunk<RES>(a, v[i], rstd, row, chunk, row < a.rows && chunk < n);
    }
  }
}

// Longer rows: a CTA to a row, which is read twice (the second time from L2)
template <int RES>
__global__ void __launch_bounds__(512) rmsnorm_fwd_long_kernel(const Fwd a) {
  __shared__ float part[2][16];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t n = a.cols >> 3;
  griddep_wait();
  griddep_launch_dependents();
  int it = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, ++it) {
    float sum = 0.f;
    for (int64_t c0 = 0; c0 < n; c0 += 2048) {
      Loaded<RES> raw[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) raw[i].load(a, row, c0 + threadIdx.x + 512 * i, c0 + threadIdx.x + 512 * i < n);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v[8];
        raw[i].sum(v);
        sum = dot8(v, v, sum);
      }
    }
    sum = warp_sum(sum);
    if (lane == 0) part[it & 1][warp] = sum;
    __syncthreads();
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < 16; ++w) sum += part[it & 1][w];
    const float rstd = rstd_of(sum, a.cols, a.eps);
    if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
    for (int64_t c0 = 0; c0 < n; c0 += 1024) {
      Loaded<RES> raw[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) raw[i].load(a, row, c0 + threadIdx.x + 512 * i, c0 + threadIdx.x + 512 * i < n);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int64_t chunk = c0 + threadIdx.x + 512 * i;
        float v[8];
        raw[i].sum(v);
        finish_chunk<RES>(a, v, rstd, row, chunk, chunk < n);
      }
    }
  }
}

template <int RES, int WPR, int KEEP>
cudaError_t launch_fwd_kept(const Fwd& a, int sms, cudaStream_t s) {
  constexpr int kWarps = kWarpsOf<WPR>, kRows = kWarps / WPR;
  const int64_t want = (a.rows + kRows - 1) / kRows, cap = (int64_t)sms * (64 / kWarps) * 4;
  return launch_divided(kStreamingCarveout, rmsnorm_fwd_kernel<RES, WPR, KEEP>, dim3((unsigned)(want < cap ? want : cap)),
                        dim3(32 * kWarps), 0, s, a);
}

template <int RES>
cudaError_t launch_fwd(const Fwd& a, int sms, cudaStream_t s) {
  const int64_t groups = ((a.cols >> 3) + 31) / 32;  // of 32 chunks
  if (groups <= 2) return launch_fwd_kept<RES, 1, 2>(a, sms, s);
  if (groups <= 4) return launch_fwd_kept<RES, 2, 2>(a, sms, s);
  if (groups <= 8) return launch_fwd_kept<RES, 4, 2>(a, sms, s);
  if (groups <= 20) return launch_fwd_kept<RES, 4, 5>(a, sms, s);
  if (groups <= 40) return launch_fwd_kept<RES, 8, 5>(a, sms, s);
  if (groups <= 80) return launch_fwd_kept<RES, 16, 5>(a, sms, s);
  const int64_t cap = (int64_t)sms * 4;
  return launch_divided(kStreamingCarveout, rmsnorm_fwd_long_kernel<RES>, dim3((unsigned)(a.rows < cap ? a.rows : cap)), dim3(512), 0, s, a);
}

// ------------------------------------------------------------------------------------------------ gradient ----
struct Bwd {
  const uint16_t* dy;
  const void* h;
  Copy8 h8;
  const float* gain;
  const float* rstd;
  const void* residual_grad;
  void* dh;
  float* partial;  // a row of column sums per CTA (NULL: dgain is not wanted)
  float* dots;     // rows too long for registers: c of every row
  int64_t rows, cols, lddy, ldh, ldrg, lddh, chunk_rows;
};

// H: 0 = bf16, 1 = binary32, 2 = copy in 8 bits
template <int H>
struct LoadedH {
  Raw8<H == 1> raw;
  uint2 codes;
  uint32_t byte;
  __device__ __forceinline__ void load(const Bwd& a, int64_t row, int64_t chunk) {
    if (H == 2) {
      codes = ldg64_stream(a.h8.codes + row * a.cols + chunk * 8);
      byte = ldg8(a.h8.scales + row * a.h8.blocks + (chunk >> 2));
    } else {
      raw.load(a.h, row * a.ldh + chunk * 8);
    }
  }
  __device__ __forceinline__ void zero() {
    if (H == 2) {
      codes = make_uint2(0u, 0u);
      byte = 0u;
    } else {
      raw.zero();
    }
  }
  __device__ __forceinline__ void normalised(float rstd, float (&n)[8]) const {
    if (H == 2) {
      decode8(codes, decode_scale8(byte), n);
    } else {
      raw.values(n);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) n[i] *= rstd;
  }
};

__device__ __forceinline__ void times_gain(const Bwd& a, int64_t chunk, const float (&d)[8], float (&g)[8]) {
  load_gain(a.gain, chunk * 8, g);
#pragma unroll
  for (int i = 0; i < 8; ++i) g[i] *= d[i];
}

template <bool F32>
__device__ __forceinline__ void store_dh(const Bwd& a, const float (&g)[8], const float (&n)[8], const Raw8<F32>& rg, float rstd,
                                         float c, int64_t row, int64_t chunk) {
  float out[8], w[8];
  rg.values(w);
#pragma unroll
  for (int i = 0; i < 8; ++i) out[i] = fmaf(rstd, fmaf(-n[i], c, g[i]), w[i]);
  store8<F32>(a.dh, row * a.lddh + chunk * 8, out);
}

constexpr int kBwdWarps = 16;

// A CTA of sixteen warps, WPR of them to a row: 16 / WPR rows at a time, each group of warps at its own pace.  A lane keeps the sums
// of its columns in registers over all its rows; at the end the groups add theirs in their order.
template <int H, bool F32, int WPR, int KEEP>
__global__ void __launch_bounds__(32 * kBwdWarps, 1) rmsnorm_bwd_kernel(const Bwd a) {
  constexpr int kGroups = kBwdWarps / WPR;
  extern __shared__ float columns[];  // (more than one group) cols sums
  __shared__ float part[2][kBwdWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, seg = warp % WPR, group = warp / WPR;
  const int64_t n8 = a.cols >> 3;
  griddep_wait();
  griddep_launch_dependents();
  float acc[KEEP][8] = {};
  int it = 0;
  for (int64_t row = (int64_t)blockIdx.x * kGroups + group; row < a.rows; row += (int64_t)gridDim.x * kGroups, ++it) {
    Raw8<false> dy[KEEP];
    LoadedH<H> h[KEEP];
    Raw8<F32> rg[KEEP];
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
      const int64_t chunk = lane + 32 * (seg + WPR * i);
      rg[i].zero();
      if (chunk < n8) {
        dy[i].load(a.dy, row * a.lddy + chunk * 8);
        h[i].load(a, row, chunk);
        if (a.residual_grad) rg[i].load(a.residual_grad, row * a.ldrg + chunk * 8);
      } else {
        dy[i].zero();
        h[i].zero();
      }
    }
    const float rstd = a.rstd[row];
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
      const int64_t chunk = lane + 32 * (seg + WPR * i);
      if (chunk >= n8) continue;
      float d[8], n[8], g[8];
      dy[i].values(d);
      h[i].normalised(rstd, n);
      times_gain(a, chunk, d, g);
      sum = dot8(g, n, sum);
#pragma unroll
      for (int k = 0; k < 8; ++k) acc[i][k] = fmaf(d[k], n[k], acc[i][k]);
    }
    sum = warp_sum(sum);
    if (WPR > 1) {
      if (lane == 0) part[it & 1][warp] = sum;
      asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(32 * WPR) : "memory");
      sum = 0.f;
#pragma unroll
      for (int w = 0; w < WPR; ++w) sum += part[it & 1][group * WPR + w];
    }
    const float c = __fdiv_rn(sum, (float)a.cols);
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
      const int64_t chunk = lane + 32 * (seg + WPR * i);
      if (chunk >= n8) continue;
      float d[8], n[8], g[8];
      dy[i].values(d);
      h[i].normalised(rstd, n);
      times_gain(a, chunk, d, g);
      store_dh<F32>(a, g, n, rg[i], rstd, c, row, chunk);
    }
  }
  if (!a.partial) return;
  float* const out = a.partial + (int64_t)blockIdx.x * a.cols;
  for (int g = 0; g < kGroups; ++g) {
    if (g == group) {
#pragma unroll
      for (int i = 0; i < KEEP; ++i) {
        const int64_t chunk = lane + 32 * (seg + WPR * i);
        if (chunk >= n8) continue;
        if (g > 0) {
          const float4* const p = reinterpret_cast<const float4*>(columns + chunk * 8);
          const float4 u = p[0], v = p[1];
          acc[i][0] += u.x; acc[i][1] += u.y; acc[i][2] += u.z; acc[i][3] += u.w;
          acc[i][4] += v.x; acc[i][5] += v.y; acc[i][6] += v.z; acc[i][7] += v.w;
        }
        store8<true>(g == kGroups - 1 ? out : columns, chunk * 8, acc[i]);
      }
    }
    if (g < kGroups - 1) __syncthreads();
  }
}

// Rows too long for registers: c of every row, a CTA to a row
template <int H>
__global__ void __launch_bounds__(512) rmsnorm_dots_kernel(const Bwd a) {
  __shared__ float part[2][16];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t n8 = a.cols >> 3;
  griddep_wait();
  griddep_launch_dependents();
  int it = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, ++it) {
    const float rstd = a.rstd[row];
    float sum = 0.f;
    for (int64_t c0 = 0; c0 < n8; c0 += 1024) {
      Raw8<false> dy[2];
      LoadedH<H> h[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int64_t chunk = c0 + threadIdx.x + 512 * i;
        if (chunk < n8) {
          dy[i].load(a.dy, row * a.lddy + chunk * 8);
          h[i].load(a, row, chunk);
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int64_t chunk = c0 + threadIdx.x + 512 * i;
        if (chunk >= n8) continue;
        float d[8], n[8], g[8];
        dy[i].values(d);
        h[i].normalised(rstd, n);
        times_gain(a, chunk, d, g);
        sum = dot8(g, n, sum);
      }
    }
    sum = warp_sum(sum);
    if (lane == 0) part[it & 1][warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
      sum = 0.f;
      for (int w = 0; w < 16; ++w) sum += part[it & 1][w];
      a.dots[row] = __fdiv_rn(sum, (float)a.cols);
    }
  }
}
// ... and dh with the column sums: 256 columns and a run of rows to a CTA of eight warps, eight columns to a lane
template <int H, bool F32>
__global__ void __launch_bounds__(256) rmsnorm_bwd_long_kernel(const Bwd a) {
  __shared__ float part[8][256];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t chunk = (int64_t)blockIdx.x * 32 + lane;
  const bool live = chunk < (a.cols >> 3);
  const int64_t r0 = (int64_t)blockIdx.y * a.chunk_rows, r1 = min(r0 + a.chunk_rows, a.rows);
  griddep_wait();
  griddep_launch_dependents();
  float acc[8] = {};
  for (int64_t r = r0 + warp; live && r < r1; r += 16) {
    Raw8<false> dy[2];
    LoadedH<H> h[2];
    Raw8<F32> rg[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int64_t row = r + 8 * u;
      if (row >= r1) break;
      dy[u].load(a.dy, row * a.lddy + chunk * 8);
      h[u].load(a, row, chunk);
      rg[u].zero();
      if (a.residual_grad) rg[u].load(a.residual_grad, row * a.ldrg + chunk * 8);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int64_t row = r + 8 * u;
      if (row >= r1) break;
      const float rstd = a.rstd[row], c = a.dots[row];
      float d[8], n[8], g[8];
      dy[u].values(d);
      h[u].normalised(rstd, n);
      times_gain(a, chunk, d, g);
#pragma unroll
      for (int k = 0; k < 8; ++k) acc[k] = fmaf(d[k], n[k], acc[k]);
      store_dh<F32>(a, g, n, rg[u], rstd, c, row, chunk);
    }
  }
  if (!a.partial) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) part[warp][lane * 8 + i] = acc[i];
  __syncthreads();
  const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (c >= a.cols) return;
  float total = 0.f;
#pragma unroll
  for (int w = 0; w < 8; ++w) total += part[w][threadIdx.x];
  a.partial[(int64_t)blockIdx.y * a.cols + c] = total;
}

constexpr int64_t kKeptCols = 20480;  // 16 warps x 5 chunks x 32 lanes x 8 elements
constexpr int kMaxParts = 256;        // CTAs that leave column sums (one per SM, and no GPU of this kind has more)

int warps_per_row(int64_t cols) {
  const int64_t groups = ((cols >> 3) + 31) / 32;
  return groups <= 2 ? 1 : groups <= 4 ? 2 : groups <= 20 ? 4 : groups <= 40 ? 8 : 16;
}

template <int H, bool F32, int WPR, int KEEP>
cudaError_t launch_bwd_kept(const Bwd& k, const NormBwd& a, int sms, cudaStream_t s) {
  constexpr int kGroups = kBwdWarps / WPR;
  const int64_t want = (a.rows + kGroups - 1) / kGroups, cap = sms < kMaxParts ? sms : kMaxParts;
  const int64_t grid = want < cap ? want : cap;
  const size_t smem = kGroups > 1 ? (size_t)a.cols * 4 : 0;
  const cudaError_t e = launch_divided(20, rmsnorm_bwd_kernel<H, F32, WPR, KEEP>, dim3((unsigned)grid), dim3(32 * kBwdWarps), smem, s, k);
  count_launch();
  if (e != cudaSuccess || !a.dgain) return e;
  return launch_column_sums(k.partial, grid, a.cols, a.dgain, a.accumulate, s);
}

template <int H, bool F32>
cudaError_t launch_bwd(const Bwd& k, const NormBwd& a, int sms, cudaStream_t s) {
  if (a.cols <= kKeptCols) {
    const int64_t groups = ((a.cols >> 3) + 31) / 32;
    switch (warps_per_row(a.cols)) {
      case 1: return launch_bwd_kept<H, F32, 1, 2>(k, a, sms, s);
      case 2: return launch_bwd_kept<H, F32, 2, 2>(k, a, sms, s);
      case 4: return groups <= 8 ? launch_bwd_kept<H, F32, 4, 2>(k, a, sms, s) : launch_bwd_kept<H, F32, 4, 5>(k, a, sms, s);
      case 8: return launch_bwd_kept<H, F32, 8, 5>(k, a, sms, s);
      default: return launch_bwd_kept<H, F32, 16, 5>(k, a, sms, s);
    }
  }
  const int64_t cap = (int64_t)sms * 4, chunks = (a.rows + k.chunk_rows - 1) / k.chunk_rows;
  cudaError_t e = launch_divided(kStreamingCarveout, rmsnorm_dots_kernel<H>, dim3((unsigned)(a.rows < cap ? a.rows : cap)), dim3(512), 0, s, k);
  count_launch();
  if (e != cudaSuccess) return e;
  e = launch_divided(kStreamingCarveout, rmsnorm_bwd_long_kernel<H, F32>, dim3((unsigned)((a.cols + 255) / 256), (unsigned)chunks), dim3(256), 0,
                     s, k);
  count_launch();
  if (e != cudaSuccess || !a.dgain) return e;
  return launch_column_sums(k.partial, chunks, a.cols, a.dgain, a.accumulate, s);
}

// Rows of a CTA of the long form: 128, or more where there would be more chunks than a grid's second dimension takes
int64_t long_rows(int64_t rows) {
  const int64_t n = (rows + 32767) / 32768;
  return n < 128 ? 128 : (n + 15) / 16 * 16;
}
int64_t dots_floats(int64_t rows) { return (rows + 63) / 64 * 64; }

}  // namespace

bool rmsnorm_bwd_needs_workspace(int64_t cols) { return cols > kKeptCols; }
int64_t rmsnorm_bwd_workspace_floats(int64_t rows, int64_t cols) {
  if (cols > kKeptCols) return dots_floats(rows) + (rows + long_rows(rows) - 1) / long_rows(rows) * cols;
  const int64_t groups = kBwdWarps / warps_per_row(cols), parts = (rows + groups - 1) / groups;
  return (parts < kMaxParts ? parts : kMaxParts) * cols;
}

cudaError_t launch_rmsnorm_fwd(const NormFwd& a, cudaStream_t s) {
  Fwd k{};
  k.x = static_cast<const uint16_t*>(a.x);
  k.residual = a.residual;
  k.gain = a.gain;
  k.h = a.h;
  k.y = static_cast<uint16_t*>(a.y);
  k.rstd = a.rstd;
  if (a.y8) k.y8 = Copy8{a.y8->codes, a.y8->scales, blocks8(a.cols)};
  if (a.h8) k.h8 = Copy8{a.h8->codes, a.h8->scales, blocks8(a.cols)};
  k.rows = a.rows; k.cols = a.cols;
  k.ldx = a.ldx; k.ldr = a.ldr; k.ldh = a.ldh; k.ldy = a.ldy;
  k.eps = a.eps;
  int sms = 0;
  cudaError_t e = sm_count(&sms);
  if (e != cudaSuccess) return e;
  e = !a.residual ? launch_fwd<0>(k, sms, s) : a.fp32 ? launch_fwd<2>(k, sms, s) : launch_fwd<1>(k, sms, s);
  count_launch();
  return e;
}

cudaError_t launch_rmsnorm_bwd(const NormBwd& a, cudaStream_t s) {
  Bwd k{};
  k.dy = static_cast<const uint16_t*>(a.dy);
  k.h = a.h;
  if (a.h8) k.h8 = Copy8{a.h8->codes, a.h8->scales, blocks8(a.cols)};
  k.gain = a.gain;
  k.rstd = a.rstd;
  k.residual_grad = a.residual_grad;
  k.dh = a.dh;
  k.rows = a.rows; k.cols = a.cols;
  k.lddy = a.lddy; k.ldh = a.ldh; k.ldrg = a.ldrg; k.lddh = a.lddh;
  float* partial = a.workspace;
  if (a.cols > kKeptCols) {
    k.dots = a.workspace;
    k.chunk_rows = long_rows(a.rows);
    partial += dots_floats(a.rows);
  }
  k.partial = a.dgain ? partial : nullptr;
  int sms = 0;
  const cudaError_t e = sm_count(&sms);
  if (e != cudaSuccess) return e;
  if (a.h8) return a.dh_fp32 ? launch_bwd<2, true>(k, a, sms, s) : launch_bwd<2, false>(k, a, sms, s);
  if (a.h_fp32) return a.dh_fp32 ? launch_bwd<1, true>(k, a, sms, s) : launch_bwd<1, false>(k, a, sms, s);
  return a.dh_fp32 ? launch_bwd<0, true>(k, a, sms, s) : launch_bwd<0, false>(k, a, sms, s);
}

}  // namespace nvfp4

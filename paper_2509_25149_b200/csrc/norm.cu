// Root-mean-square norm with the residual's addition, and its gradient.
//   forward   h = x + residual (one binary32 addition);  rstd = 1 / sqrt(mean(h^2) + eps);  y = h rstd gain
//   gradient  n = h rstd;  g = dy gain;  c = mean(g n);  dh = rstd (g - n c) + residual_grad;  dgain = sum over rows of dy n
// y and the copies in 8 bits are taken of the binary32 h, before it is rounded to the residual's type: y is as exact as it can be,
// and what the backward pass reads (the stored h) is off by that one rounding.
//
// Both are bound by HBM, so a row is read once: it stays on the SM (forward: in the registers, gradient: in shared memory) of one to
// sixteen warps, up to five chunks of eight elements a lane, between the statistic and its use, and warps of a row exchange partial sums
// through shared memory.  Of the measured copy rate: forward of 8192 x 5120 with a bf16 residual 54.5 us (94 %), gradient from bf16 57.6 us
// (89 %), from 8 bits 50.9 us (89 %), from and to binary32 115 us (78 %).
#include "around.h"
#include "copy8.cuh"

namespace nvfp4 {

namespace {

template <class T>
__device__ __forceinline__ T warp_sum(T v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
template <int N>
__device__ __forceinline__ double sum_of(const double* part) {
  double s[4] = {};
#pragma unroll
  for (int w = 0; w < N; ++w) s[w & 3] += part[w];
  return (s[0] + s[1]) + (s[2] + s[3]);
}
// Sums of squares of a lane, eight apart: short chains of additions round less, and do not wait for one another
struct Squares {
  float2 s[4] = {};
  __device__ __forceinline__ void add(const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 p = make_float2(v[2 * i], v[2 * i + 1]);
      s[i] = fma2(p, p, s[i]);
    }
  }
  __device__ __forceinline__ void add(const float (&v)[8], float scale) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 p = mul2(make_float2(v[2 * i], v[2 * i + 1]), both(scale));
      s[i] = fma2(p, p, s[i]);
    }
  }
  __device__ __forceinline__ float sum() const {
    const float2 t = add2(add2(s[0], s[1]), add2(s[2], s[3]));
    return t.x + t.y;
  }
};
// Finite values of 1e17 and more have squares, or sums of them, that binary32 does not hold: a lane that lost its sum takes it of its values
// times 2^-70 once more.  (Some value is above 2^50 then, and what vanishes beside it in 24 bits may vanish here.)  The question costs all rows up to
// 2 %: 8192 x 5120 from binary32 81.3 -> 82.9 us, from bf16 54.7 / 54.6, 8192 x 2056 without a residual 17.8 -> 18.2.
__device__ __forceinline__ bool lost(float sum) { return __builtin_expect(!(sum <= 3.402823466e38f), 0); }

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

// 1 / sqrt(mean + eps) as the sum of two floats: a value in binary32, e off by some 2^-23 of itself, and one step of Newton's method in 64 bits,
// which leaves 1.5 e^2.  The copy of y in 8 bits wants it: of its codes those come out a step off whose y crosses a border by its error, and with
// the root and both products rounded to 24 bits they were twice as many.  (8192 x 5120 with the copy 61.3 -> 61.8 us, 16384 x 256 8.7 -> 7.8, 2048 x 20480 64.6 ->
// 67.0: mean and root in binary32 took divisions and roots of their own.)
struct Rstd {
  float hi, lo;
};
__device__ __forceinline__ Rstd rstd_of(double sum, double per_col, float eps) {
  const double m = fma(sum, per_col, (double)eps);
  double y = (double)rsqrtf((float)m);
  if (y == 0.) y = (double)rsqrtf((float)(m * 0x1p-160)) * 0x1p-80;  // (m is beyond binary32, and below 2^256)
  const double r = y > 0. ? fma(0.5 * y, fma(-m * y, y, 1.), y) : y;
  const float hi = (float)r;
  return {hi, (float)(r - (double)hi)};
}

// RES: 0 = no residual, 1 = bf16, 2 = binary32.  What follows the statistic, for one chunk.
template <int RES>
__device__ __forceinline__ void finish_chunk(const Fwd& a, const float (&v)[8], const Rstd& rstd, int64_t row, int64_t chunk, bool live) {
  if (RES && a.h && live) store8<RES == 2>(a.h, row * a.ldh + chunk * 8, v);
  if (a.h8.codes) store_chunk8(a.h8, v, row, chunk, a.cols, live);
  if (!a.y && !a.y8.codes) return;
  float g[8], y[8] = {};
  if (live) {
    load_gain(a.gain, chunk * 8, g);
#pragma unroll
    for (int i = 0; i < 8; i += 2) {  // v (hi + lo) g, rounded once
      const float2 w = make_float2(v[i], v[i + 1]), gain = make_float2(g[i], g[i + 1]), n = mul2(w, both(rstd.hi));
      const float2 off = fma2(w, both(rstd.lo), fma2(w, both(rstd.hi), make_float2(-n.x, -n.y)));
      const float2 t = fma2(n, gain, mul2(off, gain));
      y[i] = t.x;
      y[i + 1] = t.y;
    }
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
// (64 registers hold a row's values but for binary32 residuals of the longest rows; one more costs an eighth of the warps)
template <int RES, int WPR, int KEEP>
__global__ void __launch_bounds__(32 * kWarpsOf<WPR>, RES == 2 && WPR > 4 ? 1 : 32 / kWarpsOf<WPR>) rmsnorm_fwd_kernel(const Fwd a) {
  constexpr int kWarps = kWarpsOf<WPR>, kRows = kWarps / WPR;
  __shared__ double part[2][kWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, seg = warp % WPR, sub = warp / WPR;
  const int64_t n = a.cols >> 3;
  const double per_col = 1. / (double)a.cols;
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
    float v[KEEP][8];
    Squares squares;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
      raw[i].sum(v[i]);
      squares.add(v[i]);
    }
    double sum = squares.sum();
    if (lost(squares.sum())) {
      Squares scaled;
#pragma unroll
      for (int i = 0; i < KEEP; ++i) scaled.add(v[i], 0x1p-70f);
      sum = scaled.sum() * 0x1p140;
    }
    sum = warp_sum(sum);
    if (WPR > 1) {
      if (lane == 0) part[it & 1][warp] = sum;
      __syncthreads();
      sum = sum_of<WPR>(part[it & 1] + sub * WPR);
    }
    const Rstd rstd = rstd_of(sum, per_col, a.eps);
    if (a.rstd && seg == 0 && lane == 0 && row < a.rows) a.rstd[row] = rstd.hi;
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
  __shared__ double part[2][16];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t n = a.cols >> 3;
  const double per_col = 1. / (double)a.cols;
  griddep_wait();
  griddep_launch_dependents();
  int it = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, ++it) {
    Squares squares;
    for (int64_t c0 = 0; c0 < n; c0 += 2048) {
      Loaded<RES> raw[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) raw[i].load(a, row, c0 + threadIdx.x + 512 * i, c0 + threadIdx.x + 512 * i < n);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v[8];
        raw[i].sum(v);
        squares.add(v);
      }
    }
    double sum = squares.sum();
    if (lost(squares.sum())) {
      Squares scaled;
#pragma unroll 1
      for (int64_t c = threadIdx.x; c < n; c += 512) {
        Loaded<RES> raw;
        float v[8];
        raw.load(a, row, c, true);
        raw.sum(v);
        scaled.add(v, 0x1p-70f);
      }
      sum = scaled.sum() * 0x1p140;
    }
    sum = warp_sum(sum);
    if (lane == 0) part[it & 1][warp] = sum;
    __syncthreads();
    sum = sum_of<16>(part[it & 1]);
    const Rstd rstd = rstd_of(sum, per_col, a.eps);
    if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd.hi;
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
  if (groups <= 12) return launch_fwd_kept<RES, 4, 3>(a, sms, s);
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
  __device__ __forceinline__ void normalised(float rstd, float2 (&n)[4]) const {
    if (H == 2) {
      // The scale is a power of two, so 2^E rstd is exact and the product rounded once, as the value times rstd is.  (Below 2^-126, where 2^E
      // rstd is cut to a multiple of 2^-149, n is below 2^-117.)
      decode8(codes, decode_scale8(byte) * rstd, n);
      return;
    }
    values2(raw, n);
#pragma unroll
    for (int i = 0; i < 4; ++i) n[i] = mul2(n[i], both(rstd));
  }
};

__device__ __forceinline__ void times_gain(const float* gain, int64_t chunk, const float2 (&d)[4], float2 (&g)[4]) {
  float v[8];
  load_gain(gain, chunk * 8, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) g[i] = mul2(d[i], make_float2(v[2 * i], v[2 * i + 1]));
}

template <bool F32>
__device__ __forceinline__ void store_dh(const Bwd& a, const float2 (&g)[4], const float2 (&n)[4], const Raw8<F32>& rg, float rstd,
                                         float c, int64_t row, int64_t chunk) {
  float2 out[4], w[4];
  values2(rg, w);
#pragma unroll
  for (int i = 0; i < 4; ++i) out[i] = fma2(both(rstd), fma2(n[i], both(-c), g[i]), w[i]);
  store8<F32>(a.dh, row * a.lddh + chunk * 8, out);
}

// A CTA of G groups of WPR warps, a row to a group at a time, each group at its own pace.  dy and h of the rows to come are on
// their way into a ring of ST rows in shared memory, in which every thread has places of its own (so that no group waits for another,
// and a thread only for its own copies); so is the residual path's gradient where there is room, else it is loaded when its row's turn
// begins.
// A lane keeps the sums of its columns in registers over all its rows; at the end those of the groups are added in their order.
template <int H, bool F32, int WPR, int KEEP>
struct BwdShape {
  static constexpr int kH = H == 2 ? 8 : H == 1 ? 32 : 16;  // bytes of a chunk of h
  // sixteen warps (a register file of 128 per thread), eight where five chunks of a binary32 h would not leave the ring two rows
  static constexpr int kGroups = WPR == 16 ? 1 : (H == 1 && KEEP == 5 ? 8 : 16) / WPR;
  static_assert(WPR == 1 || kGroups < 16, "named barriers 1 .. 15");
  static constexpr int kThreads = 32 * WPR * kGroups;
  static constexpr int kGain = 32 * WPR * KEEP * 32;  // the gain of all columns
  static constexpr int fit(int chunk_bytes) { return (220 * 1024 - kGain) / (KEEP * chunk_bytes * kThreads); }
  // the residual path's gradient goes through the ring as well where two rows of all three fit
  static constexpr bool kRingRg = fit(16 + kH + (F32 ? 32 : 16)) >= 2;
  static constexpr int kRg = kRingRg ? (F32 ? 32 : 16) : 0;
  static constexpr int kStage = KEEP * (16 + kH + kRg) * kThreads;
  static constexpr int ST = fit(16 + kH + kRg) > 4 ? 4 : fit(16 + kH + kRg);
  static constexpr int kBytes = ST * kStage + kGain;
  static_assert(ST >= 1 && kGroups * 32 * WPR * KEEP * 32 <= ST * kStage, "the column sums reuse the ring");
};

template <int H, bool F32, int WPR, int KEEP>
__global__ void __launch_bounds__(BwdShape<H, F32, WPR, KEEP>::kThreads, 1) rmsnorm_bwd_kernel(const Bwd a) {
  using S = BwdShape<H, F32, WPR, KEEP>;
  constexpr int ST = S::ST, kGroups = S::kGroups, T = S::kThreads;
  extern __shared__ __align__(16) uint8_t smem[];
  float* const columns = reinterpret_cast<float*>(smem);
  float4* const gain_s = reinterpret_cast<float4*>(smem + ST * S::kStage);  // [half of a chunk][chunk]
  __shared__ float part[2][WPR * kGroups];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, seg = warp % WPR, group = warp / WPR;
  const int n8 = (int)(a.cols >> 3);
  const uint32_t ring = smem_u32(smem), mine_dy = ring + threadIdx.x * 16,
                 mine_rg = ring + KEEP * T * 16 + threadIdx.x * 16,
                 mine_h = ring + KEEP * T * (16 + S::kRg) + threadIdx.x * (H == 2 ? 8 : 16);
  const int c0 = lane + 32 * seg;  // the lane's first chunk; the others are 32 * WPR apart
  auto chunk_of = [&](int i) { return c0 + 32 * WPR * i; };
  const int64_t step = (int64_t)gridDim.x * kGroups;
  auto fetch = [&](int64_t row, int slot) {
    if (row < a.rows) {
      const uint16_t* const dy = a.dy + row * a.lddy + c0 * 8;
      const uint8_t* const h = H == 2 ? a.h8.codes + row * a.cols + c0 * 8
                                      : static_cast<const uint8_t*>(a.h) + (row * a.ldh + c0 * 8) * (H == 1 ? 4 : 2);
      const uint8_t* const rg = static_cast<const uint8_t*>(a.residual_grad) + (row * a.ldrg + c0 * 8) * (F32 ? 4 : 2);
#pragma unroll
      for (int i = 0; i < KEEP; ++i) {
        if (chunk_of(i) >= n8) break;
        if (S::kRingRg && a.residual_grad) {
          const uint32_t dst = mine_rg + slot * S::kStage + i * T * S::kRg;
          copy_async<16>(dst, rg + i * (F32 ? 1024 : 512) * WPR, true);
          if (F32) copy_async<16>(dst + T * 16, rg + i * 1024 * WPR + 16, true);
        }
        copy_async<16>(mine_dy + slot * S::kStage + i * T * 16, dy + i * 256 * WPR, true);
        const uint32_t dst = mine_h + slot * S::kStage + i * T * S::kH;
        if (H == 2) {
          copy_async<8>(dst, h + i * 256 * WPR, true);
        } else if (H == 1) {
          copy_async<16>(dst, h + i * 1024 * WPR, true);
          copy_async<16>(dst + T * 16, h + i * 1024 * WPR + 16, true);
        } else {
          copy_async<16>(dst, h + i * 512 * WPR, true);
        }
      }
    }
    copy_commit();  // (an empty group where there is no row: the count of groups stays that of the rows)
  };
  // what a copy cannot bring one by one: the scale bytes and rstd of the next row
  uint32_t byte[KEEP] = {};
  float rstd_next = 0.f;
  auto fetch_small = [&](int64_t row) {
    if (row >= a.rows) return;
    rstd_next = a.rstd[row];
    if (H == 2)
#pragma unroll
      for (int i = 0; i < KEEP; ++i)
        if (chunk_of(i) < n8) byte[i] = ldg8(a.h8.scales + row * a.h8.blocks + (chunk_of(i) >> 2));
  };
  const float per_col = __frcp_rn((float)a.cols);  // (rounded twice instead of once: 2^-24 of c)
  const int64_t first = (int64_t)blockIdx.x + (int64_t)gridDim.x * group;
  griddep_wait();
#pragma unroll
  for (int u = 0; u < ST - 1; ++u) fetch(first + u * step, u);
  fetch_small(first);
  for (int c = threadIdx.x; c < n8; c += T) {
    float g[8];
    load_gain(a.gain, (int64_t)c * 8, g);
    gain_s[c] = make_float4(g[0], g[1], g[2], g[3]);
    gain_s[32 * WPR * KEEP + c] = make_float4(g[4], g[5], g[6], g[7]);
  }
  __syncthreads();
  griddep_launch_dependents();
  float2 acc[KEEP][4] = {};
  int it = 0, slot = 0, next = ST - 1;
  for (int64_t row = first; row < a.rows; row += step, ++it) {
    Raw8<F32> rg[KEEP];
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
      if (!S::kRingRg && a.residual_grad && chunk_of(i) < n8)
        rg[i].load(a.residual_grad, row * a.ldrg + chunk_of(i) * 8);
      else
        rg[i].zero();
    }
    if (ST == 1) fetch(row, 0);  // (no room for a row ahead)
    copy_wait<(ST > 2 ? ST - 2 : 0)>();
    const float rstd = rstd_next;
    uint32_t scale[KEEP];
#pragma unroll
    for (int i = 0; i < KEEP; ++i) scale[i] = byte[i];
    fetch_small(row + step);
    float2 sum2 = make_float2(0.f, 0.f);
    auto operands = [&](int i, float2 (&d)[4], float2 (&n)[4], float2 (&g)[4]) {
      // (read again for the second use: in registers they would not all fit)
      unpack8(lds16(mine_dy + slot * S::kStage + i * T * 16), d);
      const uint32_t src = mine_h + slot * S::kStage + i * T * S::kH;
      LoadedH<H> h;
      if (H == 2) {
        h.codes = lds8(src);
        h.byte = scale[i];
      } else {
        h.raw.w[0] = lds16(src);
        if (H == 1) h.raw.w[H == 1 ? 1 : 0] = lds16(src + T * 16);
      }
      h.normalised(rstd, n);
      const float4 u = gain_s[chunk_of(i)], v = gain_s[32 * WPR * KEEP + chunk_of(i)];
      g[0] = mul2(d[0], make_float2(u.x, u.y));
      g[1] = mul2(d[1], make_float2(u.z, u.w));
      g[2] = mul2(d[2], make_float2(v.x, v.y));
      g[3] = mul2(d[3], make_float2(v.z, v.w));
    };
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
      if (chunk_of(i) >= n8) break;
      float2 d[4], n[4], g[4];
      operands(i, d, n, g);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        sum2 = fma2(g[k], n[k], sum2);
        acc[i][k] = fma2(d[k], n[k], acc[i][k]);
      }
    }
    float sum = sum2.x + sum2.y;
    if (ST > 1) fetch(row + (ST - 1) * step, next);  // into the slot of the row before, which is done
    sum = warp_sum(sum);
    if (WPR > 1) {
      if (lane == 0) part[it & 1][warp] = sum;
      asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(32 * WPR) : "memory");
      sum = 0.f;
#pragma unroll
      for (int w = 0; w < WPR; ++w) sum += part[it & 1][group * WPR + w];
    }
    const float c = sum * per_col;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
      if (chunk_of(i) >= n8) break;
      float2 d[4], n[4], g[4];
      operands(i, d, n, g);
      if (S::kRingRg && a.residual_grad) {
        const uint32_t src = mine_rg + slot * S::kStage + i * T * S::kRg;
        rg[i].w[0] = lds16(src);
        if (F32) rg[i].w[F32 ? 1 : 0] = lds16(src + T * 16);
      }
      store_dh<F32>(a, g, n, rg[i], rstd, c, row, chunk_of(i));
    }
    slot = slot + 1 == ST ? 0 : slot + 1;
    next = next + 1 == ST ? 0 : next + 1;
  }
  copy_wait<0>();
  if (!a.partial) return;
  __syncthreads();  // the ring is empty; the sums take its place
  constexpr int kWidth = 32 * WPR * KEEP * 8;  // columns that a group has lanes for
#pragma unroll
  for (int i = 0; i < KEEP; ++i)
    if (chunk_of(i) < n8) store8<true>(columns, group * kWidth + chunk_of(i) * 8, acc[i]);
  __syncthreads();
  const int64_t left = (a.rows - blockIdx.x + gridDim.x - 1) / gridDim.x;  // (few rows: not every group had one)
  const int groups = (int)(left < kGroups ? left : kGroups);
  float* const out = a.partial + (int64_t)blockIdx.x * a.cols;
  for (int c = threadIdx.x * 4; c < n8 * 8; c += T * 4) {
    float4 t = *reinterpret_cast<const float4*>(columns + c);
    for (int g = 1; g < groups; ++g) {
      const float4 u = *reinterpret_cast<const float4*>(columns + g * kWidth + c);
      t = make_float4(t.x + u.x, t.y + u.y, t.z + u.z, t.w + u.w);
    }
    *reinterpret_cast<float4*>(out + c) = t;
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
    float2 sum2 = make_float2(0.f, 0.f);
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
        float2 d[4], n[4], g[4];
        unpack8(dy[i].w[0], d);
        h[i].normalised(rstd, n);
        times_gain(a.gain, chunk, d, g);
#pragma unroll
        for (int k = 0; k < 4; ++k) sum2 = fma2(g[k], n[k], sum2);
      }
    }
    float sum = warp_sum(sum2.x + sum2.y);
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
  float2 acc[4] = {};
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
      float2 d[4], n[4], g[4];
      unpack8(dy[u].w[0], d);
      h[u].normalised(rstd, n);
      times_gain(a.gain, chunk, d, g);
#pragma unroll
      for (int k = 0; k < 4; ++k) acc[k] = fma2(d[k], n[k], acc[k]);
      store_dh<F32>(a, g, n, rg[u], rstd, c, row, chunk);
    }
  }
  if (!a.partial) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) *reinterpret_cast<float2*>(&part[warp][lane * 8 + 2 * i]) = acc[i];
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

template <int H, bool F32, int WPR, int KEEP>
cudaError_t launch_bwd_kept(const Bwd& k, const NormBwd& a, int sms, cudaStream_t s) {
  using S = BwdShape<H, F32, WPR, KEEP>;
  auto kern = rmsnorm_bwd_kernel<H, F32, WPR, KEEP>;
  static std::atomic<uint64_t> configured{0};  // per instantiation and device
  int dev;
  if (device_needs_config(configured, &dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kBytes);
    if (e != cudaSuccess) return e;
    device_configured(configured, dev);
  }
  const int64_t cap = sms < kMaxParts ? sms : kMaxParts, grid = a.rows < cap ? a.rows : cap;  // (few rows: one to a CTA)
  const cudaError_t e = launch_kernel(kern, dim3((unsigned)grid), dim3(S::kThreads), S::kBytes, s, k);
  count_launch();
  if (e != cudaSuccess || !a.dgain) return e;
  return launch_column_sums(k.partial, grid, a.cols, a.dgain, a.accumulate, s);
}

template <int H, bool F32>
cudaError_t launch_bwd(const Bwd& k, const NormBwd& a, int sms, cudaStream_t s) {
  if (a.cols <= kKeptCols) {
    const int64_t groups = ((a.cols >> 3) + 31) / 32;
    // The gradient wants threads more than long runs of its own: 8192 x 5120 with four / eight warps to a row, from 8 bits 54.1 / 51.4 us,
    // from and to binary32 135.5 / 115.8.  With a single chunk a lane it loses again: 8192 x 2048 25.9 us, with eight warps to a row 30.3.
    if (groups <= 2) return launch_bwd_kept<H, F32, 1, 2>(k, a, sms, s);
    if (groups <= 4) return launch_bwd_kept<H, F32, 2, 2>(k, a, sms, s);
    if (groups <= 8) return launch_bwd_kept<H, F32, 4, 2>(k, a, sms, s);
    if (groups <= 12) return launch_bwd_kept<H, F32, 4, 3>(k, a, sms, s);
    if (groups <= 16) return launch_bwd_kept<H, F32, 8, 2>(k, a, sms, s);
    if (groups <= 24) return launch_bwd_kept<H, F32, 8, 3>(k, a, sms, s);
    if (groups <= 40) return launch_bwd_kept<H, F32, 8, 5>(k, a, sms, s);
    if (groups <= 48) return launch_bwd_kept<H, F32, 16, 3>(k, a, sms, s);
    return launch_bwd_kept<H, F32, 16, 5>(k, a, sms, s);
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
  return (rows < kMaxParts ? rows : kMaxParts) * cols;
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

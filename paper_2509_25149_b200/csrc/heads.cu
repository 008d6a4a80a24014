// Norms of query and key heads with the rotation by position, and their gradient.
//   forward   n = x / sqrt(mean(x^2) + eps),  u = n gain,  y = u turned by the angles p inv_freq
//   gradient  u' = dy turned back;  dgain = sum of u' n;  g = u' gain;  dx = rstd (g - n mean(g n))
// Both are bound by HBM (4 and 6 bytes an element).  A head stays within G neighbouring lanes of a warp, eight elements to a lane (so its
// statistic takes log2 G shuffles, and the partner of a rotated element is a shuffle away), and a warp takes the heads of a row one
// step of 32 / G heads after the other.  Sine and cosine of a row's angles are the same for all its heads: the warp makes them once,
// the angle in 64 bits (a far position times a frequency has its last bits below binary32), and keeps them in shared memory.
#include <algorithm>

#include "around.h"
#include "copy8.cuh"
#include "ends.h"

namespace nvfp4 {

namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps, kMaxHalf = 128, kMaxCtas = 592;
enum { kPlain = 0, kHalves = 1, kNeighbours = 2 };  // which elements turn together

struct Args {
  const uint16_t* x;
  const uint16_t* dy;
  uint16_t* y;
  const float* gain_q;
  const float* gain_k;
  const float* inv_freq;
  Indices positions;
  float* partial;  // gradient: a row of 2 dim sums per CTA, or NULL
  int64_t rows, ldx, lddy, ldy, items;
  int heads_q, heads_k, dim, half, parts, steps_per_part;
  float eps, per_elem;
};

// cosine and sine of p f, f a binary32 number: the product, its multiples of pi and what is left of a turn in 64 bits
__device__ __forceinline__ float2 turn_of(int64_t p, float f) {
  double t = (double)p * (double)f * 0.31830988618379067154;  // in half turns
  t -= 2. * rint(0.5 * t);
  float s, c;
  sincospif((float)t, &s, &c);
  return make_float2(c, s);
}

// A lane's place in a head, and its share of the row's rotation
template <int G, int MODE>
struct Lane {
  int e0, partner;
  bool live;
  float c[8], s[8];  // a turned element is its own times c plus its partner's times s
  __device__ __forceinline__ Lane(const Args& a) {
    const int lane = threadIdx.x & 31;
    e0 = (lane % G) * 8;
    live = e0 < a.dim;
    partner = MODE != kHalves || e0 >= 2 * a.half ? lane : e0 < a.half ? lane + (a.half >> 3) : lane - (a.half >> 3);
  }
  // the warp makes the row's table in shared memory and every lane takes what it needs of it
  __device__ __forceinline__ void turn(const Args& a, float2* table, int64_t row) {
    if (MODE == kPlain) return;
    const int64_t p = a.positions.p ? a.positions[row] : row;
    for (int i = threadIdx.x & 31; i < a.half; i += 32) table[i] = turn_of(p, a.inv_freq[i]);
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float2 t = make_float2(1.f, 0.f);
      bool first;
      if (MODE == kHalves) {
        first = e0 < a.half;
        if (e0 < 2 * a.half) t = table[first ? e0 + j : e0 - a.half + j];
      } else {
        first = j % 2 == 0;
        if (e0 < 2 * a.half) t = table[(e0 + j) >> 1];
      }
      c[j] = t.x;
      s[j] = first ? -t.y : t.y;
    }
    __syncwarp();  // (the table is the next row's)
  }
  // what stands beside the elements of a chunk: their partners' values
  __device__ __forceinline__ void partners(uint4 raw, float (&v)[8]) const {
    if (MODE == kHalves) {
      uint4 r;
      r.x = __shfl_sync(0xffffffffu, raw.x, partner);
      r.y = __shfl_sync(0xffffffffu, raw.y, partner);
      r.z = __shfl_sync(0xffffffffu, raw.z, partner);
      r.w = __shfl_sync(0xffffffffu, raw.w, partner);
      unpack8(r, v);
    } else if (MODE == kNeighbours) {
      float w[8];
      unpack8(raw, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = w[j ^ 1];
    }
  }
};

template <int G>
__device__ __forceinline__ float head_sum(float v) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float dot8(const float (&a)[8], const float (&b)[8]) {
  float2 s = make_float2(a[0] * b[0], a[1] * b[1]);
#pragma unroll
  for (int j = 2; j < 8; j += 2) s = fma2(make_float2(a[j], a[j + 1]), make_float2(b[j], b[j + 1]), s);
  return s.x + s.y;
}
// 1 / sqrt(mean(x^2) + eps) of the head that a lane's group holds.  Finite values whose squares, or the sum of them, binary32 does not hold
// are taken times 2^-70 once more (one of them is above 2^50 then, and eps nothing beside it).
template <int G>
__device__ __forceinline__ float rstd_of(const Args& a, const float (&x)[8]) {
  float sum = head_sum<G>(dot8(x, x));
  if (__builtin_expect(__any_sync(0xffffffffu, !(sum <= 3.402823466e38f)), 0)) {
    float w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = x[j] * 0x1p-70f;
    const float scaled = head_sum<G>(dot8(w, w));
    if (!(sum <= 3.402823466e38f)) return rsqrtf(scaled * a.per_elem) * 0x1p-70f;
  }
  return rsqrtf(fmaf(sum, a.per_elem, a.eps));
}

// The steps of one kind of heads (queries, then keys) that an item has: where they begin and end
struct Range {
  int from, to, head0, heads;
  __device__ __forceinline__ Range(const Args& a, int part, int kind, int per_step) {
    const int nq = (a.heads_q + per_step - 1) / per_step, nk = (a.heads_k + per_step - 1) / per_step, begin = kind ? nq : 0;
    const int t0 = part * a.steps_per_part, t1 = min(t0 + a.steps_per_part, nq + nk);
    from = max(t0, begin) - begin;
    to = min(t1, begin + (kind ? nk : nq)) - begin;
    head0 = kind ? a.heads_q : 0;
    heads = kind ? a.heads_k : a.heads_q;
  }
};

template <int G, int MODE>
__global__ void __launch_bounds__(kThreads) headnorm_fwd_kernel(const Args a) {
  constexpr int kHeads = 32 / G, kAhead = 4;  // heads of a step, steps whose loads are on their way together
  __shared__ float2 tables[kWarps][MODE == kPlain ? 1 : kMaxHalf];
  const int64_t item = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  Lane<G, MODE> l(a);
  griddep_wait();
  griddep_launch_dependents();
  if (item >= a.items) return;
  const int64_t row = item / a.parts;
  const int part = (int)(item - row * a.parts), sub = (threadIdx.x & 31) / G;
  l.turn(a, tables[threadIdx.x >> 5], row);
  const uint16_t* const x = a.x + row * a.ldx;
  uint16_t* const y = a.y + row * a.ldy;
#pragma unroll 1
  for (int kind = 0; kind < 2; ++kind) {
    const Range r(a, part, kind, kHeads);
    if (r.from >= r.to) continue;
    float gc[8], gs[8];
    load_gain(l.live ? (kind ? a.gain_k : a.gain_q) : nullptr, l.e0, gc);
    if (MODE != kPlain) {
#pragma unroll
      for (int j = 0; j < 8; ++j) gs[j] = (MODE == kHalves ? __shfl_sync(0xffffffffu, gc[j], l.partner) : gc[j ^ 1]) * l.s[j];
#pragma unroll
      for (int j = 0; j < 8; ++j) gc[j] *= l.c[j];
    }
#pragma unroll 1
    for (int t0 = r.from; t0 < r.to; t0 += kAhead) {
      uint4 raw[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int head = (t0 + u) * kHeads + sub;
        const bool there = l.live && t0 + u < r.to && head < r.heads;
        raw[u] = there ? ldg128_stream(x + (int64_t)(r.head0 + head) * a.dim + l.e0) : make_uint4(0u, 0u, 0u, 0u);
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (t0 + u >= r.to) break;
        const int head = (t0 + u) * kHeads + sub;
        float v[8], p[8], out[8];
        unpack8(raw[u], v);
        const float rstd = rstd_of<G>(a, v);
        l.partners(raw[u], p);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          out[j] = v[j] * rstd * gc[j];
          if (MODE != kPlain) out[j] = fmaf(p[j] * rstd, gs[j], out[j]);
        }
        if (l.live && head < r.heads) store8<false>(y, (int64_t)(r.head0 + head) * a.dim + l.e0, out);
      }
    }
  }
}

// A warp keeps the sums of its lanes' elements over all its rows and heads in registers; at the end those of a CTA are added in a fixed
// order and leave as a row of partial sums, which a second kernel adds.
template <int G, int MODE>
__global__ void __launch_bounds__(kThreads) headnorm_bwd_kernel(const Args a) {
  constexpr int kHeads = 32 / G, kAhead = 2;
  __shared__ float2 tables[kWarps][MODE == kPlain ? 1 : kMaxHalf];
  __shared__ float sums[kWarps][2][G * 8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane / G;
  Lane<G, MODE> l(a);
  griddep_wait();
  griddep_launch_dependents();
  float acc[2][8] = {};
  for (int64_t item = (int64_t)blockIdx.x * kWarps + warp; item < a.items; item += (int64_t)gridDim.x * kWarps) {
    const int64_t row = item / a.parts;
    const int part = (int)(item - row * a.parts);
    l.turn(a, tables[warp], row);
    const uint16_t* const x = a.x + row * a.ldx;
    const uint16_t* const dy = a.dy + row * a.lddy;
    uint16_t* const dx = a.y + row * a.ldy;
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
      const Range r(a, part, kind, kHeads);
      if (r.from >= r.to) continue;
      float gain[8];
      load_gain(l.live ? (kind ? a.gain_k : a.gain_q) : nullptr, l.e0, gain);
#pragma unroll 1
      for (int t0 = r.from; t0 < r.to; t0 += kAhead) {
        uint4 rx[kAhead], rd[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          const int head = (t0 + u) * kHeads + sub;
          const bool there = l.live && t0 + u < r.to && head < r.heads;
          const int64_t at = (int64_t)(r.head0 + head) * a.dim + l.e0;
          rx[u] = there ? ldg128_stream(x + at) : make_uint4(0u, 0u, 0u, 0u);
          rd[u] = there ? ldg128_stream(dy + at) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          if (t0 + u >= r.to) break;
          const int head = (t0 + u) * kHeads + sub;
          float n[8], d[8], p[8], g[8];
          unpack8(rx[u], n);
          unpack8(rd[u], d);
          const float rstd = rstd_of<G>(a, n);
          l.partners(rd[u], p);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            n[j] *= rstd;
            if (MODE != kPlain) d[j] = fmaf(p[j], -l.s[j], d[j] * l.c[j]);
            acc[kind][j] = fmaf(d[j], n[j], acc[kind][j]);
            g[j] = d[j] * gain[j];
          }
          const float m = head_sum<G>(dot8(g, n)) * a.per_elem;
#pragma unroll
          for (int j = 0; j < 8; ++j) g[j] = rstd * fmaf(-n[j], m, g[j]);
          if (l.live && head < r.heads) store8<false>(dx, (int64_t)(r.head0 + head) * a.dim + l.e0, g);
        }
      }
    }
  }
  if (!a.partial) return;
#pragma unroll
  for (int kind = 0; kind < 2; ++kind)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float v = acc[kind][j];
#pragma unroll
      for (int o = G; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
      if (lane < G) sums[warp][kind][l.e0 + j] = v;
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * a.dim; i += kThreads) {
    const int kind = i >= a.dim, e = i - kind * a.dim;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) v += sums[w][kind][e];
    a.partial[(int64_t)blockIdx.x * 2 * a.dim + i] = v;
  }
}

int lanes_of(int dim) {
  int g = 1;
  while (g * 8 < dim) g *= 2;
  return g;
}
// Items of a row: as many as give every SM two CTAs where the rows alone do not
struct Split {
  int parts, per_part;
  int64_t items;
  Split(int64_t rows, int heads_q, int heads_k, int dim) {
    const int per_step = 32 / lanes_of(dim), steps = (heads_q + per_step - 1) / per_step + (heads_k + per_step - 1) / per_step;
    const int64_t want = std::max<int64_t>(1, (2 * 148 * kWarps + rows - 1) / rows);
    per_part = (int)((steps + std::min<int64_t>(want, steps) - 1) / std::min<int64_t>(want, steps));
    parts = (steps + per_part - 1) / per_part;
    items = rows * parts;
  }
};
int64_t bwd_ctas(int64_t items) { return std::min<int64_t>((items + kWarps - 1) / kWarps, kMaxCtas); }

Args args_of(const Heads& h, const Split& split) {
  Args a{};
  a.x = static_cast<const uint16_t*>(h.x);
  a.dy = static_cast<const uint16_t*>(h.dy);
  a.y = static_cast<uint16_t*>(h.y);
  a.gain_q = h.gain_q; a.gain_k = h.gain_k;
  a.inv_freq = h.inv_freq;
  a.positions = h.positions;
  a.rows = h.rows; a.ldx = h.ldx; a.lddy = h.lddy; a.ldy = h.ldy;
  a.items = split.items; a.parts = split.parts; a.steps_per_part = split.per_part;
  a.heads_q = h.heads_q; a.heads_k = h.heads_k;
  a.dim = h.dim; a.half = h.rotary / 2;
  a.eps = h.eps; a.per_elem = 1.f / (float)h.dim;
  return a;
}

template <int G, int MODE>
cudaError_t launch(bool bwd, const Args& a, unsigned grid, cudaStream_t s) {
  return bwd ? launch_divided(15, headnorm_bwd_kernel<G, MODE>, dim3(grid), dim3(kThreads), 0, s, a)
             : launch_divided(15, headnorm_fwd_kernel<G, MODE>, dim3(grid), dim3(kThreads), 0, s, a);
}
template <int G>
cudaError_t launch(bool bwd, bool interleaved, const Args& a, unsigned grid, cudaStream_t s) {
  if (a.half == 0) return launch<G, kPlain>(bwd, a, grid, s);
  return interleaved ? launch<G, kNeighbours>(bwd, a, grid, s) : launch<G, kHalves>(bwd, a, grid, s);
}
cudaError_t launch(bool bwd, bool interleaved, const Args& a, unsigned grid, cudaStream_t s) {
  cudaError_t e;
  switch (lanes_of(a.dim)) {
    case 1: e = launch<1>(bwd, interleaved, a, grid, s); break;
    case 2: e = launch<2>(bwd, interleaved, a, grid, s); break;
    case 4: e = launch<4>(bwd, interleaved, a, grid, s); break;
    case 8: e = launch<8>(bwd, interleaved, a, grid, s); break;
    case 16: e = launch<16>(bwd, interleaved, a, grid, s); break;
    default: e = launch<32>(bwd, interleaved, a, grid, s); break;
  }
  count_launch();
  return e;
}

}  // namespace

cudaError_t launch_headnorm_fwd(const Heads& h, cudaStream_t s) {
  const Split split(h.rows, h.heads_q, h.heads_k, h.dim);
  return launch(false, h.interleaved, args_of(h, split), (unsigned)((split.items + kWarps - 1) / kWarps), s);
}

int64_t headnorm_bwd_workspace_floats(int64_t rows, int heads_q, int heads_k, int dim) {
  return bwd_ctas(Split(rows, heads_q, heads_k, dim).items) * 2 * dim;
}

cudaError_t launch_headnorm_bwd(const Heads& h, cudaStream_t s) {
  const Split split(h.rows, h.heads_q, h.heads_k, h.dim);
  Args a = args_of(h, split);
  const bool sums = h.dgain_q || h.dgain_k;
  a.partial = sums ? h.workspace : nullptr;
  const int64_t ctas = bwd_ctas(split.items);
  const cudaError_t e = launch(true, h.interleaved, a, (unsigned)ctas, s);
  if (e != cudaSuccess || !sums) return e;
  return launch_column_sums(h.workspace, ctas, 2 * h.dim, h.dgain_q, h.accumulate, s, h.dgain_k, h.dim);
}

}  // namespace nvfp4

// Norms of query and key heads with the rotation by position, and their gradient.
//   forward   n = x / sqrt(mean(x^2) + eps),  u = n gain,  y = u turned by the angles p inv_freq
//   gradient  u' = dy turned back;  dgain = sum of u' n;  g = u' gain;  dx = rstd (g - n mean(g n))
// Both are bound by HBM (4 and 6 bytes an element).  A head stays within G neighbouring lanes of a warp, eight elements to a lane (so its
// statistic takes log2 G shuffles; both elements of a pair that turns are the same lane's: where they are half a rotation apart it takes two runs
// of four).  A step of a warp is 32 / G or twice as many heads of one kind of a row (two heads to a lane halve what a step costs beside its arithmetic,
// and their statistics do not wait for each other); all rows' steps stand in one line, of which every resident warp takes an equal
// share.  What a lane is going to need comes by cp.async through a ring in shared memory in which every thread has places of its own, so that loads
// stay in flight whatever the registers hold and over the end of a row.  Sine and cosine of a row's angles are the same for all its heads: the warp makes them once a row, the angle in 64 bits (a far position
// times a frequency has its last bits below binary32), and keeps them in shared memory.
// 8192 rows of 40 + 8 heads of 128: 39.2 us (79 % of the copy rate) and 59 with 4.3 for the sums of the gains' gradients (78 %).  What they wait for is latency: 94 and 155
// instructions a lane for eight elements, shuffles behind one another; 24 warps an SM with one head to a lane took 41 and 65.
#include <algorithm>

#include "around.h"
#include "copy8.cuh"
#include "ends.h"

namespace nvfp4 {

namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps, kMaxHalf = 128;
template <int N>
constexpr int kFwdRing = 8;  // steps that a warp's ring has room for, with N heads to a lane
template <int N>
constexpr int kBwdRing = N == 2 ? 4 : 8;
constexpr int kFwdCtas = 148 * 2, kBwdCtas = 148 * 2;  // as many as are resident
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
  float* dgain_q;  // the gains' gradients where the CTAs are one cluster, which adds up its sums itself, or NULL
  float* dgain_k;
  bool joined, accumulate;
  int64_t ldx, lddy, ldy, steps;  // steps: of all rows
  int heads_q, heads_k, dim, half, steps_q, per_row;  // steps of a row's query heads, and of all its heads
  float eps, per_elem;
};

// What a CTA's warps read again and again
struct Shared {
  double per_turn[kMaxHalf];  // inverse frequencies over pi
  float gain[2][256];         // of query and key heads
  float2 table[kWarps][kMaxHalf];
  __device__ __forceinline__ void fill(const Args& a) {
    for (int i = threadIdx.x; i < a.half; i += kThreads) per_turn[i] = (double)a.inv_freq[i] * 0.31830988618379067154;
    for (int i = threadIdx.x; i < a.dim; i += kThreads) {
      gain[0][i] = a.gain_q ? a.gain_q[i] : 1.f;
      gain[1][i] = a.gain_k ? a.gain_k[i] : 1.f;
    }
    for (int i = 2 * 256 - 1 - threadIdx.x; i >= 0; i -= kThreads)
      if (i % 256 >= a.dim) gain[i / 256][i % 256] = 0.f;  // (of lanes beyond the head)
  }
};
// cosine and sine of an angle of p f half turns: the product, its whole turns and what is left in 64 bits
__device__ __forceinline__ float2 turn_of(double p, double f) {
  double t = p * f;
  t -= 2. * rint(0.5 * t);
  float s, c;
  sincospif((float)t, &s, &c);
  return make_float2(c, s);
}

// A lane's place in a head, and its share of the row's rotation
template <int G, int MODE>
struct Lane {
  int sub, e0, gap;  // its group's number in the warp; its elements are e0 .. e0 + 3 and e0 + gap .. e0 + gap + 3
  bool live;
  float2 c[4], s[4];  // a turned element is its own times c plus its partner's times s
  __device__ __forceinline__ Lane(const Args& a) {
    const int l = (threadIdx.x & 31) % G;
    sub = (threadIdx.x & 31) / G;
    live = l * 8 < a.dim;
    const bool apart = MODE == kHalves && l * 4 < a.half;
    e0 = apart ? l * 4 : l * 8;
    gap = apart ? a.half : 4;
  }
  __device__ __forceinline__ int element(int j) const { return e0 + (j < 2 ? 2 * j : gap + 2 * j - 4); }  // of pair j
  // the warp makes the row's table in shared memory and every lane takes what it needs of it
  __device__ __forceinline__ void turn(const Args& a, Shared& sh, int64_t row) {
    if (MODE == kPlain) return;
    float2* const table = sh.table[threadIdx.x >> 5];
    const double p = (double)(a.positions.p ? a.positions[row] : row);
    for (int i = threadIdx.x & 31; i < a.half; i += 32) table[i] = turn_of(p, sh.per_turn[i]);
    __syncwarp();
    const float2 still = make_float2(1.f, 0.f);
#pragma unroll
    for (int j = 0; j < (MODE == kHalves ? 2 : 4); ++j) {
      if (MODE == kHalves) {
        const bool turns = gap != 4;  // (half a rotation is eight elements or more)
        const float2 t = turns ? table[e0 + 2 * j] : still, u = turns ? table[e0 + 2 * j + 1] : still;
        c[j] = c[j + 2] = make_float2(t.x, u.x);
        s[j] = make_float2(-t.y, -u.y);
        s[j + 2] = make_float2(t.y, u.y);
      } else {
        const float2 t = e0 < 2 * a.half ? table[(e0 >> 1) + j] : still;
        c[j] = both(t.x);
        s[j] = make_float2(-t.y, t.y);
      }
    }
    __syncwarp();  // (the table is the next row's)
  }
  // what stands beside the elements: their partners
  __device__ __forceinline__ static float2 partner(const float2 (&v)[4], int j) {
    return MODE == kHalves ? v[j ^ 2] : make_float2(v[j].y, v[j].x);
  }
  __device__ __forceinline__ void load_gains(const Shared& sh, int key, float2 (&g)[4]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) g[j] = *reinterpret_cast<const float2*>(&sh.gain[key][element(j)]);
  }
  __device__ __forceinline__ void fetch(uint32_t dst, const uint16_t* p, bool there) const {
    if (MODE == kHalves) {
      copy_async<8>(dst, p, there);
      copy_async<8>(dst + 8, p + (there ? gap : 0), there);
    } else {
      copy_async<16>(dst, p, there);
    }
  }
  // (first to leave L2: 8192 rows of 48 heads 41.0 -> 40.0 us)
  __device__ __forceinline__ void store(uint16_t* p, const float2 (&v)[4]) const {
    if (MODE == kHalves) {
      __stcs(reinterpret_cast<uint2*>(p), make_uint2(pack2(v[0].x, v[0].y), pack2(v[1].x, v[1].y)));
      __stcs(reinterpret_cast<uint2*>(p + gap), make_uint2(pack2(v[2].x, v[2].y), pack2(v[3].x, v[3].y)));
    } else {
      __stcs(reinterpret_cast<uint4*>(p), make_uint4(pack2(v[0].x, v[0].y), pack2(v[1].x, v[1].y), pack2(v[2].x, v[2].y), pack2(v[3].x, v[3].y)));
    }
  }
};

template <int G>
__device__ __forceinline__ float head_sum(float v) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float dot8(const float2 (&a)[4], const float2 (&b)[4]) {
  const float2 s = add2(fma2(a[1], b[1], mul2(a[0], b[0])), fma2(a[3], b[3], mul2(a[2], b[2])));
  return s.x + s.y;
}
__device__ __forceinline__ float rsqrt_fast(float v) {  // (of normal numbers: eps is one at least)
  float r;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
// 1 / sqrt(mean(x^2) + eps) of the N heads that a lane's group holds.  Finite values whose squares, or the sum of them and eps, binary32 does not hold
// are multiplied by 2^-70, eps by 2^-140, and the result is that of what they are now; `shift` says so.  True where the warp had such a head.
template <int G, int N>
__device__ __forceinline__ bool rstd_of(const Args& a, float2 (&x)[N][4], float (&rstd)[N], float (*shift)[N] = nullptr) {
  float sum[N];
  bool lost = false;
#pragma unroll
  for (int k = 0; k < N; ++k) sum[k] = dot8(x[k], x[k]);
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < N; ++k) sum[k] += __shfl_xor_sync(0xffffffffu, sum[k], o);
#pragma unroll
  for (int k = 0; k < N; ++k) {
    sum[k] = fmaf(sum[k], a.per_elem, a.eps);
    lost |= !(sum[k] <= 3.402823466e38f);
    rstd[k] = rsqrt_fast(sum[k]);
  }
  if (__builtin_expect(!__any_sync(0xffffffffu, lost), 1)) return false;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const bool far = !(sum[k] <= 3.402823466e38f);
    float2 w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = mul2(x[k][j], both(0x1p-70f));
    const float scaled = head_sum<G>(dot8(w, w));
    if (!far) continue;
    rstd[k] = rsqrt_fast(fmaf(scaled, a.per_elem, a.eps * 0x1p-140f));
#pragma unroll
    for (int j = 0; j < 4; ++j) x[k][j] = w[j];
    if (shift) (*shift)[k] = 0x1p-70f;
  }
  return true;
}

// Where a warp is in its share of the steps: `left` more of this kind of heads in the row, of which the lane's group has head h
struct Walk {
  int64_t row;
  int key, h, left;  // key: 0 the query heads, 1 the key heads
  __device__ __forceinline__ Walk(const Args& a, int64_t step, int per_step, int sub) : row(step / a.per_row) {
    const int t = (int)(step - row * a.per_row);
    key = t >= a.steps_q;
    h = (key ? t - a.steps_q : t) * per_step + sub;
    left = (key ? a.per_row : a.steps_q) - t;
  }
  __device__ __forceinline__ int heads(const Args& a) const { return key ? a.heads_k : a.heads_q; }
  __device__ __forceinline__ int64_t offset(const Args& a, int64_t ld, int e0) const { return row * ld + (int64_t)((key ? a.heads_q : 0) + h) * a.dim + e0; }
  // one step on; true where another kind of heads, or another row, begins
  __device__ __forceinline__ bool next(const Args& a, int per_step, int sub) {
    h += per_step;
    if (--left > 0) return false;
    h = sub;
    if (!key && a.per_row > a.steps_q) {
      key = 1;
      left = a.per_row - a.steps_q;
    } else {
      ++row;
      key = a.steps_q == 0;
      left = key ? a.per_row : a.steps_q;
    }
    return true;
  }
};

template <int G, int MODE, int N, bool FULL>
__global__ void __launch_bounds__(kThreads, 2) headnorm_fwd_kernel(const Args a) {
  constexpr int kHeads = 32 / G, kStep = kHeads * N, kRing = kFwdRing<N>, kSlot = kThreads * 16 * N;  // heads of a step, bytes of a step of all warps
  __shared__ Shared sh;
  extern __shared__ __align__(16) uint8_t ring[];
  const int64_t warps = (int64_t)gridDim.x * kWarps, w = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int64_t first = a.steps * w / warps;
  const int steps = (int)(a.steps * (w + 1) / warps - first), head = kHeads * a.dim;  // head: from a lane's first one to its second
  Lane<G, MODE> l(a);
  const uint32_t mine = smem_u32(ring) + threadIdx.x * 16;
  Walk ahead(a, first, kStep, l.sub), at = ahead;
  const uint16_t* from = a.x + ahead.offset(a, a.ldx, l.e0);
  uint16_t* to = a.y + at.offset(a, a.ldy, l.e0);
  auto fetch = [&](int i) {
    if (i < steps) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const bool there = FULL || (l.live && ahead.h + k * kHeads < ahead.heads(a));
        l.fetch(mine + (i % kRing) * kSlot + k * (kThreads * 16), there ? from + k * head : a.x, there);
      }
      from += N * head;
      if (ahead.next(a, kStep, l.sub)) from = a.x + ahead.offset(a, a.ldx, l.e0);
    }
    copy_commit();  // (an empty group where there is no step: the count of groups stays that of the steps)
  };
  griddep_wait();
  griddep_launch_dependents();
#pragma unroll
  for (int u = 0; u < kRing - 1; ++u) fetch(u);
  sh.fill(a);
  __syncthreads();
  float2 gc[4], gs[4];
  int64_t turned = -1;  // the row whose rotation the lane has
  bool corner = true;
  for (int i = 0; i < steps; ++i) {
    if (corner) {
      if (turned != at.row) l.turn(a, sh, at.row);
      turned = at.row;
      float2 g[4];
      l.load_gains(sh, at.key, g);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        gc[j] = MODE == kPlain ? g[j] : mul2(g[j], l.c[j]);
        if (MODE != kPlain) gs[j] = mul2(l.partner(g, j), l.s[j]);
      }
    }
    copy_wait<kRing - 2>();
    float2 v[N][4];
    float rstd[N];
#pragma unroll
    for (int k = 0; k < N; ++k) unpack8(lds16(mine + (i % kRing) * kSlot + k * (kThreads * 16)), v[k]);
    fetch(i + kRing - 1);  // into the slot of the step before, whose values went into registers a turn ago
    rstd_of<G, N>(a, v, rstd);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      float2 out[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[k][j] = mul2(v[k][j], both(rstd[k]));  // (first: x gain may be too small for binary32)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        out[j] = mul2(v[k][j], gc[j]);
        if (MODE != kPlain) out[j] = fma2(l.partner(v[k], j), gs[j], out[j]);
      }
      if (FULL || (l.live && at.h + k * kHeads < at.heads(a))) l.store(to + k * head, out);
    }
    to += N * head;
    corner = at.next(a, kStep, l.sub);
    if (corner) to = a.y + at.offset(a, a.ldy, l.e0);
  }
  copy_wait<0>();
}

// A warp keeps the sums of its lanes' elements over all its steps in registers; at the end those of a CTA are added in a fixed
// order and leave as a row of partial sums, which a second kernel adds.
template <int G, int MODE, int N, bool FULL>
__global__ void __launch_bounds__(kThreads, 2) headnorm_bwd_kernel(const Args a) {
  constexpr int kHeads = 32 / G, kStep = kHeads * N, kRing = kBwdRing<N>, kSlot = kThreads * 32 * N;
  __shared__ Shared sh;
  extern __shared__ __align__(16) uint8_t ring[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t warps = (int64_t)gridDim.x * kWarps, w = (int64_t)blockIdx.x * kWarps + warp;
  const int64_t first = a.steps * w / warps;
  const int steps = (int)(a.steps * (w + 1) / warps - first), head = kHeads * a.dim;
  Lane<G, MODE> l(a);
  const uint32_t mine = smem_u32(ring) + threadIdx.x * 16;
  Walk ahead(a, first, kStep, l.sub), at = ahead;
  const uint16_t* from_x = a.x + ahead.offset(a, a.ldx, l.e0);
  const uint16_t* from_dy = a.dy + ahead.offset(a, a.lddy, l.e0);
  uint16_t* to = a.y + at.offset(a, a.ldy, l.e0);
  auto fetch = [&](int i) {
    if (i < steps) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const bool there = FULL || (l.live && ahead.h + k * kHeads < ahead.heads(a));
        const uint32_t dst = mine + (i % kRing) * kSlot + k * (kThreads * 32);
        l.fetch(dst, there ? from_x + k * head : a.x, there);
        l.fetch(dst + kThreads * 16, there ? from_dy + k * head : a.dy, there);
      }
      from_x += N * head;
      from_dy += N * head;
      if (ahead.next(a, kStep, l.sub)) {
        from_x = a.x + ahead.offset(a, a.ldx, l.e0);
        from_dy = a.dy + ahead.offset(a, a.lddy, l.e0);
      }
    }
    copy_commit();
  };
  griddep_wait();
  griddep_launch_dependents();
#pragma unroll
  for (int u = 0; u < kRing - 1; ++u) fetch(u);
  sh.fill(a);
  __syncthreads();
  // acc: of the kind of heads at hand; the other kind's wait in `other`
  float2 acc[4] = {}, other[4] = {}, gain[4];
  auto change = [&] {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 t = acc[j];
      acc[j] = other[j];
      other[j] = t;
    }
  };
  int64_t turned = -1;
  int key = 0;  // the kind that acc belongs to
  bool corner = true;
  for (int i = 0; i < steps; ++i) {
    if (corner) {
      if (turned != at.row) l.turn(a, sh, at.row);
      turned = at.row;
      l.load_gains(sh, at.key, gain);
      if (key != at.key) change();
      key = at.key;
    }
    copy_wait<kRing - 2>();
    float2 n[N][4], y[N][4];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const uint32_t src = mine + (i % kRing) * kSlot + k * (kThreads * 32);
      unpack8(lds16(src), n[k]);
      unpack8(lds16(src + kThreads * 16), y[k]);
    }
    fetch(i + kRing - 1);
    float rstd[N], m[N], shift[N];
#pragma unroll
    for (int k = 0; k < N; ++k) shift[k] = 1.f;
    const bool far = rstd_of<G, N>(a, n, rstd, &shift);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      float2 g[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        n[k][j] = mul2(n[k][j], both(rstd[k]));
        // turned back: the sines change their sign, which those of the partner's have
        g[j] = MODE == kPlain ? y[k][j] : fma2(l.partner(y[k], j), l.partner(l.s, j), mul2(y[k][j], l.c[j]));
        acc[j] = fma2(g[j], n[k][j], acc[j]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) y[k][j] = mul2(g[j], gain[j]);
      m[k] = dot8(y[k], n[k]);
    }
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1)
#pragma unroll
      for (int k = 0; k < N; ++k) m[k] += __shfl_xor_sync(0xffffffffu, m[k], o);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float r = far ? rstd[k] * shift[k] : rstd[k];
      float2 out[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) out[j] = mul2(fma2(n[k][j], both(-m[k] * a.per_elem), y[k][j]), both(r));
      if (FULL || (l.live && at.h + k * kHeads < at.heads(a))) l.store(to + k * head, out);
    }
    to += N * head;
    corner = at.next(a, kStep, l.sub);
    if (corner) to = a.y + at.offset(a, a.ldy, l.e0);
  }
  copy_wait<0>();
  if (!a.partial && !a.joined) return;
  if (key) change();
  __syncthreads();  // the ring is empty; the sums take its place
  auto sums = reinterpret_cast<float(*)[2][256]>(ring);
  static_assert(kWarps * 2 * 256 * 4 <= kRing * kSlot, "the sums reuse the ring");
#pragma unroll
  for (int kind = 0; kind < 2; ++kind)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float2 v = kind ? other[j] : acc[j];
#pragma unroll
      for (int o = G; o < 32; o <<= 1) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
      }
      if (lane < G && l.live) *reinterpret_cast<float2*>(&sums[warp][kind][l.element(j)]) = v;
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * a.dim; i += kThreads) {
    const int kind = i >= a.dim, e = i - kind * a.dim;
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) v += sums[k][kind][e];
    if (a.joined)
      sh.gain[kind][e] = v;  // (nobody needs the gains any more)
    else
      a.partial[(int64_t)blockIdx.x * 2 * a.dim + i] = v;
  }
  if (!a.joined) return;
  cluster_sync();
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < 2 * a.dim; i += kThreads) {
      const int kind = i >= a.dim, e = i - kind * a.dim;
      float* const to = kind ? a.dgain_k : a.dgain_q;
      if (!to) continue;
      float v = sh.gain[kind][e];
      for (uint32_t r = 1; r < gridDim.x; ++r) v += ld_of_rank(&sh.gain[kind][e], r);
      to[e] = a.accumulate ? to[e] + v : v;
    }
  cluster_sync();  // none may go while its sums are read
}

int lanes_of(int dim) {  // (heads of less than 32 elements leave lanes idle)
  int g = 4;
  while (g * 8 < dim) g *= 2;
  return g;
}
int64_t steps_of_row(int heads_q, int heads_k, int per_step) { return (heads_q + per_step - 1) / per_step + (heads_k + per_step - 1) / per_step; }
// Two heads to a lane unless more than an eighth of the places would be empty for it
int heads_of_lane(int heads_q, int heads_k, int dim) {
  const int per_step = 32 / lanes_of(dim);
  return 8 * 2 * steps_of_row(heads_q, heads_k, 2 * per_step) <= 9 * steps_of_row(heads_q, heads_k, per_step) ? 2 : 1;
}
int64_t steps_of_row(int heads_q, int heads_k, int dim, int n) { return steps_of_row(heads_q, heads_k, n * (32 / lanes_of(dim))); }
// Few steps: eight CTAs at most, a cluster that adds up the gains' gradients itself, which is a launch less for the host (rows of 40 + 8 heads of 128, on the
// GPU: 1 row, 12 steps, 4.1 -> 3.8 us, 16 rows 5.0 -> 5.7, 64 rows 5.4 -> 11)
bool is_joined(int64_t steps) { return steps <= 128; }
constexpr int kJoined = 8;
unsigned ctas_of(int64_t steps, int most) { return (unsigned)std::min<int64_t>((steps + kWarps - 1) / kWarps, most); }

Args args_of(const Heads& h, int n) {
  Args a{};
  a.x = static_cast<const uint16_t*>(h.x);
  a.dy = static_cast<const uint16_t*>(h.dy);
  a.y = static_cast<uint16_t*>(h.y);
  a.gain_q = h.gain_q; a.gain_k = h.gain_k;
  a.inv_freq = h.inv_freq;
  a.positions = h.positions;
  a.ldx = h.ldx; a.lddy = h.lddy; a.ldy = h.ldy;
  a.heads_q = h.heads_q; a.heads_k = h.heads_k;
  a.dim = h.dim; a.half = h.rotary / 2;
  a.steps_q = (int)steps_of_row(h.heads_q, 0, h.dim, n);
  a.per_row = (int)steps_of_row(h.heads_q, h.heads_k, h.dim, n);
  a.steps = h.rows * a.per_row;
  a.eps = h.eps; a.per_elem = 1.f / (float)h.dim;
  return a;
}

template <int G, int MODE, int N, bool FULL>
cudaError_t launch(bool bwd, const Args& a, cudaStream_t s) {
  const auto kern = bwd ? headnorm_bwd_kernel<G, MODE, N, FULL> : headnorm_fwd_kernel<G, MODE, N, FULL>;
  const int smem = kThreads * N * (bwd ? kBwdRing<N> * 32 : kFwdRing<N> * 16);
  static std::atomic<uint64_t> configured[2]{};  // per instantiation and device
  int dev;
  if (device_needs_config(configured[bwd], &dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    device_configured(configured[bwd], dev);
  }
  const unsigned ctas = ctas_of(a.steps, bwd ? (a.joined ? kJoined : kBwdCtas) : kFwdCtas);
  if (a.joined && ctas > 1) return launch_cluster(ctas, kern, dim3(ctas), dim3(kThreads), smem, s, a);
  return launch_divided(100, kern, dim3(ctas), dim3(kThreads), smem, s, a);
}
template <int G, int MODE>
cudaError_t launch(bool bwd, int n, const Args& a, cudaStream_t s) {
  const int of_step = n * (32 / G);
  const bool full = a.dim == 8 * G && a.heads_q % of_step == 0 && a.heads_k % of_step == 0;  // no place of any step is empty
  if (n == 2) return full ? launch<G, MODE, 2, true>(bwd, a, s) : launch<G, MODE, 2, false>(bwd, a, s);
  return full ? launch<G, MODE, 1, true>(bwd, a, s) : launch<G, MODE, 1, false>(bwd, a, s);
}
template <int G>
cudaError_t launch(bool bwd, bool interleaved, int n, const Args& a, cudaStream_t s) {
  if (a.half == 0) return launch<G, kPlain>(bwd, n, a, s);
  return interleaved ? launch<G, kNeighbours>(bwd, n, a, s) : launch<G, kHalves>(bwd, n, a, s);
}
cudaError_t launch(bool bwd, bool interleaved, int n, const Args& a, cudaStream_t s) {
  cudaError_t e;
  switch (lanes_of(a.dim)) {
    case 4: e = launch<4>(bwd, interleaved, n, a, s); break;
    case 8: e = launch<8>(bwd, interleaved, n, a, s); break;
    case 16: e = launch<16>(bwd, interleaved, n, a, s); break;
    default: e = launch<32>(bwd, interleaved, n, a, s); break;
  }
  count_launch();
  return e;
}

}  // namespace

cudaError_t launch_headnorm_fwd(const Heads& h, cudaStream_t s) {
  const int n = heads_of_lane(h.heads_q, h.heads_k, h.dim);
  return launch(false, h.interleaved, n, args_of(h, n), s);
}

int64_t headnorm_bwd_workspace_floats(int64_t rows, int heads_q, int heads_k, int dim) {
  return (int64_t)ctas_of(rows * steps_of_row(heads_q, heads_k, dim, heads_of_lane(heads_q, heads_k, dim)), kBwdCtas) * 2 * dim;
}

cudaError_t launch_headnorm_bwd(const Heads& h, cudaStream_t s) {
  const int n = heads_of_lane(h.heads_q, h.heads_k, h.dim);
  Args a = args_of(h, n);
  const bool sums = h.dgain_q || h.dgain_k;
  a.joined = sums && is_joined(a.steps);
  a.partial = sums && !a.joined ? h.workspace : nullptr;
  a.dgain_q = h.dgain_q; a.dgain_k = h.dgain_k;
  a.accumulate = h.accumulate;
  const cudaError_t e = launch(true, h.interleaved, n, a, s);
  if (e != cudaSuccess || !a.partial) return e;
  return launch_column_sums(h.workspace, ctas_of(a.steps, kBwdCtas), 2 * h.dim, h.dgain_q, h.accumulate, s, h.dgain_k, h.dim);
}

}  // namespace nvfp4

// Log probabilities of given tokens with entropy and the likeliest alternatives, and their gradient.
//   z = scale logit;  lse = ln sum e^z;  log p = z - lse;  H = - sum p log p
//   gradient by a logit  scale (dlogprob ((j == target) - p) - dentropy p (log p + H))
// Bound by HBM: the forward pass reads a row once, with the running maximum and the sums of e^(z - m) and (z - m) e^(z - m) in registers; the
// gradient reads it once more and writes.  Differences from the maximum are taken of the logits before they are scaled: a row of the type's
// lowest values keeps its distribution, and minus infinity gives e^z = 0 whatever stands beside it.
#include <algorithm>

#include "around.h"
#include "copy8.cuh"
#include "ends.h"

namespace nvfp4 {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kMaxCluster = 8;
constexpr int kRing = 5, kStage = kThreads * 32;  // what is on its way to a CTA: 32 bytes a thread and stage
constexpr int kShortRow = 4096;                   // up to here a warp takes a row by itself
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f, kLowest = -3.402823466e38f, kFar = -300.f;

__device__ __forceinline__ float exp2_fast(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float minus_infinity() { return __uint_as_float(0xff800000u); }

// Whole numbers in the order of the values (both zeros are one), and keys in the order (value, lower index first)
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_ordered(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ uint64_t key_of(float v, uint32_t index) { return ((uint64_t)ordered(v) << 32) | (uint32_t)~index; }

struct Fwd {
  const void* logits;
  Indices targets;
  float* logprob;
  float* lse;
  float2* stats;
  float* entropy;
  int* top_ids;
  float* top_logprobs;
  int64_t rows, vocab, ld;
  float scale;
  int top;
};

// What a lane holds of its elements: the largest logit m (minus infinity: none), and for d = (x - max(m, lowest)) scale in powers of two the sums of 2^d and d 2^d
template <bool ENTROPY>
struct Running {
  float m;
  float2 s, t;
  __device__ __forceinline__ Running() : m(minus_infinity()), s(make_float2(0.f, 0.f)), t(make_float2(0.f, 0.f)) {}
  __device__ __forceinline__ float base() const { return fmaxf(m, kLowest); }
  // the sums as those of differences from a larger maximum
  __device__ __forceinline__ void raise(float to, float per) {
    const float d = (base() - to) * per, f = exp2_fast(d);
    if (ENTROPY) t = mul2(fma2(both(fmaxf(d, kFar)), s, t), both(f));  // (f is 0 below)
    s = mul2(s, both(f));
  }
  template <int N>
  __device__ __forceinline__ void add(const float2 (&v)[N], float largest, float per) {
    if (largest > m) {
      raise(fmaxf(largest, kLowest), per);
      m = largest;
    }
    const float b = base();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float2 d = mul2(sub2(v[i], both(b)), both(per));
      const float2 e = make_float2(exp2_fast(d.x), exp2_fast(d.y));
      s = add2(s, e);
      if (ENTROPY) t = fma2(e, make_float2(fmaxf(d.x, kFar), fmaxf(d.y, kFar)), t);
    }
  }
};

template <bool F32>
__device__ __forceinline__ float logit_at(const void* logits, int64_t at) {
  return F32 ? static_cast<const float*>(logits)[at] : bf16_lo(static_cast<const uint16_t*>(logits)[at]);
}
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 r = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// Sixteen bytes of a row: eight or four neighbouring logits
template <bool F32>
struct Chunk {
  static constexpr int E = F32 ? 4 : 8, kPairs = E / 2;
  uint4 w;
  __device__ __forceinline__ void nothing() { w.x = w.y = w.z = w.w = F32 ? 0xff800000u : 0xff80ff80u; }  // minus infinities
  __device__ __forceinline__ void load(const void* row, int64_t c) { w = ldg128_stream(static_cast<const uint8_t*>(row) + c * 16); }
  __device__ __forceinline__ void values(float2* v) const {
    if (F32) {
      v[0] = make_float2(__uint_as_float(w.x), __uint_as_float(w.y));
      v[1] = make_float2(__uint_as_float(w.z), __uint_as_float(w.w));
    } else {
      v[0] = make_float2(bf16_lo(w.x), bf16_hi(w.x));
      v[1] = make_float2(bf16_lo(w.y), bf16_hi(w.y));
      v[2] = make_float2(bf16_lo(w.z), bf16_hi(w.z));
      v[3] = make_float2(bf16_lo(w.w), bf16_hi(w.w));
    }
  }
  __device__ __forceinline__ float largest() const {
    if (F32) return fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
    const uint32_t m = max_bf16x2(max_bf16x2(w.x, w.y), max_bf16x2(w.z, w.w));
    return fmaxf(bf16_lo(m), bf16_hi(m));
  }
};

// A row belongs to a group of W warps
template <int W>
__device__ __forceinline__ void group_sync() {
  if (W == 1) __syncwarp(); else __syncthreads();
}
template <int W>
struct TopShared {
  static constexpr int kCandidates = W == 1 ? 256 : 2048;  // places for elements that may be among the likeliest
  uint64_t keys[kCandidates];
  uint64_t best[32];  // the group's likeliest, in order
  uint32_t top_of_thread[32 * W];
  uint64_t least;
  int count, asked;
  uint16_t asks[32 * W];  // threads whose elements are read again
};

// The likeliest of a group's share of a row.  Among the threads' maxima the top-th largest is no larger than the top-th largest element, so
// that only the few threads whose maximum reaches it have elements to offer, and those are read once more.  Where too many offer (equal
// values), the bound is raised to the top-th of those that found room, which is exact in (value, index), and the threads are asked again.
template <bool F32, int W>
__device__ void select_top(const Fwd& a, TopShared<W>& sh, const void* row, float m, int64_t c0, int64_t c1, int64_t whole, int want) {
  constexpr int E = Chunk<F32>::E, T = 32 * W, kCandidates = TopShared<W>::kCandidates;
  const int tid = threadIdx.x % T, lane = tid & 31;
  sh.top_of_thread[tid] = ordered(m);
  group_sync<W>();
  if (tid < 32) {
    uint32_t k[W], bound = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) k[i] = sh.top_of_thread[32 * i + lane];
    for (int bit = 31; bit >= (F32 ? 0 : 16); --bit) {  // (the lower half of a bf16 number's order is that of its sign)
      const uint32_t trial = bound | (1u << bit);
      int n = 0;
#pragma unroll
      for (int i = 0; i < W; ++i) n += k[i] >= trial;
      if (__reduce_add_sync(0xffffffffu, n) >= want) bound = trial;
    }
    if (lane == 0) sh.least = bound <= ordered(minus_infinity()) ? 0ull : (uint64_t)bound << 32;
  }
  const int per = (int)((c1 - c0 + T - 1) / T);  // chunks of a thread, but for some threads' last one
  while (true) {
    if (tid == 0) sh.count = sh.asked = 0;
    group_sync<W>();
    const uint64_t least = sh.least;
    if (ordered(m) >= (uint32_t)(least >> 32)) sh.asks[atomicAdd(&sh.asked, 1)] = (uint16_t)tid;
    group_sync<W>();
    // all threads read the chunks of those that are asked, the first ones first, until there are too many candidates
    const int asked = sh.asked;
    const volatile int* const so_far = &sh.count;
#pragma unroll 4
    for (int64_t p = tid; p < (int64_t)asked * per && *so_far <= kCandidates; p += T) {
      const int turn = (int)(p / asked);
      const int64_t c = c0 + (int64_t)turn * T + sh.asks[p - (int64_t)turn * asked];
      if (c >= c1) continue;
      float2 v[E / 2];
      if (c < whole) {
        Chunk<F32> r;
        r.load(row, c);
        r.values(v);
      } else {
        for (int j = 0; j < E; ++j) (j % 2 ? v[j / 2].y : v[j / 2].x) = c * E + j < a.vocab ? logit_at<F32>(row, c * E + j) : 0.f;
      }
#pragma unroll
      for (int j = 0; j < E; ++j) {
        const uint64_t key = key_of(j % 2 ? v[j / 2].y : v[j / 2].x, (uint32_t)(c * E + j));
        if (key >= least && c * E + j < a.vocab) {
          const int at = atomicAdd(&sh.count, 1);
          if (at < kCandidates) sh.keys[at] = key;
        }
      }
    }
    group_sync<W>();
    const int count = sh.count, held = min(count, kCandidates);
    for (int i = tid; i < held; i += T) {
      const uint64_t key = sh.keys[i];
      int larger = 0;
#pragma unroll 8
      for (int j = 0; j < held; ++j) larger += sh.keys[j] > key;
      if (larger < want) sh.best[larger] = key;
    }
    group_sync<W>();
    if (count <= kCandidates) return;
    if (tid == 0) sh.least = sh.best[want - 1];
    // (read behind the next barrier)
  }
}

struct Partial {
  float m, s, t;
};

// W warps to a row: one (up to kShortRow columns; a CTA has kWarps rows), or a CTA, or a cluster of gridDim.y CTAs, each with a run of the row's
// sixteen-byte chunks, whose findings the first one joins.
template <bool F32, bool ENTROPY, bool TOP, int W>
__global__ void __launch_bounds__(kThreads, 4) logprob_fwd_kernel(const Fwd a) {
  constexpr int T = 32 * W, E = Chunk<F32>::E, kChunks = 2;  // of a stage
  __shared__ Partial of_warp[kWarps], of_cta;
  extern __shared__ __align__(16) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tid = threadIdx.x % T;
  TopShared<W>& sh = reinterpret_cast<TopShared<W>*>(smem + kRing * kStage)[threadIdx.x / T];
  griddep_wait();
  griddep_launch_dependents();
  const int64_t row = W == 1 ? (int64_t)blockIdx.x * kWarps + warp : blockIdx.x;
  if (W == 1 && row >= a.rows) return;
  const unsigned parts = W == 1 ? 1u : gridDim.y, part = W == 1 ? 0u : blockIdx.y;
  const uint8_t* const x = static_cast<const uint8_t*>(a.logits) + row * a.ld * (F32 ? 4 : 2);
  const int64_t whole = a.vocab / E, chunks = (a.vocab + E - 1) / E;
  const int64_t c0 = chunks * part / parts, c1 = chunks * (part + 1) / parts, full = min(c1, whole);
  const float per = a.scale * kLog2e;
  Running<ENTROPY> run;
  // the row comes through a ring in which every thread has places of its own
  const uint32_t mine = smem_u32(smem) + threadIdx.x * 16;
  int64_t ahead = c0 + tid;
  auto fetch = [&](int slot) {
#pragma unroll
    for (int u = 0; u < kChunks; ++u, ahead += T)
      if (ahead < full) copy_async<16>(mine + slot * kStage + u * (kThreads * 16), x + ahead * 16, true);
    copy_commit();  // (an empty group where there is no chunk: the count of groups stays that of the stages)
  };
#pragma unroll
  for (int u = 0; u < kRing - 1; ++u) fetch(u);
  int slot = 0, next = kRing - 1;
  for (int64_t c = c0 + tid; c < full; c += T * kChunks) {
    copy_wait<kRing - 2>();
    Chunk<F32> raw[kChunks];
#pragma unroll
    for (int u = 0; u < kChunks; ++u) {
      raw[u].w = lds16(mine + slot * kStage + u * (kThreads * 16));
      if (u > 0 && c + u * T >= full) raw[u].nothing();
    }
    fetch(next);  // the slot of the stage before, whose values went into registers a turn ago
    slot = slot + 1 == kRing ? 0 : slot + 1;
    next = next + 1 == kRing ? 0 : next + 1;
    float2 v[kChunks * E / 2];
    float largest = minus_infinity();
#pragma unroll
    for (int u = 0; u < kChunks; ++u) {
      raw[u].values(v + u * (E / 2));
      largest = fmaxf(largest, raw[u].largest());
    }
    run.add(v, largest, per);
  }
  copy_wait<0>();
  if (c1 > whole && tid == (int)((whole - c0) % T)) {  // a last chunk that is not full, to the thread whose turn it is
    for (int64_t j = whole * E; j < a.vocab; ++j) {
      const float2 v[1] = {make_float2(logit_at<F32>(x, j), minus_infinity())};
      run.add(v, v[0].x, per);
    }
  }
  const float own = run.m;
  // the group's maximum, then sums of differences from it
  float m = own;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (W > 1) {
    if (lane == 0) of_warp[warp].m = m;
    __syncthreads();
    m = of_warp[lane % kWarps].m;
#pragma unroll
    for (int o = kWarps / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  }
  run.raise(fmaxf(m, kLowest), per);
  float s = run.s.x + run.s.y, t = run.t.x + run.t.y;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    s += __shfl_xor_sync(0xffffffffu, s, o);
    if (ENTROPY) t += __shfl_xor_sync(0xffffffffu, t, o);
  }
  if (W > 1) {
    if (lane == 0) {
      of_warp[warp].s = s;
      of_warp[warp].t = t;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 1; w < kWarps; ++w) {
        s += of_warp[w].s;
        t += of_warp[w].t;
      }
      of_cta = Partial{m, s, t};
    }
  }
  // (top is at most vocab, and a part of a cluster has more columns than any top)
  if (TOP) select_top<F32, W>(a, sh, x, own, c0, c1, whole, a.top);
  if (W > 1) {
    if (parts > 1) cluster_sync(); else __syncthreads();
  }
  if (part == 0) {
    if (W > 1) {
      m = of_cta.m;
      s = of_cta.s;
      t = of_cta.t;
      if (parts > 1) {
        for (uint32_t r = 1; r < parts; ++r) m = fmaxf(m, ld_of_rank(&of_cta.m, r));
        s = t = 0.f;
        for (uint32_t r = 0; r < parts; ++r) {
          const float d = (fmaxf(ld_of_rank(&of_cta.m, r), kLowest) - fmaxf(m, kLowest)) * per, f = exp2_fast(d), sr = ld_of_rank(&of_cta.s, r);
          s += f * sr;
          if (ENTROPY) t += f * fmaf(fmaxf(d, kFar), sr, ld_of_rank(&of_cta.t, r));
        }
      }
    }
    const float base = fmaxf(m, kLowest), log_total = logf(s);
    if (tid == 0) {
      if (a.lse) a.lse[row] = fmaf(base, a.scale, log_total);
      if (a.stats) a.stats[row] = make_float2(m, log_total);
      if (a.entropy) a.entropy[row] = s == 0.f ? 0.f : log_total - kLn2 * (t / s);
      if (a.logprob) {
        const int64_t target = a.targets[row];
        a.logprob[row] = target < 0 || target >= a.vocab ? 0.f : s == 0.f ? minus_infinity() : (logit_at<F32>(x, target) - base) * a.scale - log_total;
      }
    }
    if (TOP) {
      auto put = [&](int place, uint64_t key) {
        if (a.top_ids) a.top_ids[row * a.top + place] = (int)~(uint32_t)key;
        if (a.top_logprobs)
          a.top_logprobs[row * a.top + place] = s == 0.f ? minus_infinity() : (of_ordered((uint32_t)(key >> 32)) - base) * a.scale - log_total;
      };
      if (parts == 1) {
        if (tid < a.top) put(tid, sh.best[tid]);
      } else {  // the CTAs' likeliest ones in one order: a key's place is the number of larger ones
        const int all = a.top * (int)parts;
        for (int i = tid; i < all; i += T) {
          const uint32_t r = i / a.top;
          const float* const p = reinterpret_cast<const float*>(&sh.best[i - r * a.top]);
          sh.keys[i] = ((uint64_t)__float_as_uint(ld_of_rank(p + 1, r)) << 32) | __float_as_uint(ld_of_rank(p, r));
        }
        group_sync<W>();
        for (int i = tid; i < all; i += T) {
          const uint64_t key = sh.keys[i];
          int larger = 0;
#pragma unroll 8
          for (int j = 0; j < all; ++j) larger += sh.keys[j] > key;
          if (larger < a.top) put(larger, key);
        }
      }
    }
  }
  if (W > 1 && parts > 1) cluster_sync();  // none may go while it is read
}

struct Bwd {
  const void* logits;
  Indices targets;
  const float2* stats;
  const float* entropy;
  const float* dlogprob;
  const float* dentropy;
  void* dlogits;
  int64_t rows, vocab, ld, lddl, dcols, steps, per_row;
  float scale;
};
constexpr int kBwdCtas = 148 * 4, kBwdSteps = 32;  // as many as are resident; steps of a warp where there are more

// Four or eight neighbours
template <bool OUT32, int P>
__device__ __forceinline__ void put(void* out, int64_t at, const float2 (&v)[P]) {
  if (OUT32) {
#pragma unroll
    for (int j = 0; j < P; j += 2) *reinterpret_cast<float4*>(static_cast<float*>(out) + at + 2 * j) = make_float4(v[j].x, v[j].y, v[j + 1].x, v[j + 1].y);
  } else if (P == 4) {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(out) + at) =
        make_uint4(pack2(v[0].x, v[0].y), pack2(v[1].x, v[1].y), pack2(v[P - 2].x, v[P - 2].y), pack2(v[P - 1].x, v[P - 1].y));
  } else {
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + at) = make_uint2(pack2(v[0].x, v[0].y), pack2(v[1].x, v[1].y));
  }
}

// What a row's gradient is made of: p = 2^(d per - total) with d = x - top, and the gradient p (a + b log2 p), with `hit` more at the target
struct RowGrad {
  float top, total, a, b, hit;
  int64_t target;
  template <bool ENTROPY>
  __device__ __forceinline__ void load(const Bwd& g, int64_t row) {
    const float2 st = g.stats[row];
    const int64_t t = g.targets.p ? g.targets[row] : -1;
    const float w = g.dlogprob ? g.dlogprob[row] * g.scale : 0.f, e = ENTROPY ? g.dentropy[row] * g.scale : 0.f, h = ENTROPY ? g.entropy[row] : 0.f;
    const bool empty = st.x == minus_infinity(), there = t >= 0 && t < g.vocab && !empty;
    top = empty ? 0.f : st.x;  // (all of an empty row is p = 0 then)
    total = empty ? 0.f : st.y * kLog2e;
    hit = there ? w : 0.f;
    a = -fmaf(e, h, hit);
    b = -e * kLn2;
    target = there ? t : -1;
  }
};

// Every warp takes an equal share of all rows' steps of 32 chunks, 32 steps (16 KB) where there are enough for all: CTAs that end and make room for the
// next ones keep to neighbouring memory, resident ones that go through long shares drift apart (8192 x 131072: 592 CTAs 760 us, 9472 640 us; 1003
// x 50257 in binary32 with 592 / 1184 / 2368 / 9472 69 / 69 / 66 / 86); the logits come through a ring as in the forward pass, and a row's
// numbers while the one before is worked on.
template <bool F32, bool OUT32, bool ENTROPY>
__global__ void __launch_bounds__(kThreads, 4) logprob_bwd_kernel(const Bwd a) {
  constexpr int E = Chunk<F32>::E, kSlots = kRing * 2, kSlot = kThreads * 16;
  extern __shared__ __align__(16) uint8_t smem[];
  const int lane = threadIdx.x & 31;
  const int64_t warps = (int64_t)gridDim.x * kWarps, w = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int64_t first = a.steps * w / warps, steps = a.steps * (w + 1) / warps - first, whole = a.vocab / E;
  const uint32_t mine = smem_u32(smem) + threadIdx.x * 16;
  int64_t row = first / a.per_row, c = (first - row * a.per_row) * 32 + lane;  // a lane's chunk
  int64_t ahead_row = row, ahead = c, fetched = 0;
  const uint8_t* const x = static_cast<const uint8_t*>(a.logits);
  auto fetch = [&](int slot) {
    if (fetched < steps) {
      if (ahead < whole) copy_async<16>(mine + slot * kSlot, x + ahead_row * a.ld * (F32 ? 4 : 2) + ahead * 16, true);
      ++fetched;
      ahead += 32;
      if (ahead >= a.per_row * 32) {
        ahead = lane;
        ++ahead_row;
      }
    }
    copy_commit();
  };
  griddep_wait();
  griddep_launch_dependents();
  if (steps == 0) return;
#pragma unroll
  for (int u = 0; u < kSlots - 1; ++u) fetch(u);
  int slot = 0, next = kSlots - 1;
  RowGrad now, then;
  now.load<ENTROPY>(a, row);
  then = now;
  if (row + 1 < a.rows) then.load<ENTROPY>(a, row + 1);
  const float per = a.scale * kLog2e;
  auto grad = [&](float2 v) {
    const float2 l = fma2(sub2(v, both(now.top)), both(per), both(-now.total)), p = make_float2(exp2_fast(l.x), exp2_fast(l.y));
    if (!ENTROPY) return mul2(p, both(now.a));
    return mul2(p, fma2(make_float2(fmaxf(l.x, kFar), fmaxf(l.y, kFar)), both(now.b), both(now.a)));  // (p is 0 below)
  };
  for (int64_t i = 0; i < steps; ++i) {
    copy_wait<kSlots - 2>();
    if (c < whole) {
      Chunk<F32> raw;
      raw.w = lds16(mine + slot * kSlot);
      float2 v[E / 2];
      raw.values(v);
#pragma unroll
      for (int j = 0; j < E / 2; ++j) v[j] = grad(v[j]);
      if (c == now.target / E && now.target >= 0) {
        const int at = (int)(now.target % E);
#pragma unroll
        for (int j = 0; j < E / 2; ++j) {
          if (at == 2 * j) v[j].x += now.hit;
          if (at == 2 * j + 1) v[j].y += now.hit;
        }
      }
      put<OUT32>(a.dlogits, row * a.lddl + c * E, v);
    } else {  // what is left of the columns, and zeros behind them
      for (int64_t j = c * E; j < min(c * E + E, a.dcols); ++j) {
        float g = 0.f;
        if (j < a.vocab) g = grad(both(logit_at<F32>(x, row * a.ld + j))).x + (j == now.target ? now.hit : 0.f);
        if (OUT32)
          static_cast<float*>(a.dlogits)[row * a.lddl + j] = g;
        else
          static_cast<__nv_bfloat16*>(a.dlogits)[row * a.lddl + j] = __float2bfloat16_rn(g);
      }
    }
    fetch(next);
    slot = slot + 1 == kSlots ? 0 : slot + 1;
    next = next + 1 == kSlots ? 0 : next + 1;
    c += 32;
    if (c >= a.per_row * 32) {
      c = lane;
      ++row;
      now = then;
      if (i + 1 < steps && row + 1 < a.rows) then.load<ENTROPY>(a, row + 1);
    }
  }
  copy_wait<0>();
}

// CTAs of a row: enough that every SM has one
unsigned cluster_of(int64_t rows, int64_t vocab) {
  unsigned n = 1;
  while (n < kMaxCluster && rows * n < 148 && vocab / (2 * n) >= 8 * kThreads) n *= 2;
  return n;
}

template <typename K>
cudaError_t configure(K kern, size_t smem, std::atomic<uint64_t>& configured) {
  int dev;
  if (!device_needs_config(configured, &dev)) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e == cudaSuccess) device_configured(configured, dev);
  return e;
}

template <bool F32, bool ENTROPY, bool TOP, int W>
cudaError_t launch_fwd(const Fwd& a, unsigned ctas, cudaStream_t s) {
  const auto kern = logprob_fwd_kernel<F32, ENTROPY, TOP, W>;
  constexpr size_t smem = kRing * kStage + (TOP ? sizeof(TopShared<W>) * (kWarps / W) : 0);
  static std::atomic<uint64_t> configured{0};  // per instantiation and device
  const cudaError_t e = configure(kern, smem, configured);
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)(W == 1 ? (a.rows + kWarps - 1) / kWarps : a.rows), ctas);
  return ctas > 1 ? launch_cluster(ctas, kern, grid, dim3(kThreads), smem, s, a) : launch_divided(100, kern, grid, dim3(kThreads), smem, s, a);
}
template <bool F32, bool ENTROPY, bool TOP>
cudaError_t launch_fwd(const Fwd& a, cudaStream_t s) {
  if (a.vocab <= kShortRow) return launch_fwd<F32, ENTROPY, TOP, 1>(a, 1, s);
  return launch_fwd<F32, ENTROPY, TOP, kWarps>(a, cluster_of(a.rows, a.vocab), s);
}
template <bool F32, bool OUT32>
cudaError_t launch_bwd(const Bwd& a, cudaStream_t s) {
  const unsigned ctas = (unsigned)std::max<int64_t>(a.steps / (kWarps * kBwdSteps), std::min<int64_t>((a.steps + kWarps - 1) / kWarps, kBwdCtas));
  const auto kern = a.dentropy ? logprob_bwd_kernel<F32, OUT32, true> : logprob_bwd_kernel<F32, OUT32, false>;
  return launch_divided(100, kern, dim3(ctas), dim3(kThreads), kRing * kStage, s, a);
}

}  // namespace

cudaError_t launch_logprob_fwd(const Logprob& l, cudaStream_t s) {
  Fwd a{};
  a.logits = l.logits;
  a.targets = l.targets;
  a.logprob = l.logprob; a.lse = l.lse; a.entropy = l.entropy;
  a.stats = reinterpret_cast<float2*>(l.stats);
  a.top_ids = l.top_ids; a.top_logprobs = l.top_logprobs;
  a.rows = l.rows; a.vocab = l.vocab; a.ld = l.ld;
  a.scale = l.scale;
  a.top = l.top;
  const bool top = l.top_ids || l.top_logprobs;
  cudaError_t e;
  if (l.fp32)
    e = l.entropy ? (top ? launch_fwd<true, true, true>(a, s) : launch_fwd<true, true, false>(a, s))
                  : (top ? launch_fwd<true, false, true>(a, s) : launch_fwd<true, false, false>(a, s));
  else
    e = l.entropy ? (top ? launch_fwd<false, true, true>(a, s) : launch_fwd<false, true, false>(a, s))
                  : (top ? launch_fwd<false, false, true>(a, s) : launch_fwd<false, false, false>(a, s));
  count_launch();
  return e;
}

cudaError_t launch_logprob_bwd(const Logprob& l, cudaStream_t s) {
  Bwd a{};
  a.logits = l.logits;
  a.targets = l.targets;
  a.stats = reinterpret_cast<const float2*>(l.stats); a.entropy = l.entropy;
  a.dlogprob = l.dlogprob; a.dentropy = l.dentropy;
  a.dlogits = l.dlogits;
  a.rows = l.rows; a.vocab = l.vocab; a.ld = l.ld; a.lddl = l.lddl; a.dcols = l.dcols;
  const int of_step = 32 * (l.fp32 ? Chunk<true>::E : Chunk<false>::E);
  a.per_row = (l.dcols + of_step - 1) / of_step;
  a.steps = l.rows * a.per_row;
  a.scale = l.scale;
  const cudaError_t e = l.fp32 ? (l.out_fp32 ? launch_bwd<true, true>(a, s) : launch_bwd<true, false>(a, s))
                               : (l.out_fp32 ? launch_bwd<false, true>(a, s) : launch_bwd<false, false>(a, s));
  count_launch();
  return e;
}

}  // namespace nvfp4

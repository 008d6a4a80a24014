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

constexpr int kThreads = 512, kWarps = kThreads / 32, kMaxCluster = 8;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f, kLowest = -3.402823466e38f;
constexpr int kCandidates = 2048;  // places for elements that may be among the likeliest

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

struct TopShared {
  uint64_t keys[kCandidates];
  uint64_t best[32];  // the CTA's likeliest, in order
  uint32_t top_of_thread[kThreads];
  uint64_t least;
  int count;
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
    if (ENTROPY) {
      const float far = fmaxf(d, -200.f);  // (f is 0 there)
      t = mul2(fma2(both(far), s, t), both(f));
    }
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
      if (ENTROPY) t = fma2(e, make_float2(fmaxf(d.x, -200.f), fmaxf(d.y, -200.f)), t);
    }
  }
};

template <bool F32>
__device__ __forceinline__ float logit_at(const void* logits, int64_t at) {
  return F32 ? static_cast<const float*>(logits)[at] : bf16_lo(static_cast<const uint16_t*>(logits)[at]);
}

// The likeliest of a CTA's share of a row.  Among the threads' maxima the top-th largest is no larger than the top-th largest element, so
// that only the few threads whose maximum reaches it have elements to offer; their warps read those once more.  Where too many offer (equal
// values), the bound is raised to the top-th of those that found room, which is exact in (value, index), and the threads are asked again.
template <bool F32>
__device__ void select_top(const Fwd& a, TopShared& sh, const void* row, float m, int64_t c0, int64_t c1, int64_t n8, int want) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  sh.top_of_thread[threadIdx.x] = ordered(m);
  __syncthreads();
  if (warp == 0) {
    uint32_t k[kWarps], bound = 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) k[i] = sh.top_of_thread[32 * i + lane];
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t trial = bound | (1u << bit);
      int n = 0;
#pragma unroll
      for (int i = 0; i < kWarps; ++i) n += k[i] >= trial;
      if (__reduce_add_sync(0xffffffffu, n) >= want) bound = trial;
    }
    if (lane == 0) sh.least = bound <= ordered(minus_infinity()) ? 0ull : (uint64_t)bound << 32;
  }
  while (true) {
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    const uint64_t least = sh.least;
    const bool offers = ordered(m) >= (uint32_t)(least >> 32);
    uint32_t asked = __ballot_sync(0xffffffffu, offers);
    const volatile int* const so_far = &sh.count;
    auto offer = [&](int64_t c) {
      float v[8];
      if (c < n8) {
        Raw8<F32> r;
        r.load(row, c * 8);
        r.values(v);
      } else {
        for (int j = 0; j < 8; ++j) v[j] = c * 8 + j < a.vocab ? logit_at<F32>(row, c * 8 + j) : 0.f;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint64_t key = key_of(v[j], (uint32_t)(c * 8 + j));
        if (key >= least && c * 8 + j < a.vocab) {
          const int at = atomicAdd(&sh.count, 1);
          if (at < kCandidates) sh.keys[at] = key;
        }
      }
    };
    if (__popc(asked) > 4) {  // every lane its own chunks
      if (offers)
#pragma unroll 4
        for (int64_t c = c0 + threadIdx.x; c < c1 && *so_far <= kCandidates; c += kThreads) offer(c);
    } else {  // the lanes one after the other, a chunk to every lane
      for (; asked; asked &= asked - 1)
        for (int64_t c = c0 + warp * 32 + __ffs(asked) - 1 + (int64_t)lane * kThreads; c < c1; c += 32 * kThreads) offer(c);
    }
    __syncthreads();
    const int count = sh.count, held = min(count, kCandidates);
    for (int i = threadIdx.x; i < held; i += kThreads) {
      const uint64_t key = sh.keys[i];
      int larger = 0;
      for (int j = 0; j < held; ++j) larger += sh.keys[j] > key;
      if (larger < want) sh.best[larger] = key;
    }
    __syncthreads();
    if (count <= kCandidates) return;
    if (threadIdx.x == 0) sh.least = sh.best[want - 1];
    // (read behind the next barrier)
  }
}

struct Partial {
  float m, s, t;
};

// A row to a cluster of gridDim.y CTAs.  Every CTA takes a run of the row's chunks of eight; the first one joins what they found.
template <bool F32, bool ENTROPY, bool TOP>
__global__ void __launch_bounds__(kThreads, 2) logprob_fwd_kernel(const Fwd a) {
  constexpr int kAhead = F32 ? 2 : 4;
  __shared__ Partial of_warp[kWarps], of_cta;
  extern __shared__ __align__(16) uint8_t smem[];
  TopShared& sh = *reinterpret_cast<TopShared*>(smem);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  griddep_wait();
  griddep_launch_dependents();
  const int64_t row = blockIdx.x;
  const void* const x = static_cast<const uint8_t*>(a.logits) + row * a.ld * (F32 ? 4 : 2);
  const int64_t n8 = a.vocab >> 3, chunks = (a.vocab + 7) >> 3;
  const int64_t c0 = chunks * blockIdx.y / gridDim.y, c1 = chunks * (blockIdx.y + 1) / gridDim.y, full = min(c1, n8);
  const float per = a.scale * kLog2e;
  Running<ENTROPY> run;
  for (int64_t c = c0 + threadIdx.x; c < full; c += kThreads * kAhead) {
    Raw8<F32> raw[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (c + u * kThreads < full) {
        raw[u].load(x, (c + u * kThreads) * 8);
      } else {
#pragma unroll
        for (int i = 0; i < (F32 ? 2 : 1); ++i) raw[u].w[i] = F32 ? make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u)
                                                                  : make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u);
      }
    }
    float2 v[kAhead * 4];
    float largest = minus_infinity();
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      float2 w[4];
      values2(raw[u], w);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[u * 4 + i] = w[i];
        largest = fmaxf(largest, fmaxf(w[i].x, w[i].y));
      }
    }
    run.add(v, largest, per);
  }
  if (c1 > n8 && threadIdx.x == (unsigned)((n8 - c0) % kThreads)) {  // a last chunk that is not full, to the thread whose turn it is
    for (int64_t j = n8 * 8; j < a.vocab; ++j) {
      const float2 v[1] = {make_float2(logit_at<F32>(x, j), minus_infinity())};
      run.add(v, v[0].x, per);
    }
  }
  const float own = run.m;
  // the CTA's maximum, then sums of differences from it
  float m = own;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (lane == 0) of_warp[warp].m = m;
  __syncthreads();
  m = of_warp[lane % kWarps].m;
#pragma unroll
  for (int o = kWarps / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  run.raise(fmaxf(m, kLowest), per);
  float s = run.s.x + run.s.y, t = run.t.x + run.t.y;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    s += __shfl_xor_sync(0xffffffffu, s, o);
    if (ENTROPY) t += __shfl_xor_sync(0xffffffffu, t, o);
  }
  if (lane == 0) {
    of_warp[warp].s = s;
    of_warp[warp].t = t;
  }
  __syncthreads();
  const int want = TOP ? (int)min((int64_t)a.top, min(c1 * 8, a.vocab) - c0 * 8) : 0;
  if (threadIdx.x == 0) {
    for (int w = 1; w < kWarps; ++w) {
      s += of_warp[w].s;
      t += of_warp[w].t;
    }
    of_cta = Partial{m, s, t};
  }
  if (TOP && want > 0) select_top<F32>(a, sh, x, own, c0, c1, n8, want);
  if (gridDim.y > 1) cluster_sync(); else __syncthreads();
  if (blockIdx.y == 0) {
    float total = of_cta.s, weighted = of_cta.t;
    m = of_cta.m;
    if (gridDim.y > 1) {
      for (uint32_t r = 1; r < gridDim.y; ++r) m = fmaxf(m, ld_of_rank(&of_cta.m, r));
      total = weighted = 0.f;
      for (uint32_t r = 0; r < gridDim.y; ++r) {
        const float d = (fmaxf(ld_of_rank(&of_cta.m, r), kLowest) - fmaxf(m, kLowest)) * per, f = exp2_fast(d), sr = ld_of_rank(&of_cta.s, r);
        total += f * sr;
        if (ENTROPY) weighted += f * fmaf(fmaxf(d, -200.f), sr, ld_of_rank(&of_cta.t, r));
      }
    }
    const float base = fmaxf(m, kLowest), log_total = logf(total);
    if (threadIdx.x == 0) {
      if (a.lse) a.lse[row] = fmaf(base, a.scale, log_total);
      if (a.stats) a.stats[row] = make_float2(m, log_total);
      if (a.entropy) a.entropy[row] = total == 0.f ? 0.f : log_total - kLn2 * (weighted / total);
      if (a.logprob) {
        const int64_t target = a.targets[row];
        a.logprob[row] = target < 0 || target >= a.vocab ? 0.f : total == 0.f ? minus_infinity()
                                                                 : (logit_at<F32>(x, target) - base) * a.scale - log_total;
      }
    }
    if (TOP) {
      // the CTAs' likeliest ones in one order: a key's place is the number of larger ones
      const int of_each = a.top, all = of_each * (int)gridDim.y;
      auto key_at = [&](int i) {
        const uint32_t r = i / of_each;
        const int k = i - (int)r * of_each;
        const int64_t b = chunks * r / gridDim.y * 8, e = min(chunks * (r + 1) / gridDim.y * 8, a.vocab);
        if (k >= e - b) return (uint64_t)0;
        const float* const p = reinterpret_cast<const float*>(&sh.best[k]);
        return ((uint64_t)__float_as_uint(ld_of_rank(p + 1, r)) << 32) | __float_as_uint(ld_of_rank(p, r));
      };
      if (gridDim.y > 1) {
        for (int i = threadIdx.x; i < all; i += kThreads) sh.keys[i] = key_at(i);
        __syncthreads();
      } else {
        for (int i = threadIdx.x; i < all; i += kThreads) sh.keys[i] = sh.best[i];
        __syncthreads();
      }
      for (int i = threadIdx.x; i < all; i += kThreads) {
        const uint64_t key = sh.keys[i];
        int larger = 0;
        for (int j = 0; j < all; ++j) larger += sh.keys[j] > key;
        if (key != 0 && larger < a.top) {
          const float v = of_ordered((uint32_t)(key >> 32));
          if (a.top_ids) a.top_ids[row * a.top + larger] = (int)~(uint32_t)key;
          if (a.top_logprobs) a.top_logprobs[row * a.top + larger] = total == 0.f ? minus_infinity() : (v - base) * a.scale - log_total;
        }
      }
    }
  }
  if (gridDim.y > 1) cluster_sync();  // none may go while it is read
}

struct Bwd {
  const void* logits;
  Indices targets;
  const float2* stats;
  const float* entropy;
  const float* dlogprob;
  const float* dentropy;
  void* dlogits;
  int64_t rows, vocab, ld, lddl, dcols, segments;
  float scale;
};
constexpr int kBwdThreads = 256, kBwdChunks = 4;

template <bool F32, bool OUT32, bool ENTROPY>
__global__ void __launch_bounds__(kBwdThreads) logprob_bwd_kernel(const Bwd a) {
  griddep_wait();
  griddep_launch_dependents();
  const int64_t row = blockIdx.x / a.segments, c0 = (blockIdx.x - row * a.segments) * (kBwdThreads * kBwdChunks) + threadIdx.x;
  const void* const x = static_cast<const uint8_t*>(a.logits) + row * a.ld * (F32 ? 4 : 2);
  void* const out = static_cast<uint8_t*>(a.dlogits) + row * a.lddl * (OUT32 ? 4 : 2);
  const int64_t n8 = a.vocab >> 3;
  Raw8<F32> raw[kBwdChunks];
#pragma unroll
  for (int u = 0; u < kBwdChunks; ++u)
    if (c0 + u * kBwdThreads < n8) raw[u].load(x, (c0 + u * kBwdThreads) * 8);
  const float2 stats = a.stats[row];
  const int64_t target = a.targets.p ? a.targets[row] : -1;
  const bool there = target >= 0 && target < a.vocab;
  const float weight = there && a.dlogprob ? a.dlogprob[row] * a.scale : 0.f, of_entropy = ENTROPY ? a.dentropy[row] * a.scale : 0.f,
              entropy = ENTROPY ? a.entropy[row] : 0.f;
  const bool empty = stats.x == minus_infinity();
  auto grad = [&](float v, int64_t j) {
    const float log_p = fmaf(v - stats.x, a.scale, -stats.y), p = exp2_fast(log_p * kLog2e);
    float g = -weight * p;
    if (ENTROPY) g = fmaf(-of_entropy * p, fmaxf(log_p, -200.f) + entropy, g);  // (p is 0 below)
    if (there && j == target) g += weight;
    return empty ? 0.f : g;
  };
#pragma unroll
  for (int u = 0; u < kBwdChunks; ++u) {
    const int64_t c = c0 + u * kBwdThreads;
    float v[8];
    if (c < n8) {
      raw[u].values(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = grad(v[j], c * 8 + j);
      store8<OUT32>(out, c * 8, v);
    } else if (c * 8 < a.dcols) {
      for (int64_t j = c * 8; j < min(c * 8 + 8, a.dcols); ++j) {
        const float g = j < a.vocab ? grad(logit_at<F32>(x, j), j) : 0.f;
        if (OUT32)
          static_cast<float*>(out)[j] = g;
        else
          static_cast<__nv_bfloat16*>(out)[j] = __float2bfloat16_rn(g);
      }
    }
  }
}

// CTAs of a row: enough that every SM has one
unsigned cluster_of(int64_t rows, int64_t vocab) {
  unsigned n = 1;
  while (n < kMaxCluster && rows * n < 148 && vocab / (2 * n) >= 8 * kThreads) n *= 2;
  return n;
}

template <bool F32, bool ENTROPY, bool TOP>
cudaError_t launch_fwd(const Fwd& a, cudaStream_t s) {
  const unsigned ctas = cluster_of(a.rows, a.vocab);
  const auto kern = logprob_fwd_kernel<F32, ENTROPY, TOP>;
  const size_t smem = TOP ? sizeof(TopShared) : 0;
  const dim3 grid((unsigned)a.rows, ctas);
  return ctas > 1 ? launch_cluster(ctas, kern, grid, dim3(kThreads), smem, s, a) : launch_divided(50, kern, grid, dim3(kThreads), smem, s, a);
}
template <bool F32, bool OUT32>
cudaError_t launch_bwd(const Bwd& a, cudaStream_t s) {
  const auto kern = a.dentropy ? logprob_bwd_kernel<F32, OUT32, true> : logprob_bwd_kernel<F32, OUT32, false>;
  return launch_divided(kStreamingCarveout, kern, dim3((unsigned)(a.rows * a.segments)), dim3(kBwdThreads), 0, s, a);
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
  a.segments = ((l.dcols + 7) / 8 + kBwdThreads * kBwdChunks - 1) / (kBwdThreads * kBwdChunks);
  a.scale = l.scale;
  const cudaError_t e = l.fp32 ? (l.out_fp32 ? launch_bwd<true, true>(a, s) : launch_bwd<true, false>(a, s))
                               : (l.out_fp32 ? launch_bwd<false, true>(a, s) : launch_bwd<false, false>(a, s));
  count_launch();
  return e;
}

}  // namespace nvfp4

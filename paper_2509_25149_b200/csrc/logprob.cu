// Log probabilities of given tokens with entropy and the likeliest alternatives, and their gradient.
//   z = scale logit;  lse = ln sum e^z;  log p = z - lse;  H = - sum p log p
//   gradient by a logit  scale (dlogprob ((j == target) - p) - dentropy p (log p + H))
// Bound by HBM: the forward pass reads a row once, with the running maximum and the sums of e^(z - m) and (z - m) e^(z - m) in registers; the
// gradient reads it once more and writes: 8192 x 131072 in bf16 339 us (97 % of the copy rate) and 648 (101 %), in a long run 405 and 651.  There the GPU is
// at its power limit, at 1.5 GHz for 1.96, and what an element costs in instructions tells: everything is in powers of two, z log2(e) = x per, and a
// difference is one fused multiply-add, d = x per - ref.
//   ref is the binary32 number nearest to m per, and what the sums are relative to: its rounding is the same in all differences of a row, which it
//   moves by half a power of two at most, since this form is for |m per| <= 2^24.  Rows whose largest logit is beyond that, those that are masked with a large
//   finite number, say, take differences of the logits as they are, (x - m) per.
//   Logits more than 400 powers of two below the largest are taken for that far: p is 0 there all the same, and minus infinity has a finite
//   difference, so that p d is 0 too.
#include <algorithm>

#include "around.h"
#include "copy8.cuh"
#include "ends.h"

namespace nvfp4 {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kMaxCluster = 8;
constexpr int kRing = 5, kStage = kThreads * 32;  // what is on its way to a CTA: 32 bytes a thread and stage
constexpr float kLn2 = 0.69314718055994530942f, kLowest = -3.402823466e38f, kFar = -300.f, kReach = 400.f;

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
  float scale, per;  // per: scale in powers of two, rounded once
  int top;
};

__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 r = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// the larger ones, NaN where there is one
__device__ __forceinline__ uint32_t max_nan_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t max_nan(uint32_t a, uint32_t b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(__uint_as_float(a)), "f"(__uint_as_float(b)));
  return __float_as_uint(r);
}
// Sixteen bytes of a row: eight or four neighbouring logits
template <bool F32>
struct Chunk {
  static constexpr int E = F32 ? 4 : 8, kPairs = E / 2;
  uint4 w;
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
  // the same with every value no lower than `least`: a binary32 number, or twice a bf16 one
  __device__ __forceinline__ Chunk above(uint32_t least) const {
    Chunk r;
    r.w = F32 ? make_uint4(max_nan(w.x, least), max_nan(w.y, least), max_nan(w.z, least), max_nan(w.w, least))
              : make_uint4(max_nan_bf16x2(w.x, least), max_nan_bf16x2(w.y, least), max_nan_bf16x2(w.z, least), max_nan_bf16x2(w.w, least));
    return r;
  }
  // `least` of a number: rounded down
  __device__ __forceinline__ static uint32_t held(float v) {
    const uint32_t b = __float_as_uint(v);
    if (F32) return b;
    const uint32_t down = (b & 0x80000000u ? b + 0xffffu : b) >> 16;
    return down << 16 | down;
  }
  __device__ __forceinline__ float largest() const {
    if (F32) return fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
    const uint32_t m = max_bf16x2(max_bf16x2(w.x, w.y), max_bf16x2(w.z, w.w));
    return fmaxf(bf16_lo(m), bf16_hi(m));
  }
};

constexpr float kNear = 0x1p24f;  // powers of two: what m per rounds off is far below those that 2^d has room for, and m - 400 / per is not m

// What a row's differences are taken from: its largest logit (of the elements so far), m, minus infinity where there is none
struct Reference {
  float from, ref;  // near: 0 and fl(m per);  far: max(m, lowest) and 0
  bool near;
  __device__ __forceinline__ Reference(float m, float per) {
    ref = m * per;
    near = fabsf(ref) <= kNear;
    from = near ? 0.f : fmaxf(m, kLowest);
    ref = near ? ref : 0.f;
  }
  // of a logit, in powers of two
  __device__ __forceinline__ float distance(float x, float per) const { return fmaf(x - from, per, -ref); }
  // of what another reference stands for, which is from + ref / per
  __device__ __forceinline__ float distance(const Reference& r, float per) const { return fmaf(r.from - from, per, r.ref - ref); }
};

// What a lane holds of its elements: the largest logit m, and the sums of 2^d and d 2^d
template <bool F32, bool ENTROPY>
struct Running {
  float m;
  float2 s, t;
  Reference at;
  uint32_t least;
  __device__ __forceinline__ Running(float per) : m(minus_infinity()), s(make_float2(0.f, 0.f)), t(make_float2(0.f, 0.f)), at(m, per), least(0u) {}
  // the sums as those of differences from a larger maximum
  __device__ __forceinline__ void raise(float to, float per, float reach) {
    const Reference r(to, per);
    const float d = r.distance(at, per), f = exp2_fast(d);
    if (ENTROPY) t = mul2(fma2(both(fmaxf(d, kFar)), s, t), both(f));  // (f is 0 below)
    s = mul2(s, both(f));
    m = to;
    at = r;
    if (ENTROPY) least = Chunk<F32>::held(to - reach);
  }
  // TOGETHER: all lanes of the warp are here, and have one maximum: some ten times in a row there is a larger one, where every lane's own would be
  // exceeded in one lane or another nearly every time.  Returns the largest of these.
  template <bool TOGETHER, int N>
  __device__ __forceinline__ float add(const Chunk<F32> (&raw)[N], float per, float reach) {
    constexpr int P = Chunk<F32>::kPairs;
    float largest = raw[0].largest();
#pragma unroll
    for (int u = 1; u < N; ++u) largest = fmaxf(largest, raw[u].largest());
    if (TOGETHER) {
      if (__any_sync(0xffffffffu, largest > m)) raise(of_ordered(__reduce_max_sync(0xffffffffu, ordered(largest))), per, reach);
    } else if (largest > m) {
      raise(largest, per, reach);
    }
    if (__builtin_expect(at.near, 1)) {
#pragma unroll
      for (int u = 0; u < N; ++u) {
        float2 v[P];
        (ENTROPY ? raw[u].above(least) : raw[u]).values(v);
#pragma unroll
        for (int i = 0; i < P; ++i) {
          const float2 d = fma2(v[i], both(per), both(-at.ref)), e = make_float2(exp2_fast(d.x), exp2_fast(d.y));
          s = add2(s, e);
          if (ENTROPY) t = fma2(e, d, t);
        }
      }
    } else {
#pragma unroll
      for (int u = 0; u < N; ++u) {
        float2 v[P];
        raw[u].values(v);
#pragma unroll
        for (int i = 0; i < P; ++i) {
          one(v[i].x, per);
          one(v[i].y, per);
        }
      }
    }
    return largest;
  }
  // a single one, no larger than m
  __device__ __forceinline__ void one(float x, float per) {
    const float d = at.distance(x, per), e = exp2_fast(d);
    s.x += e;
    if (ENTROPY) t.x = fmaf(e, fmaxf(d, kFar), t.x);
  }
};

template <bool F32>
__device__ __forceinline__ float logit_at(const void* logits, int64_t at) {
  return F32 ? static_cast<const float*>(logits)[at] : bf16_lo(static_cast<const uint16_t*>(logits)[at]);
}
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

// W warps to a row: one (see warp_rows(); a CTA has kWarps rows), or a CTA, or a cluster of gridDim.y CTAs, each with a run of the row's
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
  const float per = a.per, reach = kReach / per;
  Running<F32, ENTROPY> run(per);
  // the row comes through a ring in which every thread has places of its own
  const uint32_t mine = smem_u32(smem) + threadIdx.x * 16;
  auto chunks_of = [&](int t) { return (int)max((full - c0 - t + T - 1) / T, (int64_t)0); };
  const int n = chunks_of(tid), stages = chunks_of(tid | 31) / kChunks;  // the thread's chunks; stages that are full for all of its warp
  float own = minus_infinity();  // (a NaN is nobody's maximum)
  const uint8_t* from = x + (c0 + tid) * 16;
  int asked = 0;
  auto fetch = [&](uint32_t to) {
#pragma unroll
    for (int u = 0; u < kChunks; ++u)
      if (asked + u < n) copy_async<16>(to + u * (kThreads * 16), from + u * (T * 16), true);
    asked += kChunks;
    from += kChunks * T * 16;
    copy_commit();  // (an empty group where there is no chunk: the count of groups stays that of the stages)
  };
#pragma unroll
  for (int u = 0; u < kRing - 1; ++u) fetch(mine + u * kStage);
  uint32_t at = mine, before = mine + (kRing - 1) * kStage;
  for (int i = 0; i < stages; ++i) {
    copy_wait<kRing - 2>();
    Chunk<F32> raw[kChunks];
#pragma unroll
    for (int u = 0; u < kChunks; ++u) raw[u].w = lds16(at + u * (kThreads * 16));
    fetch(before);  // the place of the stage before, whose values went into registers a turn ago
    before = at;
    at = at == mine + (kRing - 1) * kStage ? mine : at + kStage;
    const float largest = run.template add<true>(raw, per, reach);
    if (TOP) own = fmaxf(own, largest);
  }
  copy_wait<0>();
  for (int i = stages * kChunks; i < n; ++i) {  // (two at most)
    Chunk<F32> raw[1];
    raw[0].w = lds16(at + (i % kChunks) * (kThreads * 16));
    if (i % kChunks == kChunks - 1) at = at == mine + (kRing - 1) * kStage ? mine : at + kStage;
    own = fmaxf(own, run.template add<false>(raw, per, reach));
  }
  if (c1 > whole && tid == (int)((whole - c0) % T)) {  // a last chunk that is not full, to the thread whose turn it is
    for (int64_t j = whole * E; j < a.vocab; ++j) {
      const float v = logit_at<F32>(x, j);
      own = fmaxf(own, v);
      if (v > run.m) run.raise(v, per, reach);
      run.one(v, per);
    }
  }
  // the group's maximum, then sums of differences from it
  float m = run.m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (W > 1) {
    if (lane == 0) of_warp[warp].m = m;
    __syncthreads();
    m = of_warp[lane % kWarps].m;
#pragma unroll
    for (int o = kWarps / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  }
  run.raise(m, per, reach);
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
      if (parts > 1) {  // a lane to a CTA
        const uint32_t r = lane < (int)parts ? lane : 0;
        const float mr = ld_of_rank(&of_cta.m, r), sr = ld_of_rank(&of_cta.s, r), tr = ENTROPY ? ld_of_rank(&of_cta.t, r) : 0.f;
        m = mr;
#pragma unroll
        for (int o = kMaxCluster / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        m = __shfl_sync(0xffffffffu, m, 0);
        const float d = Reference(m, per).distance(Reference(mr, per), per), f = lane < (int)parts ? exp2_fast(d) : 0.f;
        s = f * sr;
        t = f * fmaf(fmaxf(d, kFar), sr, tr);
#pragma unroll
        for (int o = kMaxCluster / 2; o > 0; o >>= 1) {
          s += __shfl_xor_sync(0xffffffffu, s, o);
          if (ENTROPY) t += __shfl_xor_sync(0xffffffffu, t, o);
        }
        s = __shfl_sync(0xffffffffu, s, 0);
        if (ENTROPY) t = __shfl_sync(0xffffffffu, t, 0);
      }
    }
    const Reference ref(m, per);
    const float log_total = log2f(s);
    auto log_p = [&](float v) {
      const float d = ref.distance(v, per);
      if (!(s > 0.f)) return s == 0.f ? minus_infinity() : s;  // (NaN where the row has one, whatever is at v)
      // (far out, nothing beside the difference counts; its product with the scale may fit binary32 where that many powers of two, or the difference, do not)
      return d < -0x1p60f ? (0.5f * v - 0.5f * fmaxf(m, kLowest)) * a.scale * 2.f : kLn2 * (d - log_total);
    };
    if (tid == 0) {
      if (a.lse) a.lse[row] = fmaf(fmaxf(m, kLowest), a.scale, kLn2 * log_total);
      if (a.stats) a.stats[row] = make_float2(m, log_total);
      if (a.entropy) a.entropy[row] = s == 0.f ? 0.f : kLn2 * (log_total - t / s);
      if (a.logprob) {
        const int64_t target = a.targets[row];
        a.logprob[row] = target < 0 || target >= a.vocab ? 0.f : log_p(logit_at<F32>(x, target));
      }
    }
    if (TOP) {
      auto put = [&](int place, uint64_t key) {
        if (a.top_ids) a.top_ids[row * a.top + place] = (int)~(uint32_t)key;
        if (a.top_logprobs) a.top_logprobs[row * a.top + place] = log_p(of_ordered((uint32_t)(key >> 32)));
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
  float scale, per;
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

// What a row's gradient is made of: log2 p = d - total, d the distance from the row's reference, and the gradient p (a + b log2 p), with `hit` more at the target
struct RowGrad {
  Reference at;
  float total, a, b, hit;
  uint32_t least;
  int target_chunk, target_place;  // -1: none
  __device__ __forceinline__ RowGrad() : at(0.f, 0.f) {}
  template <bool F32, bool ENTROPY>
  __device__ __forceinline__ void load(const Bwd& g, int64_t row) {
    const float2 st = g.stats[row];
    const int64_t t = g.targets.p ? g.targets[row] : -1;
    const float w = g.dlogprob ? g.dlogprob[row] * g.scale : 0.f, e = ENTROPY ? g.dentropy[row] * g.scale : 0.f, h = ENTROPY ? g.entropy[row] : 0.f;
    const bool empty = st.x == minus_infinity() && st.y == minus_infinity(), there = t >= 0 && t < g.vocab && !empty;
    const float m = empty ? 0.f : st.x, per = g.per;  // (all of an empty row is p = 0 then; a NaN beside minus infinities is in the sum)
    at = Reference(m, per);
    least = Chunk<F32>::held(m - kReach / per);
    total = empty ? 0.f : st.y;
    hit = there ? w : 0.f;
    a = -fmaf(e, h, hit);
    b = -e * kLn2;
    target_chunk = there ? (int)(t / Chunk<F32>::E) : -1;
    target_place = (int)(t % Chunk<F32>::E);
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
  // (the last rows first: of what the forward pass read last some is still in L2)
  const int64_t warps = (int64_t)gridDim.x * kWarps, w = (int64_t)(gridDim.x - 1 - blockIdx.x) * kWarps + (threadIdx.x >> 5), first = a.steps * w / warps;
  const int steps = (int)(a.steps * (w + 1) / warps - first), whole = (int)(a.vocab / E), of_row = (int)a.per_row * 32;
  const uint32_t mine = smem_u32(smem) + threadIdx.x * 16;
  int64_t row = first / a.per_row;
  int c = (int)(first - row * a.per_row) * 32 + lane;  // a lane's chunk
  const int64_t pitch = a.ld * (F32 ? 4 : 2), out_pitch = a.lddl * (OUT32 ? 4 : 2);
  const uint8_t* ahead_row = static_cast<const uint8_t*>(a.logits) + row * pitch;
  uint8_t* out = static_cast<uint8_t*>(a.dlogits) + row * out_pitch + (int64_t)c * (E * (OUT32 ? 4 : 2));
  int ahead = c, asked = 0;
  const uint8_t* from = ahead_row + (int64_t)ahead * 16;
  auto fetch = [&](uint32_t to) {
    if (asked < steps) {
      if (ahead < whole) copy_async<16>(to, from, true);
      ++asked;
      ahead += 32;
      from += 512;
      if (ahead >= of_row) {
        ahead = lane;
        ahead_row += pitch;
        from = ahead_row + lane * 16;
      }
    }
    copy_commit();
  };
  griddep_wait();
  griddep_launch_dependents();
  if (steps == 0) return;
#pragma unroll
  for (int u = 0; u < kSlots - 1; ++u) fetch(mine + u * kSlot);
  uint32_t at = mine, before = mine + (kSlots - 1) * kSlot;
  RowGrad now, then;
  now.load<F32, ENTROPY>(a, row);
  then = now;
  if (row + 1 < a.rows) then.load<F32, ENTROPY>(a, row + 1);
  const float per = a.per;
  auto distance = [&](float v) { return __uint_as_float(max_nan(__float_as_uint(now.at.distance(v, per)), __float_as_uint(-kReach))); };
  auto grad = [&](float2 v) {  // of distances
    const float2 l = add2(v, both(-now.total)), p = make_float2(exp2_fast(l.x), exp2_fast(l.y));
    return mul2(p, ENTROPY ? fma2(l, both(now.b), both(now.a)) : both(now.a));
  };
  for (int i = 0; i < steps; ++i) {
    copy_wait<kSlots - 2>();
    if (c < whole) {
      Chunk<F32> raw;
      raw.w = lds16(at);
      float2 v[E / 2];
      if (__builtin_expect(now.at.near, 1)) {
        (ENTROPY ? raw.above(now.least) : raw).values(v);
#pragma unroll
        for (int j = 0; j < E / 2; ++j) v[j] = fma2(v[j], both(per), both(-now.at.ref));
      } else {
        raw.values(v);
#pragma unroll
        for (int j = 0; j < E / 2; ++j) v[j] = make_float2(distance(v[j].x), distance(v[j].y));
      }
#pragma unroll
      for (int j = 0; j < E / 2; ++j) v[j] = grad(v[j]);
      if (c == now.target_chunk) {
#pragma unroll
        for (int j = 0; j < E / 2; ++j) {
          if (now.target_place == 2 * j) v[j].x += now.hit;
          if (now.target_place == 2 * j + 1) v[j].y += now.hit;
        }
      }
      put<OUT32>(out, 0, v);
    } else {  // what is left of the columns, and zeros behind them
      const int left = (int)min((int64_t)E, a.dcols - (int64_t)c * E), held = (int)min((int64_t)E, a.vocab - (int64_t)c * E);
      for (int j = 0; j < left; ++j) {
        float g = 0.f;
        if (j < held)
          g = grad(both(distance(logit_at<F32>(static_cast<const uint8_t*>(a.logits) + row * pitch, (int64_t)c * E + j)))).x +
              (c == now.target_chunk && j == now.target_place ? now.hit : 0.f);
        if (OUT32)
          reinterpret_cast<float*>(out)[j] = g;
        else
          reinterpret_cast<__nv_bfloat16*>(out)[j] = __float2bfloat16_rn(g);
      }
    }
    fetch(before);
    before = at;
    at = at == mine + (kSlots - 1) * kSlot ? mine : at + kSlot;
    c += 32;
    out += 32 * E * (OUT32 ? 4 : 2);
    if (c >= of_row) {
      c = lane;
      ++row;
      out = static_cast<uint8_t*>(a.dlogits) + row * out_pitch + lane * (E * (OUT32 ? 4 : 2));
      now = then;
      if (i + 1 < steps && row + 1 < a.rows) then.load<F32, ENTROPY>(a, row + 1);
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

// Whether a warp takes a row by itself: it has no barriers to wait at, and takes longer by the row's length.  By one warp / by a CTA, us: 512 x 4096 4.2 / 4.2, 512 x 8192
// 5.9 / 5.1; 2048 x 8192 9.7 / 14.6, 2048 x 32768 26.3 / 28.4, 16384 x 1000 13.4 / 74, 16384 x 32768 166 / 193; with the eight likeliest tokens 2048 x 8192 21 / 30,
// 2048 x 16384 38 / 35, 16384 x 16384 151 / 256, 16384 x 32768 345 / 310.
bool warp_rows(int64_t rows, int64_t vocab, bool top) { return vocab <= 4096 || (rows >= 2048 && vocab <= (top ? 16384 : 32768)); }

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
  if (warp_rows(a.rows, a.vocab, TOP)) return launch_fwd<F32, ENTROPY, TOP, 1>(a, 1, s);
  return launch_fwd<F32, ENTROPY, TOP, kWarps>(a, cluster_of(a.rows, a.vocab), s);
}
template <bool F32, bool OUT32>
cudaError_t launch_bwd(const Bwd& a, cudaStream_t s) {
  const unsigned ctas = (unsigned)std::max<int64_t>(a.steps / (kWarps * kBwdSteps), std::min<int64_t>((a.steps + kWarps - 1) / kWarps, kBwdCtas));
  const auto kern = a.dentropy ? logprob_bwd_kernel<F32, OUT32, true> : logprob_bwd_kernel<F32, OUT32, false>;
  return launch_divided(100, kern, dim3(ctas), dim3(kThreads), kRing * kStage, s, a);
}

float in_powers_of_two(float scale) { return (float)((double)scale * 1.44269504088896340736); }

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
  a.per = in_powers_of_two(l.scale);
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
  a.per = in_powers_of_two(l.scale);
  const cudaError_t e = l.fp32 ? (l.out_fp32 ? launch_bwd<true, true>(a, s) : launch_bwd<true, false>(a, s))
                               : (l.out_fp32 ? launch_bwd<false, true>(a, s) : launch_bwd<false, false>(a, s));
  count_launch();
  return e;
}

}  // namespace nvfp4

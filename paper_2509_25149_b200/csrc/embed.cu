// Embedding lookup and the table's gradient.
//   out[i] = scale table[token i];   dtable[v] (+)= scale sum of dout[i] over the i whose token is v
// Both are bound by HBM: rows read, rows written.  For the gradient the tokens are sorted (stable, so that the order of a token's additions is that of
// its places) and every sum is a run of the sorted list: no atomics, the same bits in every run.  Three launches:
//   sort_kernel    a cluster of eight CTAs sorts (token, place) pairs by digits of up to nine bits; where the gradient is not added to what is
//                  there, all other CTAs fill the table with zeros meanwhile
//   runs_kernel    chunks of the sorted list: a run that lies in a chunk is written, one that crosses a border leaves partial sums
//   joined_kernel  the runs that cross borders
#include <algorithm>

#include "around.h"
#include "copy8.cuh"
#include "ends.h"

namespace nvfp4 {

namespace {

// -------------------------------------------------------------------------------------------------- forward ----
struct Fwd {
  Indices tokens;
  const void* table;
  void* out;
  int64_t n, vocab, cols, ldt, ldo, segments, items;
  float scale;
};
constexpr int kFwdThreads = 256, kFwdChunks = 4;  // chunks of a lane: a warp takes 1024 columns of a row

template <bool F32, bool OUT32>
__global__ void __launch_bounds__(kFwdThreads) embedding_fwd_kernel(const Fwd a) {
  const int64_t item = (int64_t)blockIdx.x * (kFwdThreads / 32) + (threadIdx.x >> 5);
  griddep_wait();
  griddep_launch_dependents();
  if (item >= a.items) return;
  const int64_t i = item / a.segments, first = (item - i * a.segments) * (32 * kFwdChunks) + (threadIdx.x & 31), n8 = a.cols >> 3;
  const int64_t token = a.tokens[i];
  const bool there = token >= 0 && token < a.vocab;
  Raw8<F32> raw[kFwdChunks];
#pragma unroll
  for (int u = 0; u < kFwdChunks; ++u) {
    if (there && first + 32 * u < n8)
      raw[u].load(a.table, token * a.ldt + (first + 32 * u) * 8);
    else
      raw[u].zero();
  }
#pragma unroll
  for (int u = 0; u < kFwdChunks; ++u) {
    float v[8];
    raw[u].values(v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = there ? v[j] * a.scale : 0.f;
    if (first + 32 * u < n8) store8<OUT32>(a.out, i * a.ldo + (first + 32 * u) * 8, v);
  }
}

// ------------------------------------------------------------------------------------------------- gradient ----
struct Entry {
  uint32_t token, place;  // token: vocab for padding, so that it stands at the end
};
__device__ __forceinline__ Entry load_entry(const Entry* p) {
  const uint2 v = __ldcg(reinterpret_cast<const uint2*>(p));
  return Entry{v.x, v.y};
}

constexpr int kSortCtas = 8, kSortThreads = 1024, kSortWarps = kSortThreads / 32, kBins = 512;
struct Sort {
  Indices tokens;
  Entry* sorted;
  Entry* other;
  float* zero;  // NULL: the table's rows stay as they are
  int64_t n, vocab, cols, ldt;
  int passes, bits;  // digits of `bits` bits
};
struct SortShared {
  uint32_t counts[kSortWarps][kBins];
  uint32_t total[kBins], base[kBins], of_warp[32];
};

// Zeros from shared memory, a piece at a time: one instruction stores 32 KB, so that a warp keeps an SM's stores going
constexpr int kPiece = 32768;
__device__ __forceinline__ void bulk_store(void* dst, uint32_t src, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void fill_with_zeros(const Sort& a, uint8_t* smem) {
  for (int i = threadIdx.x; i < kPiece / 16; i += kSortThreads) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0u, 0u, 0u, 0u);
  fence_proxy_async_smem();
  __syncthreads();
  if (threadIdx.x >= 32) return;
  const bool packed = a.ldt == a.cols;  // one long row then
  const int64_t rows = packed ? 1 : a.vocab, bytes = (packed ? a.vocab : 1) * a.cols * 4, per_row = (bytes + kPiece - 1) / kPiece;
  const int64_t stride = (int64_t)(gridDim.x - kSortCtas) * 32;
  for (int64_t p = (int64_t)(blockIdx.x - kSortCtas) * 32 + threadIdx.x; p < rows * per_row; p += stride) {
    const int64_t r = p / per_row, at = (p - r * per_row) * kPiece;
    bulk_store(reinterpret_cast<uint8_t*>(a.zero + r * a.ldt) + at, smem_u32(smem), (uint32_t)min((int64_t)kPiece, bytes - at));
  }
  asm volatile("cp.async.bulk.commit_group;\n\tcp.async.bulk.wait_group 0;" ::: "memory");
}

__global__ void __launch_bounds__(kSortThreads) sort_kernel(const Sort a) {
  extern __shared__ __align__(16) uint8_t smem[];
  SortShared& sh = *reinterpret_cast<SortShared*>(smem);
  griddep_wait();
  griddep_launch_dependents();
  if (blockIdx.x >= kSortCtas) {
    fill_with_zeros(a, smem);
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = blockIdx.x;
  const int64_t c0 = a.n * rank / kSortCtas, c1 = a.n * (rank + 1) / kSortCtas;
  const int64_t lo = c0 + (c1 - c0) * warp / kSortWarps, hi = c0 + (c1 - c0) * (warp + 1) / kSortWarps;
  const uint32_t below = (1u << lane) - 1u, mask = (1u << a.bits) - 1u;
  for (int pass = 0; pass < a.passes; ++pass) {
    const bool even = (a.passes - 1 - pass) % 2 == 0;
    const Entry* const src = even ? a.other : a.sorted;
    Entry* const dst = even ? a.sorted : a.other;
    const int shift = pass * a.bits;
    auto entry = [&](int64_t i) {
      if (pass > 0) return load_entry(src + i);
      const int64_t t = a.tokens[i];
      return Entry{t >= 0 && t < a.vocab ? (uint32_t)t : (uint32_t)a.vocab, (uint32_t)i};
    };
    for (int b = threadIdx.x; b < kSortWarps * kBins; b += kSortThreads) (&sh.counts[0][0])[b] = 0u;
    __syncthreads();
    // how often each digit occurs in the warp's part of the list
    for (int64_t i0 = lo; i0 < hi; i0 += 32) {
      const bool live = i0 + lane < hi;
      const uint32_t digit = live ? (entry(i0 + lane).token >> shift) & mask : ~0u;
      const uint32_t same = __match_any_sync(0xffffffffu, digit);
      if (live && (same & below) == 0u) sh.counts[warp][digit] += __popc(same);
      __syncwarp();
    }
    __syncthreads();
    // where its first one goes: behind all smaller digits, and behind the same one in the parts before
    uint32_t all = 0, before = 0;
    if (threadIdx.x < kBins) {
      uint32_t sum = 0;
#pragma unroll 8
      for (int w = 0; w < kSortWarps; ++w) {
        const uint32_t c = sh.counts[w][threadIdx.x];
        sh.counts[w][threadIdx.x] = sum;
        sum += c;
      }
      sh.total[threadIdx.x] = sum;
    }
    cluster_sync();
    if (threadIdx.x < kBins) {
#pragma unroll
      for (int r = 0; r < kSortCtas; ++r) {
        const uint32_t c = __float_as_uint(ld_of_rank(reinterpret_cast<const float*>(&sh.total[threadIdx.x]), r));
        before += r < rank ? c : 0u;
        all += c;
      }
    }
    uint32_t scan = all;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t v = __shfl_up_sync(0xffffffffu, scan, o);
      if (lane >= o) scan += v;
    }
    if (lane == 31) sh.of_warp[warp] = scan;
    __syncthreads();
    if (threadIdx.x < kBins) {
      for (int w = 0; w < warp; ++w) scan += sh.of_warp[w];
      const uint32_t base = scan - all + before;
#pragma unroll 8
      for (int w = 0; w < kSortWarps; ++w) sh.counts[w][threadIdx.x] += base;
    }
    __syncthreads();
    for (int64_t i0 = lo; i0 < hi; i0 += 32) {
      const bool live = i0 + lane < hi;
      Entry e{};
      if (live) e = entry(i0 + lane);
      const uint32_t digit = live ? (e.token >> shift) & mask : ~0u;
      const uint32_t same = __match_any_sync(0xffffffffu, digit);
      uint32_t at = 0;
      if (live) at = sh.counts[warp][digit];
      __syncwarp();
      if (live) {
        *reinterpret_cast<uint2*>(dst + at + __popc(same & below)) = make_uint2(e.token, e.place);
        if ((same & below) == 0u) sh.counts[warp][digit] = at + __popc(same);
      }
      __syncwarp();
    }
    cluster_sync();  // the list is written, and nobody reads the totals any more
  }
}

constexpr int kRunThreads = 128, kBatch = 8;  // rows whose loads are on their way together
struct Runs {
  const Entry* sorted;
  const void* dout;
  float* dtable;
  float* head;  // per chunk: the sum of the run that reaches into it from the chunk before
  float* tail;  // and of the run that begins in it and reaches into the next
  int64_t n, vocab, cols, lddo, ldt, chunk, chunks;
  int strips, threads;  // threads of a strip of columns; kRunThreads / threads chunks to a CTA
  float scale;
  int accumulate;
};

__device__ __forceinline__ void add_to_table(const Runs& a, uint32_t token, int64_t col, const float (&sum)[8]) {
  float* const p = a.dtable + (int64_t)token * a.ldt + col;
  float v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = sum[j] * a.scale;
  if (a.accumulate) {
    const float4 x = reinterpret_cast<const float4*>(p)[0], y = reinterpret_cast<const float4*>(p)[1];
    v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
    v[4] += y.x; v[5] += y.y; v[6] += y.z; v[7] += y.w;
  }
  store8<true>(p, 0, v);
}

template <bool F32>
__global__ void __launch_bounds__(kRunThreads) runs_kernel(const Runs a) {
  griddep_wait();
  griddep_launch_dependents();
  const int64_t group = blockIdx.x / a.strips, strip = blockIdx.x - group * a.strips;
  const int64_t c = group * (kRunThreads / a.threads) + threadIdx.x / a.threads;
  const int64_t col = (strip * a.threads + threadIdx.x % a.threads) * 8;
  if (c >= a.chunks || col >= a.cols) return;
  const int64_t first = c * a.chunk, end = min(first + a.chunk, a.n);
  const uint32_t before = first > 0 ? load_entry(a.sorted + first - 1).token : ~0u;
  const uint32_t after = end < a.n ? load_entry(a.sorted + end).token : ~0u;
  uint32_t token = load_entry(a.sorted + first).token;
  bool from_before = token == before;
  float sum[8] = {};
  auto leave = [&](bool goes_on) {
    if (token >= (uint32_t)a.vocab) return;
    if (from_before)
      store8<true>(a.head, c * a.cols + col, sum);
    else if (goes_on)
      store8<true>(a.tail, c * a.cols + col, sum);
    else
      add_to_table(a, token, col, sum);
  };
  for (int64_t i0 = first; i0 < end; i0 += kBatch) {
    Entry e[kBatch];
    Raw8<F32> raw[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) e[u] = i0 + u < end ? load_entry(a.sorted + i0 + u) : Entry{(uint32_t)a.vocab, 0u};
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (e[u].token < (uint32_t)a.vocab)
        raw[u].load(a.dout, (int64_t)e[u].place * a.lddo + col);
      else
        raw[u].zero();
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (i0 + u >= end) break;
      if (e[u].token != token) {
        leave(false);
        token = e[u].token;
        from_before = false;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] = 0.f;
      }
      float v[8];
      raw[u].values(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] += v[j];
    }
  }
  leave(token == after);
}

// A chunk whose last run begins in it and goes on: its tail and the heads of the chunks behind it that begin with the same token
__global__ void __launch_bounds__(kRunThreads) joined_kernel(const Runs a) {
  griddep_wait();
  griddep_launch_dependents();
  const int64_t c = blockIdx.x / a.strips, strip = blockIdx.x - c * a.strips;
  const int64_t first = c * a.chunk, next = first + a.chunk;
  if (next >= a.n) return;
  const uint32_t token = load_entry(a.sorted + next - 1).token;
  if (token >= (uint32_t)a.vocab || load_entry(a.sorted + next).token != token) return;
  if (first > 0 && load_entry(a.sorted + first - 1).token == token) return;  // (sorted: the whole chunk is this run then)
  const int lane = threadIdx.x & 31;
  int64_t more = 0;  // chunks that begin with the token
  while (true) {
    const int64_t at = (c + 1 + more + lane) * a.chunk;
    const uint32_t there = __ballot_sync(0xffffffffu, at < a.n && load_entry(a.sorted + min(at, a.n - 1)).token == token);
    const int lead = there == ~0u ? 32 : __ffs(~there) - 1;
    more += lead;
    if (lead < 32) break;
  }
  const int64_t col = (strip * kRunThreads + threadIdx.x) * 8;
  if (col >= a.cols) return;
  const float4* const t = reinterpret_cast<const float4*>(a.tail + c * a.cols + col);
  float4 x = t[0], y = t[1];
  double s[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
  const float* h = a.head + (c + 1) * a.cols + col;
#pragma unroll 4
  for (int64_t k = 0; k < more; ++k, h += a.cols) {
    const float4 u = reinterpret_cast<const float4*>(h)[0], v = reinterpret_cast<const float4*>(h)[1];
    s[0] += u.x; s[1] += u.y; s[2] += u.z; s[3] += u.w;
    s[4] += v.x; s[5] += v.y; s[6] += v.z; s[7] += v.w;
  }
  float sum[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) sum[j] = (float)s[j];
  add_to_table(a, token, col, sum);
}

// Entries of a chunk: few, so that few tokens fill the GPU, and at most some 1024 chunks, so that a run over all of them stays short
int64_t chunk_of(int64_t n) {
  if (n <= 32768) return n <= 4096 ? 8 : n <= 8192 ? 16 : 32;
  return ((n + 1023) / 1024 + 7) / 8 * 8;
}
int64_t chunks_of(int64_t n) { return (n + chunk_of(n) - 1) / chunk_of(n); }
size_t padded(size_t bytes) { return (bytes + 255) / 256 * 256; }

}  // namespace

cudaError_t launch_embedding_fwd(const Embed& e, cudaStream_t s) {
  Fwd a{};
  a.tokens = e.tokens;
  a.table = e.table;
  a.out = e.out;
  a.n = e.n; a.vocab = e.vocab; a.cols = e.cols;
  a.ldt = e.ldt; a.ldo = e.ldo;
  a.scale = e.scale;
  a.segments = (e.cols / 8 + 32 * kFwdChunks - 1) / (32 * kFwdChunks);
  a.items = e.n * a.segments;
  const auto kern = e.in_fp32 ? (e.out_fp32 ? embedding_fwd_kernel<true, true> : embedding_fwd_kernel<true, false>)
                              : (e.out_fp32 ? embedding_fwd_kernel<false, true> : embedding_fwd_kernel<false, false>);
  const cudaError_t err = launch_divided(kStreamingCarveout, kern, dim3((unsigned)((a.items + kFwdThreads / 32 - 1) / (kFwdThreads / 32))),
                                         dim3(kFwdThreads), 0, s, a);
  count_launch();
  return err;
}

size_t embedding_bwd_workspace(int64_t n, int64_t cols) {
  return 2 * padded((size_t)n * sizeof(Entry)) + 2 * padded((size_t)chunks_of(n) * cols * 4);
}

cudaError_t launch_embedding_bwd(const Embed& e, cudaStream_t s) {
  uint8_t* ws = static_cast<uint8_t*>(e.workspace);
  auto take = [&](size_t bytes) {
    uint8_t* const p = ws;
    ws += padded(bytes);
    return p;
  };
  Sort k{};
  k.tokens = e.tokens;
  k.sorted = reinterpret_cast<Entry*>(take((size_t)e.n * sizeof(Entry)));
  k.other = reinterpret_cast<Entry*>(take((size_t)e.n * sizeof(Entry)));
  k.zero = e.accumulate ? nullptr : static_cast<float*>(e.out);
  k.n = e.n; k.vocab = e.vocab; k.cols = e.cols; k.ldt = e.ldt;
  int bits = 1;
  while (((int64_t)1 << bits) <= e.vocab) ++bits;
  k.passes = (bits + 8) / 9;
  k.bits = (bits + k.passes - 1) / k.passes;
  static std::atomic<uint64_t> configured{0};
  int dev;
  cudaError_t err;
  if (device_needs_config(configured, &dev)) {
    if ((err = cudaFuncSetAttribute(sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SortShared))) != cudaSuccess)
      return err;
    device_configured(configured, dev);
  }
  unsigned grid = kSortCtas;
  if (!e.accumulate) {  // a CTA for every 64 KB of zeros, two to an SM at most
    const int64_t want = (e.vocab * e.cols * 4 + 65535) / 65536;
    grid += (unsigned)((std::min<int64_t>(want, 2 * 148 - kSortCtas) + 7) / 8 * 8);
  }
  err = launch_cluster(kSortCtas, sort_kernel, dim3(grid), dim3(kSortThreads), sizeof(SortShared), s, k);
  count_launch();
  if (err != cudaSuccess) return err;

  Runs r{};
  r.sorted = k.sorted;
  r.dout = e.table;
  r.dtable = static_cast<float*>(e.out);
  r.chunk = chunk_of(e.n);
  r.chunks = chunks_of(e.n);
  r.head = reinterpret_cast<float*>(take((size_t)r.chunks * e.cols * 4));
  r.tail = reinterpret_cast<float*>(take((size_t)r.chunks * e.cols * 4));
  r.n = e.n; r.vocab = e.vocab; r.cols = e.cols;
  r.lddo = e.ldo; r.ldt = e.ldt;
  r.scale = e.scale;
  r.accumulate = e.accumulate;
  r.threads = kRunThreads;
  while (r.threads > 8 && r.threads / 2 >= e.cols / 8) r.threads /= 2;
  r.strips = (int)((e.cols / 8 + r.threads - 1) / r.threads);
  const int per_cta = kRunThreads / r.threads;
  const int64_t ctas = (r.chunks + per_cta - 1) / per_cta * r.strips;
  err = launch_divided(kStreamingCarveout, e.in_fp32 ? runs_kernel<true> : runs_kernel<false>, dim3((unsigned)ctas), dim3(kRunThreads), 0, s, r);
  count_launch();
  if (err != cudaSuccess || r.chunks == 1) return err;
  r.strips = (int)((e.cols / 8 + kRunThreads - 1) / kRunThreads);
  err = launch_divided(kStreamingCarveout, joined_kernel, dim3((unsigned)(r.chunks * r.strips)), dim3(kRunThreads), 0, s, r);
  count_launch();
  return err;
}

}  // namespace nvfp4

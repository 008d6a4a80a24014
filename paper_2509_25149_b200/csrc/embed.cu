// Embedding lookup and the table's gradient.
//   out[i] = scale table[token i];   dtable[v] (+)= scale sum of dout[i] over the i whose token is v
// Both are bound by HBM: rows read, rows written.  For the gradient the tokens are sorted (stable, so that the order of a token's additions is that of
// its places) and every sum is a run of the sorted list: no order of additions that varies, the same bits in every run.
//   rank_kernel    few tokens: a warp counts how many stand before its token
//   sort_kernel    more: a cluster of eight CTAs sorts (token, place) pairs by digits of up to nine bits
//   digits_kernel  many: the same with a launch for each of a pass's steps, over all SMs
//   zeros_kernel   where the gradient is not added to what is there, zeros in the whole table, beside the sort
//   runs_kernel    chunks of the sorted list: whoever has the beginning of a run adds it up, over the end of its chunk too; of a run that has a whole
//                  chunk in its middle every chunk leaves a partial sum
//   joined_kernel  those long runs
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

// Tokens repeat, and with them the rows: loads that leave a row in L1, stores that leave L2 to the rows (16384 x 5120 46.9 -> 41 us, of which either is most)
template <bool F32>
__device__ __forceinline__ void load_row(Raw8<F32>& raw, const void* table, int64_t at) {
  const uint4* const p = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(table) + at * (F32 ? 4 : 2));
  raw.w[0] = p[0];
  if (F32) raw.w[F32 ? 1 : 0] = p[1];
}
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
      load_row(raw[u], a.table, token * a.ldt + (first + 32 * u) * 8);
    else
      raw[u].zero();
  }
#pragma unroll
  for (int u = 0; u < kFwdChunks; ++u) {
    float v[8];
    raw[u].values(v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = there ? v[j] * a.scale : 0.f;
    if (first + 32 * u < n8) store8_first_out<OUT32>(a.out, i * a.ldo + (first + 32 * u) * 8, v);
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

constexpr int kSortCtas = 8, kSortThreads = 1024, kSortWarps = kSortThreads / 32, kBins = 512, kSortTile = 4096;
struct Sort {
  Indices tokens;
  Entry* sorted;
  Entry* other;
  int64_t n, vocab;
  int passes, bits;     // digits of `bits` bits
  uint32_t* of_tile;    // digits_kernel: [digit][tile], how often it occurs, then how often in the tiles before
  uint32_t* of_digit;   // and in all of them
  int tiles, pass;
};
struct SortShared {
  uint32_t counts[kSortWarps][kBins];
  uint32_t total[kBins], of_warp[32];
  uint2 list[kSortTile];       // the CTA's part of the list
  uint16_t place[kSortTile];  // how many of an entry's warp have its digit and stand before it
};

// A pass of the sort as one CTA sees it, which has the entries c0 .. c1 - 1, kSortTile at most, and whose warps have a part of them each: how often each digit
// occurs in every warp's part, where each warp's first one of a digit goes (behind all smaller digits, and behind the same one in the parts before), and the
// moves, in which an entry's place is known.
struct Pass {
  const Sort& a;
  SortShared& sh;
  const Entry* src;
  Entry* dst;
  int64_t c0;
  int size, part, pass, shift, warps, warp, lane;  // part: entries of a warp
  __device__ __forceinline__ Pass(const Sort& a_, SortShared& sh_, int pass_, int64_t from, int64_t to)
      : a(a_), sh(sh_), c0(from), size((int)(to - from)), pass(pass_) {
    const bool even = (a.passes - 1 - pass) % 2 == 0;
    src = even ? a.other : a.sorted;
    dst = even ? a.sorted : a.other;
    shift = pass * a.bits;
    warp = threadIdx.x >> 5;
    lane = threadIdx.x & 31;
    part = ((size + kSortWarps - 1) / kSortWarps + 31) / 32 * 32;
    warps = (size + part - 1) / part;
  }
  __device__ __forceinline__ uint2 entry(int64_t i) const {
    if (pass > 0) {
      const Entry e = load_entry(src + i);
      return make_uint2(e.token, e.place);
    }
    const int64_t t = a.tokens[i];
    return make_uint2(t >= 0 && t < a.vocab ? (uint32_t)t : (uint32_t)a.vocab, (uint32_t)i);
  }
  __device__ __forceinline__ uint32_t digit_of(uint2 e) const { return (e.x >> shift) & ((1u << a.bits) - 1u); }
  // the lanes that have the same digit, by one vote a bit (match.any asks digit by digit, 10 % of the whole)
  __device__ __forceinline__ uint32_t alike(uint32_t digit, bool live) const {
    uint32_t same = __ballot_sync(0xffffffffu, live);
    for (int b = 0; b < a.bits; ++b) {
      const uint32_t ones = __ballot_sync(0xffffffffu, digit >> b & 1u);
      same &= digit >> b & 1u ? ones : ~ones;
    }
    return same;
  }
  // counts of every warp, turned into how many the warps before have; how often the thread's digit occurs in the CTA
  __device__ __forceinline__ uint32_t count() const {
    const uint32_t below = (1u << lane) - 1u;
    const int bins = 1 << a.bits;
    for (int i = threadIdx.x; i < size; i += kSortThreads) sh.list[i] = entry(c0 + i);
    for (int b = threadIdx.x; b < warps * bins; b += kSortThreads) sh.counts[b >> a.bits][b & (bins - 1)] = 0u;
    __syncthreads();
    for (int i0 = warp * part; i0 < min((warp + 1) * part, size); i0 += 32) {
      const bool live = i0 + lane < size;
      const uint32_t digit = live ? digit_of(sh.list[i0 + lane]) : 0u, same = alike(digit, live);
      uint32_t before = 0;
      if (live) before = sh.counts[warp][digit];
      __syncwarp();
      if (live) {
        sh.place[i0 + lane] = (uint16_t)(before + __popc(same & below));
        if ((same & below) == 0u) sh.counts[warp][digit] = before + __popc(same);
      }
      __syncwarp();
    }
    __syncthreads();
    uint32_t sum = 0;
    if (threadIdx.x < bins)
#pragma unroll 8
      for (int w = 0; w < warps; ++w) {
        const uint32_t c = sh.counts[w][threadIdx.x];
        sh.counts[w][threadIdx.x] = sum;
        sum += c;
      }
    return sum;
  }
  // all: how often the thread's digit occurs in the whole list; before: in the CTAs before
  __device__ __forceinline__ void move(uint32_t all, uint32_t before) const {
    uint32_t scan = all;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t v = __shfl_up_sync(0xffffffffu, scan, o);
      if (lane >= o) scan += v;
    }
    if (lane == 31) sh.of_warp[warp] = scan;
    __syncthreads();
    if (threadIdx.x < 1 << a.bits) {
      for (int w = 0; w < warp; ++w) scan += sh.of_warp[w];
      const uint32_t base = scan - all + before;
#pragma unroll 8
      for (int w = 0; w < warps; ++w) sh.counts[w][threadIdx.x] += base;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < size; i += kSortThreads) {
      const uint2 e = sh.list[i];
      *reinterpret_cast<uint2*>(dst + sh.counts[i / part][digit_of(e)] + sh.place[i]) = e;
    }
  }
};

// A token's place in the sorted list is the number of smaller ones and of equal ones before it.  That is n^2 / 32 steps for n tokens, without a barrier or
// a round trip to memory beside the first (1003 tokens 6.3 us; sorted by a single CTA they took 11.4); from some thousands on the sort is the shorter way.
constexpr int kRankThreads = 256, kRankMost = 4096;
__global__ void __launch_bounds__(kRankThreads) rank_kernel(const Sort a) {
  griddep_wait();
  griddep_launch_dependents();
  const int i = blockIdx.x * (kRankThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31, n = (int)a.n;
  if (i >= n) return;
  auto token = [&](int j) {
    const int64_t t = a.tokens[j];
    return t >= 0 && t < a.vocab ? (uint32_t)t : (uint32_t)a.vocab;
  };
  const uint32_t mine = token(i);
  int before = 0;
#pragma unroll 8
  for (int j = lane; j < n; j += 32) {
    const uint32_t t = token(j);
    before += t < mine || (t == mine && j < i);
  }
  before = __reduce_add_sync(0xffffffffu, before);
  if (lane == 0) *reinterpret_cast<uint2*>(a.sorted + before) = make_uint2(mine, (uint32_t)i);
}

__global__ void __launch_bounds__(kSortThreads) sort_kernel(const Sort a) {
  extern __shared__ __align__(16) uint8_t smem[];
  SortShared& sh = *reinterpret_cast<SortShared*>(smem);
  griddep_wait();
  griddep_launch_dependents();
  const int rank = blockIdx.x;
  for (int pass = 0; pass < a.passes; ++pass) {
    const Pass p(a, sh, pass, a.n * rank / kSortCtas, a.n * (rank + 1) / kSortCtas);
    const uint32_t mine = p.count();
    if (threadIdx.x < kBins) sh.total[threadIdx.x] = mine;
    cluster_sync();
    uint32_t all = 0, before = 0;
    if (threadIdx.x < 1 << a.bits) {
#pragma unroll
      for (int r = 0; r < kSortCtas; ++r) {
        const uint32_t c = __float_as_uint(ld_of_rank(reinterpret_cast<const float*>(&sh.total[threadIdx.x]), r));
        before += r < rank ? c : 0u;
        all += c;
      }
    }
    p.move(all, before);
    cluster_sync();  // the list is written, and nobody reads the totals any more
  }
}

// A pass over many tokens: every CTA counts the digits of a tile, a warp to a digit adds up what the tiles before have, and every CTA moves its tile.
template <bool MOVE>
__global__ void __launch_bounds__(kSortThreads) digits_kernel(const Sort a) {
  extern __shared__ __align__(16) uint8_t smem[];
  SortShared& sh = *reinterpret_cast<SortShared*>(smem);
  griddep_wait();
  griddep_launch_dependents();
  const int64_t c0 = (int64_t)blockIdx.x * kSortTile;
  const Pass p(a, sh, a.pass, c0, min(c0 + kSortTile, a.n));
  const uint32_t mine = p.count();
  const bool has = threadIdx.x < 1 << a.bits;
  uint32_t* const at = a.of_tile + (int64_t)threadIdx.x * a.tiles + blockIdx.x;
  if (MOVE)
    p.move(has ? __ldcg(a.of_digit + threadIdx.x) : 0u, has ? __ldcg(at) : 0u);
  else if (has)
    *at = mine;
}
__global__ void __launch_bounds__(256) before_kernel(const Sort a) {
  griddep_wait();
  griddep_launch_dependents();
  const int digit = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (digit >= 1 << a.bits) return;
  uint32_t* const row = a.of_tile + (int64_t)digit * a.tiles;
  uint32_t sum = 0;
  for (int i0 = 0; i0 < a.tiles; i0 += 32) {
    const uint32_t c = i0 + lane < a.tiles ? __ldcg(row + i0 + lane) : 0u;
    uint32_t scan = c;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t v = __shfl_up_sync(0xffffffffu, scan, o);
      if (lane >= o) scan += v;
    }
    if (i0 + lane < a.tiles) row[i0 + lane] = sum + scan - c;
    sum += __shfl_sync(0xffffffffu, scan, 31);
  }
  if (lane == 0) a.of_digit[digit] = sum;
}

// 32 KB of zeros to a CTA: CTAs that end and make room for the next ones keep to neighbouring memory, which HBM writes at 7.5 TB/s; resident ones that go
// on with a stride drift apart (2.7 GB 360 us; 430 to 450 with strides, whether of stores or of bulk copies).  The launch before it is the sort, which has
// waited for everything ahead of it and does not touch the table: the zeros need not wait for it, only the launch may not end before it.
constexpr int kZeroThreads = 256, kZeros = 8 * kZeroThreads;  // of sixteen bytes
__global__ void __launch_bounds__(kZeroThreads) zeros_kernel(float* table, int64_t rows, int64_t cols, int64_t ld) {
  griddep_launch_dependents();
  const int64_t c4 = cols >> 2, all = rows * c4, first = (int64_t)blockIdx.x * kZeros + threadIdx.x;
  const bool packed = ld == cols;
#pragma unroll
  for (int k = 0; k < kZeros / kZeroThreads; ++k) {
    const int64_t i = first + k * kZeroThreads;
    if (i >= all) break;
    const int64_t row = packed ? 0 : i / c4;
    reinterpret_cast<float4*>(table + row * ld)[i - row * c4] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  if (blockIdx.x == gridDim.x - 1) griddep_wait();
}

constexpr int kRunThreads = 128, kRunRing = 8;  // rows that are on their way to a thread, and the one it works on
struct Runs {
  const Entry* sorted;
  const void* dout;
  float* dtable;
  float* head;  // per chunk: of the long run that reaches into it from the chunk before
  float* tail;  // and of the long run that begins in it
  int64_t n, vocab, cols, lddo, ldt, chunks;
  int chunk, strips, threads;  // threads of a strip of columns; kRunThreads / threads chunks to a CTA
  float scale;
  int accumulate;
};
// what a thread has of a row: sixteen bytes
template <bool F32>
constexpr int kWide = F32 ? 4 : 8;

// Nobody else has these elements: an addition in memory instead of a load and a store leaves nothing to wait for (sums below 2^-126 come out as 0)
__device__ __forceinline__ void add_four(float* p, float4 v) {
  asm volatile("red.relaxed.gpu.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(p), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
template <int E>
__device__ __forceinline__ void add_to_table(const Runs& a, uint32_t token, int64_t col, const float (&sum)[E]) {
  float* const p = a.dtable + (int64_t)token * a.ldt + col;
#pragma unroll
  for (int j = 0; j < E; j += 4) {
    const float4 v = make_float4(sum[j] * a.scale, sum[j + 1] * a.scale, sum[j + 2] * a.scale, sum[j + 3] * a.scale);
    if (a.accumulate)
      add_four(p + j, v);
    else
      *reinterpret_cast<float4*>(p + j) = v;
  }
}

template <bool F32>
__global__ void __launch_bounds__(kRunThreads) runs_kernel(const Runs a) {
  constexpr int E = kWide<F32>;
  extern __shared__ __align__(16) uint8_t smem[];
  Entry* const list = reinterpret_cast<Entry*>(smem + kRunRing * kRunThreads * 16);
  griddep_wait();
  griddep_launch_dependents();
  const int groups = kRunThreads / a.threads;
  const int64_t group0 = blockIdx.x / a.strips * groups, strip = blockIdx.x % a.strips;
  // the entries of the CTA's chunks, of the one before (and its predecessor) and of the one behind (and its successor)
  const int64_t held0 = (group0 - 1) * a.chunk - 1;
  for (int i = threadIdx.x; i < (groups + 2) * a.chunk + 2; i += kRunThreads) {
    const int64_t at = held0 + i;
    list[i] = at >= 0 && at < a.n ? load_entry(a.sorted + at) : Entry{~0u, 0u};  // (no token)
  }
  __syncthreads();
  const int64_t c = group0 + threadIdx.x / a.threads, col = (strip * a.threads + threadIdx.x % a.threads) * E;
  if (c >= a.chunks || col >= a.cols) return;
  const Entry* const mine = list + (threadIdx.x / a.threads + 1) * a.chunk + 1;  // the chunk's first; entries from -chunk - 1 to 2 chunk are there
  const int size = (int)min((int64_t)a.chunk, a.n - c * a.chunk);
  int i = 0, end = size;
  bool from_before = mine[0].token == mine[-1].token;
  if (from_before && mine[0].token != mine[-a.chunk - 1].token && mine[0].token != mine[size].token) {  // who has its beginning adds it up
    while (i < size && mine[i].token == mine[0].token) ++i;
    from_before = false;
    if (i == size) return;
  }
  const uint32_t last = mine[size - 1].token;
  const bool goes_on = mine[size].token == last && last < (uint32_t)a.vocab, of_end = mine[i].token == last && from_before;
  const bool is_long = goes_on && (of_end || mine[size + a.chunk].token == last);
  if (goes_on && !is_long)
    while (mine[end].token == last) ++end;
  const uint32_t ring = smem_u32(smem) + threadIdx.x * 16;
  const uint8_t* const dout = static_cast<const uint8_t*>(a.dout) + col * (F32 ? 4 : 2);
  const int64_t pitch = a.lddo * (F32 ? 4 : 2);
  int ahead = i, slot = 0, next = 0;
  auto fetch = [&] {
    if (ahead < end && mine[ahead].token < (uint32_t)a.vocab) copy_async<16>(ring + next * (kRunThreads * 16), dout + mine[ahead].place * pitch, true);
    copy_commit();  // (an empty group where there is no row: the count of groups stays that of the entries)
    ++ahead;
    next = next + 1 == kRunRing ? 0 : next + 1;
  };
#pragma unroll
  for (int u = 0; u < kRunRing - 1; ++u) fetch();
  uint32_t token = mine[i].token;
  float sum[E] = {};
  for (; i < end; ++i) {
    const uint32_t now = mine[i].token;
    if (now >= (uint32_t)a.vocab) break;  // (padding stands at the end of the list)
    if (now != token) {
      if (from_before) {
#pragma unroll
        for (int j = 0; j < E; j += 4) *reinterpret_cast<float4*>(a.head + c * a.cols + col + j) = make_float4(sum[j], sum[j + 1], sum[j + 2], sum[j + 3]);
      } else {
        add_to_table(a, token, col, sum);
      }
      token = now;
      from_before = false;
#pragma unroll
      for (int j = 0; j < E; ++j) sum[j] = 0.f;
    }
    copy_wait<kRunRing - 2>();
    const uint4 raw = lds16(ring + slot * (kRunThreads * 16));
    fetch();
    slot = slot + 1 == kRunRing ? 0 : slot + 1;
    if (F32) {
      sum[0] += __uint_as_float(raw.x);
      sum[1] += __uint_as_float(raw.y);
      sum[2] += __uint_as_float(raw.z);
      sum[3] += __uint_as_float(raw.w);
    } else {
      float2 v[4];
      unpack8(raw, v);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        sum[(2 * j) % E] += v[j].x;
        sum[(2 * j + 1) % E] += v[j].y;
      }
    }
  }
  copy_wait<0>();
  if (token >= (uint32_t)a.vocab) return;
  float* const partial = from_before ? a.head : is_long ? a.tail : nullptr;
  if (partial) {
#pragma unroll
    for (int j = 0; j < E; j += 4) *reinterpret_cast<float4*>(partial + c * a.cols + col + j) = make_float4(sum[j], sum[j + 1], sum[j + 2], sum[j + 3]);
  } else {
    add_to_table(a, token, col, sum);
  }
}

// The chunks in which long runs begin: a run's tail and the heads of the chunks behind it that begin with the same token, in 64 bits.  A CTA looks for them among
// 32 chunks, a lane to a chunk, and adds up 128 columns of what it finds: a warp to a run, or 2, 4 or 8 with shares of its heads where it finds few
// (4096 tokens of one kind 112 -> 40 us with all three launches, which a CTA to every chunk took; 16384 x 5120 12.2 -> 9.1 of 438).  What follows on the stream starts when
// it ends: a sort that stood by earlier cost 10 us.
constexpr int kJoinThreads = 256, kJoinWarps = kJoinThreads / 32, kJoinChunks = 32;
__global__ void __launch_bounds__(kJoinThreads) joined_kernel(const Runs a) {
  __shared__ double4 share[kJoinWarps][32];
  griddep_wait();
  const int64_t group = blockIdx.x / a.strips, strip = blockIdx.x - group * a.strips;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  bool mine = false;
  const int64_t own = group * kJoinChunks + lane, own_next = (own + 1) * a.chunk;
  if (own_next + a.chunk < a.n) {
    const uint32_t token = load_entry(a.sorted + own_next - 1).token, behind = load_entry(a.sorted + own_next + a.chunk).token;
    const uint32_t before = own > 0 ? load_entry(a.sorted + own_next - a.chunk - 1).token : ~0u;
    mine = token == behind && token != before && token < (uint32_t)a.vocab;
  }
  const uint32_t found = __ballot_sync(0xffffffffu, mine);  // (the same in every warp)
  const int runs = __popc(found);
  if (runs == 0) return;
  int team = 1;  // warps of a run
  while (team < kJoinWarps && 2 * team * runs <= kJoinWarps) team *= 2;
  const int64_t col = (strip * 32 + lane) * 4;
  for (int r0 = 0; r0 < runs; r0 += kJoinWarps / team) {
    const int r = r0 + warp / team, part = warp % team;
    double s[4] = {};
    uint32_t token = 0;
    if (r < runs) {
      uint32_t bits = found;
      for (int k = 0; k < r; ++k) bits &= bits - 1u;
      const int64_t c = group * kJoinChunks + __ffs(bits) - 1;
      token = load_entry(a.sorted + (c + 1) * a.chunk - 1).token;
      int64_t more = 0;  // chunks that begin with the token
      while (true) {
        const int64_t k = (c + 1 + more + lane) * a.chunk;
        const uint32_t there = __ballot_sync(0xffffffffu, k < a.n && load_entry(a.sorted + min(k, a.n - 1)).token == token);
        const int lead = there == ~0u ? 32 : __ffs(~there) - 1;
        more += lead;
        if (lead < 32) break;
      }
      if (col < a.cols) {
        const int64_t k0 = more * part / team, k1 = more * (part + 1) / team;
        const float* h = a.head + (c + 1 + k0) * a.cols + col;
        if (part == 0) {
          const float4 x = *reinterpret_cast<const float4*>(a.tail + c * a.cols + col);
          s[0] = x.x; s[1] = x.y; s[2] = x.z; s[3] = x.w;
        }
#pragma unroll 8
        for (int64_t k = k0; k < k1; ++k, h += a.cols) {
          const float4 x = *reinterpret_cast<const float4*>(h);
          s[0] += x.x;
          s[1] += x.y;
          s[2] += x.z;
          s[3] += x.w;
        }
      }
    }
    if (team > 1) {
      share[warp][lane] = make_double4(s[0], s[1], s[2], s[3]);
      __syncthreads();
      if (part == 0)
        for (int k = 1; k < team; ++k) {
          const double4 x = share[warp + k][lane];
          s[0] += x.x;
          s[1] += x.y;
          s[2] += x.z;
          s[3] += x.w;
        }
      __syncthreads();
    }
    if (r < runs && part == 0 && col < a.cols) {
      const float sum[4] = {(float)s[0], (float)s[1], (float)s[2], (float)s[3]};
      add_to_table(a, token, col, sum);
    }
  }
}

// Entries of a chunk: few, so that few tokens fill the GPU, and more with their number, so that a run over all of them is of few partial sums
int64_t chunk_of(int64_t n) {
  if (n <= 32768) return n <= 4096 ? 8 : n <= 8192 ? 16 : 32;
  return std::min<int64_t>(((n + 1023) / 1024 + 7) / 8 * 8, 256);
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

constexpr int64_t kClusterMost = kSortCtas * kSortTile;  // tokens that the cluster sorts
int64_t tiles_of(int64_t n) { return n > kClusterMost ? (n + kSortTile - 1) / kSortTile : 0; }
size_t embedding_bwd_workspace(int64_t n, int64_t cols) {
  return 2 * padded((size_t)n * sizeof(Entry)) + 2 * padded((size_t)chunks_of(n) * cols * 4) + padded((size_t)(tiles_of(n) + 1) * kBins * 4);
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
  k.n = e.n; k.vocab = e.vocab;
  int bits = 1;
  while (((int64_t)1 << bits) <= e.vocab) ++bits;
  k.passes = (bits + 8) / 9;
  k.bits = (bits + k.passes - 1) / k.passes;
  static std::atomic<uint64_t> configured{0};
  int dev;
  cudaError_t err;
  if (device_needs_config(configured, &dev)) {
    if ((err = cudaFuncSetAttribute(sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SortShared))) != cudaSuccess ||
        (err = cudaFuncSetAttribute(digits_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SortShared))) != cudaSuccess ||
        (err = cudaFuncSetAttribute(digits_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SortShared))) != cudaSuccess ||
        (err = cudaFuncSetAttribute(runs_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, 64 * 1024)) != cudaSuccess ||
        (err = cudaFuncSetAttribute(runs_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, 64 * 1024)) != cudaSuccess)
      return err;
    device_configured(configured, dev);
  }
  if (e.n <= kRankMost) {
    err = launch_divided(-1, rank_kernel, dim3((unsigned)((e.n + kRankThreads / 32 - 1) / (kRankThreads / 32))), dim3(kRankThreads), 0, s, k);
    count_launch();
  } else if (e.n <= kClusterMost) {
    err = launch_cluster(kSortCtas, sort_kernel, dim3(kSortCtas), dim3(kSortThreads), sizeof(SortShared), s, k);
    count_launch();
  } else {
    k.tiles = (int)tiles_of(e.n);
    k.of_tile = reinterpret_cast<uint32_t*>(take((size_t)(k.tiles + 1) * kBins * 4));
    k.of_digit = k.of_tile + (int64_t)k.tiles * kBins;
    err = cudaSuccess;
    for (k.pass = 0; k.pass < k.passes && err == cudaSuccess; ++k.pass) {
      err = launch_divided(100, digits_kernel<false>, dim3((unsigned)k.tiles), dim3(kSortThreads), sizeof(SortShared), s, k);
      if (err == cudaSuccess) err = launch_kernel(before_kernel, dim3((1u << k.bits) / 8 + 1), dim3(256), 0, s, k);
      if (err == cudaSuccess) err = launch_divided(100, digits_kernel<true>, dim3((unsigned)k.tiles), dim3(kSortThreads), sizeof(SortShared), s, k);
      count_launch(3);
    }
  }
  if (err != cudaSuccess) return err;
  if (!e.accumulate) {
    err = launch_divided(-1, zeros_kernel, dim3((unsigned)((e.vocab * (e.cols / 4) + kZeros - 1) / kZeros)), dim3(kZeroThreads), 0, s,
                         static_cast<float*>(e.out), e.vocab, e.cols, e.ldt);
    count_launch();
    if (err != cudaSuccess) return err;
  }

  Runs r{};
  r.sorted = k.sorted;
  r.dout = e.table;
  r.dtable = static_cast<float*>(e.out);
  r.chunk = (int)chunk_of(e.n);
  r.chunks = chunks_of(e.n);
  r.head = reinterpret_cast<float*>(take((size_t)r.chunks * e.cols * 4));
  r.tail = reinterpret_cast<float*>(take((size_t)r.chunks * e.cols * 4));
  r.n = e.n; r.vocab = e.vocab; r.cols = e.cols;
  r.lddo = e.ldo; r.ldt = e.ldt;
  r.scale = e.scale;
  r.accumulate = e.accumulate;
  const int64_t wide = e.cols / (e.in_fp32 ? 4 : 8);
  r.threads = kRunThreads;
  while (r.threads > 8 && r.threads / 2 >= wide) r.threads /= 2;
  r.strips = (int)((wide + r.threads - 1) / r.threads);
  const int groups = kRunThreads / r.threads;
  const size_t smem = kRunRing * kRunThreads * 16 + ((size_t)(groups + 2) * r.chunk + 2) * sizeof(Entry);
  err = launch_divided(100, e.in_fp32 ? runs_kernel<true> : runs_kernel<false>, dim3((unsigned)((r.chunks + groups - 1) / groups * r.strips)),
                       dim3(kRunThreads), smem, s, r);
  count_launch();
  if (err != cudaSuccess || r.chunks <= 2) return err;
  r.strips = (int)((e.cols / 4 + 31) / 32);
  err = launch_divided(kStreamingCarveout, joined_kernel, dim3((unsigned)((r.chunks + kJoinChunks - 1) / kJoinChunks * r.strips)), dim3(kJoinThreads), 0, s, r);
  count_launch();
  return err;
}

}  // namespace nvfp4

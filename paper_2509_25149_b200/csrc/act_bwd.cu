// The gradient through an activation, dz = da act'(z), with the bias gradient (the column sums of dz) and, where asked, act(z) made
// again for the weight gradient of the layer behind: from the z that the product's epilogue kept, in bf16 or in 8 bits.
// Bound by HBM (da 2, z 1 + 1/32 or 2, dz 2, a 2 bytes per element), so everything is one pass: a CTA takes 256 columns and a run
// of rows, a lane eight neighbouring columns, and their sums stay in its registers.  The sums of a CTA leave as a row of partial
// sums, which a second kernel adds in a fixed order: no atomics, the same bits in every run.
#include <algorithm>

#include "act.cuh"
#include "around.h"
#include "copy8.cuh"

namespace nvfp4 {

namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps, kCols = 256, kRing = 6;  // kRing: rows of a warp that its ring has room for

// Rows of a CTA.  With four CTAs on each of 148 SMs all at once the rings are filled once only: that is for runs of up to 512 rows (4088 x
// 5128 26.8 -> 25.6 us, 16384 x 1024 21.7 -> 20.3, 256 x 20480 11.1 -> 9.7).  Longer ones drift apart and leave SMs idle at the end (8192 x
// 20480, GELU from bf16, 177 us): there eight rounds of such CTAs (154 us).
int64_t chunk_rows(int64_t rows, int64_t cols) {
  const int64_t strips = (cols + kCols - 1) / kCols;
  auto per_cta = [&](int64_t ctas) { return (rows + std::max<int64_t>(ctas / strips, 1) - 1) / std::max<int64_t>(ctas / strips, 1); };
  int64_t n = per_cta(592);
  if (n > 512) n = per_cta(8 * 592);
  return (std::max<int64_t>(n, 32) + kWarps - 1) / kWarps * kWarps;
}
// Few rows: the CTAs of a strip of columns, eight at most, are a cluster that adds up its sums itself (up to 256 rows no slower on the GPU, 8 x
// 5120 3.2 -> 1.9 us, 64 x 20480 7.1 -> 5.2, 256 x 5120 5.8 / 5.8, 512 x 5120 7.5 / 8.1, and a launch less for the host)
bool in_cluster(int64_t rows) { return rows <= 256; }
int64_t cluster_rows(int64_t rows) { return (std::max<int64_t>((rows + 7) / 8, 32) + kWarps - 1) / kWarps * kWarps; }
int64_t chunk_count(int64_t rows, int64_t cols) {
  const int64_t n = chunk_rows(rows, cols);
  return (rows + n - 1) / n;
}

struct Args {
  const uint16_t* da;
  const uint16_t* z;
  Copy8 z8;
  uint16_t* dz;
  uint16_t* a;
  float* partial;  // NULL: no bias gradient, or
  float* sums;     // the CTAs of a strip are a cluster, and its first one writes the bias gradient
  int accumulate;
  int64_t rows, cols, ldda, ldz, lddz, lda, chunk_rows;
};

template <bool Z8>
constexpr int kStageBytes = kThreads * (Z8 ? 24 : 32);  // da and z of a row of every warp

// da and z come by cp.async through a ring in shared memory, in which every thread has places of its own: five rows of a warp are in
// flight whatever the registers hold, and a thread waits for nobody else's.
template <int ACT, bool Z8>
__global__ void __launch_bounds__(kThreads, 4) act_bwd_kernel(const Args g) {
  extern __shared__ __align__(16) uint8_t ring[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t col = (int64_t)blockIdx.x * kCols + lane * 8;
  const bool live = col < g.cols, have_z = ACT != NVFP4_ACT_NONE || g.a != nullptr;
  const int64_t r0 = (int64_t)blockIdx.y * g.chunk_rows, rows = min(g.chunk_rows, g.rows - r0);
  const int steps = warp < rows ? (int)((rows - warp + kWarps - 1) / kWarps) : 0;
  const int64_t row0 = r0 + warp, at = live ? col : 0;
  const uint16_t* const da = g.da + row0 * g.ldda + at;
  const uint16_t* const zb = Z8 ? nullptr : g.z + row0 * g.ldz + at;
  const uint8_t* const codes = Z8 ? g.z8.codes + row0 * g.cols + at : nullptr;
  const uint8_t* const bytes = Z8 ? g.z8.scales + row0 * g.z8.blocks + (at >> 5) : nullptr;
  const uint32_t mine = smem_u32(ring) + threadIdx.x * 16, mine_z = smem_u32(ring) + kThreads * 16 + threadIdx.x * (Z8 ? 8 : 16);
  auto fetch = [&](int s, int slot) {
    if (live && s < steps) {
      copy_async<16>(mine + slot * kStageBytes<Z8>, da + s * (kWarps * g.ldda), true);
      if (have_z) {
        if (Z8)
          copy_async<8>(mine_z + slot * kStageBytes<Z8>, codes + s * (kWarps * g.cols), true);
        else
          copy_async<16>(mine_z + slot * kStageBytes<Z8>, zb + s * (kWarps * g.ldz), true);
      }
    }
    copy_commit();  // (an empty group where there is no row: the count of groups stays that of the rows)
  };
  uint32_t byte = 0;  // of the row to come
  auto fetch_byte = [&](int s) {
    if (Z8 && have_z && live && s < steps) byte = ldg8(bytes + s * (kWarps * g.z8.blocks));
  };
  griddep_wait();
  griddep_launch_dependents();
#pragma unroll
  for (int u = 0; u < kRing - 1; ++u) fetch(u, u);
  fetch_byte(0);
  float sum[8] = {};
  int slot = 0, next = kRing - 1;
  for (int s = 0; s < steps; ++s) {
    copy_wait<kRing - 2>();
    float d[8], z[8] = {}, out[8], a[8];
    unpack8(lds16(mine + slot * kStageBytes<Z8>), d);
    if (have_z) {
      if (Z8)
        decode8(lds8(mine_z + slot * kStageBytes<Z8>), decode_scale8(byte), z);
      else
        unpack8(lds16(mine_z + slot * kStageBytes<Z8>), z);
    }
    fetch_byte(s + 1);
    fetch(s + kRing - 1, next);  // the slot of the row before, whose values went into registers a turn ago
    slot = slot + 1 == kRing ? 0 : slot + 1;
    next = next + 1 == kRing ? 0 : next + 1;
    if (!live) continue;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      out[i] = d[i] * act_slope<ACT>(z[i], a[i]);
      sum[i] += out[i];
    }
    const int64_t row = row0 + (int64_t)s * kWarps;
    if (g.dz) store8<false>(g.dz, row * g.lddz + col, out);
    if (g.a) store8<false>(g.a, row * g.lda + col, a);
  }
  copy_wait<0>();
  if (!g.partial && !g.sums) return;
  __syncthreads();  // the ring is empty; the sums take its place
  auto part = reinterpret_cast<float(*)[kCols]>(ring);
  static_assert((kWarps + 1) * kCols * 4 <= kRing * kStageBytes<Z8>, "the sums reuse the ring");
#pragma unroll
  for (int i = 0; i < 8; ++i) part[warp][lane * 8 + i] = sum[i];
  __syncthreads();
  const int64_t c = (int64_t)blockIdx.x * kCols + threadIdx.x;
  float total = 0.f;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) total += part[w][threadIdx.x];
  if (g.sums) {
    part[kWarps][threadIdx.x] = total;
    cluster_sync();
    if (blockIdx.y == 0 && c < g.cols) {
      for (uint32_t k = 1; k < gridDim.y; ++k) total += ld_of_rank(&part[kWarps][threadIdx.x], k);
      g.sums[c] = g.accumulate ? g.sums[c] + total : total;
    }
    cluster_sync();  // none may go while its sums are read
  } else if (c < g.cols) {
    g.partial[(int64_t)blockIdx.y * g.cols + c] = total;
  }
}

// 32 columns to a CTA; every warp sums a share of the rows, one thread a column's shares
template <int kShares>
__global__ void __launch_bounds__(32 * kShares) column_sums_kernel(const float* partial, int64_t parts, int64_t cols, float* out,
                                                                   int accumulate, float* out2, int64_t split) {
  griddep_wait();
  griddep_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t c = (int64_t)blockIdx.x * 32 + lane;
  const int64_t p0 = parts * warp / kShares, p1 = parts * (warp + 1) / kShares;
  float s = 0.f;
  if (c < cols) {
    const float* p = partial + p0 * cols + c;
#pragma unroll 8
    for (int64_t k = p0; k < p1; ++k, p += cols) s += *p;
  }
  __shared__ float share[kShares][32];
  share[warp][lane] = s;
  __syncthreads();
  if (warp != 0 || c >= cols) return;
  float total = 0.f;
#pragma unroll
  for (int k = 0; k < kShares; ++k) total += share[k][lane];
  float* const to = c < split ? out : out2;
  if (!to) return;
  const int64_t at = c < split ? c : c - split;
  to[at] = accumulate ? to[at] + total : total;
}

template <int ACT, bool Z8>
cudaError_t launch_act(const Args& k, dim3 grid, cudaStream_t s) {
  constexpr int smem = kRing * kStageBytes<Z8>;
  auto kern = act_bwd_kernel<ACT, Z8>;
  static std::atomic<uint64_t> configured{0};  // per instantiation and device
  int dev;
  if (device_needs_config(configured, &dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    device_configured(configured, dev);
  }
  if (!k.sums || grid.y == 1) return launch_divided(100, kern, grid, dim3(kThreads), smem, s, k);
  return launch_cluster(grid.y, kern, grid, dim3(kThreads), smem, s, k);
}
template <int ACT>
cudaError_t launch_act(const Args& k, bool z8, dim3 grid, cudaStream_t s) {
  return z8 ? launch_act<ACT, true>(k, grid, s) : launch_act<ACT, false>(k, grid, s);
}

}  // namespace

int64_t act_bwd_workspace_floats(int64_t rows, int64_t cols) { return chunk_count(rows, cols) * cols; }

cudaError_t launch_column_sums(const float* partial, int64_t parts, int64_t cols, float* out, bool accumulate, cudaStream_t s, float* out2,
                               int64_t split) {
  // the more rows, the more warps: 148 rows of 5120 columns 5.4 us with eight of them, 8 rows of 20480 1.7 us slower with 32
  const bool many = parts > 32;
  const cudaError_t e = launch_divided(kStreamingCarveout, many ? column_sums_kernel<32> : column_sums_kernel<8>,
                                       dim3((unsigned)((cols + 31) / 32)), dim3(many ? 1024 : 256), 0, s, partial, parts, cols, out,
                                       (int)accumulate, out2, split > 0 ? split : cols);
  count_launch();
  return e;
}

cudaError_t launch_act_bwd(const ActBwd& a, cudaStream_t s) {
  Args k{};
  k.da = static_cast<const uint16_t*>(a.da);
  k.z = static_cast<const uint16_t*>(a.z);
  if (a.z8) k.z8 = Copy8{a.z8->codes, a.z8->scales, blocks8(a.cols)};
  k.dz = static_cast<uint16_t*>(a.dz);
  k.a = static_cast<uint16_t*>(a.a);
  const bool direct = a.dbias && in_cluster(a.rows);
  k.partial = a.dbias && !direct ? a.workspace : nullptr;
  k.sums = direct ? a.dbias : nullptr;
  k.accumulate = a.accumulate;
  k.rows = a.rows; k.cols = a.cols;
  k.ldda = a.ldda; k.ldz = a.ldz; k.lddz = a.lddz; k.lda = a.lda;
  k.chunk_rows = direct ? cluster_rows(a.rows) : chunk_rows(a.rows, a.cols);
  const int64_t chunks = (a.rows + k.chunk_rows - 1) / k.chunk_rows;
  const dim3 grid((unsigned)((a.cols + kCols - 1) / kCols), (unsigned)chunks);
  const bool z8 = a.z8 != nullptr;
  cudaError_t e;
  switch (a.act) {
    case NVFP4_ACT_RELU2: e = launch_act<NVFP4_ACT_RELU2>(k, z8, grid, s); break;
    case NVFP4_ACT_SILU: e = launch_act<NVFP4_ACT_SILU>(k, z8, grid, s); break;
    case NVFP4_ACT_GELU: e = launch_act<NVFP4_ACT_GELU>(k, z8, grid, s); break;
    default: e = launch_act<NVFP4_ACT_NONE>(k, z8, grid, s); break;
  }
  count_launch();
  if (e != cudaSuccess || !a.dbias || direct) return e;
  return launch_column_sums(a.workspace, chunks, a.cols, a.dbias, a.accumulate, s);
}

}  // namespace nvfp4

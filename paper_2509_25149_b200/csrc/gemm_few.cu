// BF16 product of a few rows (tokens in generation) with a weight, and its epilogue:  z = A B^T + bias, D = act(z) + residual.
// Bound by the bytes of the weight B [N x K]: 2 flops per byte and row.  The tensor-memory kernels work on 256 rows at a time and take
// as long for one row as for 256 (1 x 5120 x 5120 31 us), and those of gemm_tokens.cuh start slower (8 x 5120 x 5120 12.3 us, here 11.7); here B streams from memory straight into the registers of warp-wide
// mma.sync instructions, 16 rows of B against 8 rows of A.  The order of k within an instruction is free as long as both operands agree: a lane
// takes 16 neighbouring bytes of a row of B and the same 16 bytes of a row of A, and they are its fragments of two instructions, without
// shuffles.  They come by cp.async through a ring in shared memory that belongs to the thread alone, so that the steps to come are always
// in flight and nobody waits for anybody.
// A CTA has 32 rows of B (a block of the copy in 8 bits), its four warps a share of k each; where that leaves too few CTAs, a cluster
// of up to eight shares k once more.  Partial sums are added in the order of the shares: the same bits in every run.
#include "few.cuh"

namespace nvfp4 {

namespace {

constexpr int kWarps = 4, kRows = 32;  // of B

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// MT: groups of eight rows of A;  ST: steps of 32 k that the ring has room for
template <int MT, int ST>
struct Ring {
  static constexpr int kPlane = 32 * kWarps * 16;          // 16 bytes of every thread
  static constexpr int kStep = (4 + MT) * kPlane;          // four rows of B, MT of A
  static constexpr int kPart = kWarps * 8 * MT * (kRows + 1) * 4, kTotal = 8 * MT * kRows * 4;
  static constexpr int kBytes = ST * kStep;
  static_assert(kPart + kTotal <= kBytes, "the sums reuse the ring");
};

// SHARES: an accumulator takes no more than kShareSteps steps, 128 or 256 products, and is then added to sums in registers, rounded to nearest:
// what the instructions cut off grows with the length of a chain, and codes of 8 bits show it.  For calls that keep z in 8 bits.  65536 products of one
// sign in four chains, each a warp's, are 7.6e-5 of the sum off, in shares of 1024 8.7e-7.  Of random ones with 8 x 20480 x 4096 (12 draws) codes
// come out a step off: with the products in binary32 14, with whole chains 87, in shares of 256 / 128 products 27 / 17; 32 x 8192 x 5120 73, 165,
// 31 / 19.  One row x 5120 x 5120 takes 11.4 / 11.8 us (whole chains / these shares), x 20480 42.3 / 43.6, 16 rows 49.4 / 50.7, 32 x 16384 x 16384 120 / 128
// (the registers of the second set of sums).
template <int MT>
constexpr int kShareSteps = MT < 4 ? 4 : 8;
template <int MT, int ST, bool SHARES>
__global__ void __launch_bounds__(32 * kWarps) few_rows_kernel(const FewArgs g) {
  using R = Ring<MT, ST>;
  extern __shared__ __align__(16) uint8_t smem[];
  auto part = reinterpret_cast<float(*)[8 * MT][kRows + 1]>(smem);      // [warp][row of A][row of B]
  auto total = reinterpret_cast<float(*)[kRows]>(smem + R::kPart);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, t = lane & 3;
  const int rank = g.shares > 1 ? (int)cluster_rank() : 0;
  const int n0 = (int)(blockIdx.x / (unsigned)g.shares) * kRows;
  const int steps = (g.K + 31) / 32, share = rank * kWarps + warp, of = g.shares * kWarps;
  const int s0 = (int)((int64_t)steps * share / of), s1 = (int)((int64_t)steps * (share + 1) / of);
  const uint32_t mine = smem_u32(smem) + threadIdx.x * 16;
  // rows that do not exist are never read (copy_async), but their addresses are kept inside the operands
  const uint16_t* brow[4];
  const uint16_t* arow[MT];
  bool blive[4], alive[MT];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    blive[i] = n0 + gid + 8 * i < g.N;
    brow[i] = g.b + (int64_t)(blive[i] ? n0 + gid + 8 * i : 0) * g.ldb;
  }
#pragma unroll
  for (int j = 0; j < MT; ++j) {
    alive[j] = gid + 8 * j < g.M;
    arow[j] = g.a + (int64_t)(alive[j] ? gid + 8 * j : 0) * g.lda;
  }
  auto fetch = [&](int s, int slot) {
    if (s < s1) {
      const int k = s * 32 + t * 8;
      const bool in = k < g.K;
      const uint32_t at = mine + slot * R::kStep;
#pragma unroll
      for (int i = 0; i < 4; ++i) copy_async<16>(at + i * R::kPlane, brow[i] + (in ? k : 0), in && blive[i]);
#pragma unroll
      for (int j = 0; j < MT; ++j) copy_async<16>(at + (4 + j) * R::kPlane, arow[j] + (in ? k : 0), in && alive[j]);
    }
    copy_commit();  // (an empty group where there is no step: the count of groups stays that of the steps)
  };
  griddep_wait();
  constexpr int kOwn = 8 * MT / kWarps;
  const float bias = bias_of(g, n0 + lane);
  float res[kOwn] = {};
  residual_rows(g, res, n0 + lane, warp, kWarps);
#pragma unroll
  for (int u = 0; u < ST - 1; ++u) fetch(s0 + u, u);
  float acc[2][MT][4] = {}, sums[SHARES ? 2 : 1][SHARES ? MT : 1][4] = {};
  int slot = 0, next = ST - 1, until = s0 + kShareSteps<MT>;
  for (int s = s0; s < s1; ++s) {
    if (SHARES && s == until) {
      until += kShareSteps<MT>;
#pragma unroll
      for (int i = 0; i < 8 * MT; ++i) {
        float& a = acc[i / (4 * MT)][i / 4 % MT][i % 4];
        sums[SHARES ? i / (4 * MT) : 0][SHARES ? i / 4 % MT : 0][i % 4] += a;
        a = 0.f;
      }
    }
    copy_wait<ST - 2>();
    const uint32_t at = mine + slot * R::kStep;
    uint4 b[4], a[MT];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = lds16(at + i * R::kPlane);
#pragma unroll
    for (int j = 0; j < MT; ++j) a[j] = lds16(at + (4 + j) * R::kPlane);
    // the slot of the step before: its values have gone into instructions that are issued
    fetch(s + ST - 1, next);
    slot = slot + 1 == ST ? 0 : slot + 1;
    next = next + 1 == ST ? 0 : next + 1;
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int j = 0; j < MT; ++j) {
        const uint4 lo = b[2 * r], hi = b[2 * r + 1];
        mma16816(acc[r][j], lo.x, hi.x, lo.y, hi.y, a[j].x, a[j].y);
        mma16816(acc[r][j], lo.z, hi.z, lo.w, hi.w, a[j].z, a[j].w);
      }
  }
  griddep_launch_dependents();
  copy_wait<0>();
  __syncthreads();  // the rings are empty; the sums take their place
#pragma unroll
  for (int r = 0; r < 2; ++r)
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) part[warp][8 * j + 2 * t + (e & 1)][16 * r + gid + 8 * (e >> 1)] =
            SHARES ? sums[SHARES ? r : 0][SHARES ? j : 0][e] + acc[r][j][e] : acc[r][j][e];
  __syncthreads();
  // a warp to a row of A from here on (rows warp, warp + 4, ...), a lane to a column of D
  float v[kOwn];
#pragma unroll
  for (int j = 0; j < kOwn; ++j) {
    v[j] = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) v[j] += part[w][kWarps * j + warp][lane];
  }
  if (g.shares > 1) {
#pragma unroll
    for (int j = 0; j < kOwn; ++j) total[kWarps * j + warp][lane] = v[j];
    cluster_sync();
    if (rank == 0)
      for (int c = 1; c < g.shares; ++c)
#pragma unroll
        for (int j = 0; j < kOwn; ++j) v[j] += ld_of_rank(&total[kWarps * j + warp][lane], (uint32_t)c);
    cluster_sync();  // none may go while its sums are read
    if (rank != 0) return;
  }
  finish_rows<kOwn>(g, v, res, bias, n0, warp, kWarps, lane);
}

template <int MT, int ST, bool SHARES>
cudaError_t launch_few(const FewArgs& a, cudaStream_t s) {
  auto kern = few_rows_kernel<MT, ST, SHARES>;
  constexpr int smem = Ring<MT, ST>::kBytes;
  static std::atomic<uint64_t> configured{0};  // per instantiation and device
  int dev;
  if (device_needs_config(configured, &dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    device_configured(configured, dev);
  }
  // (with 100 % of the SM as shared memory it has room for three rings)
  const dim3 grid((unsigned)((a.N + kRows - 1) / kRows * a.shares));
  return a.shares > 1 ? launch_cluster((unsigned)a.shares, kern, grid, dim3(32 * kWarps), smem, s, a)
                      : launch_divided(100, kern, grid, dim3(32 * kWarps), smem, s, a);
}
template <int MT, int ST>
cudaError_t launch_few(const FewArgs& a, cudaStream_t s) {
  const int steps = (a.K + 31) / 32, warps = kWarps * a.shares;
  return a.z8.codes && steps > kShareSteps<MT> * warps ? launch_few<MT, ST, true>(a, s) : launch_few<MT, ST, false>(a, s);
}
}  // namespace

cudaError_t launch_gemm_few_rows(const DenseGemmArgs& g, const EpilogueArgs& e, cudaStream_t s) {
  FewArgs a = few_args(g, e);
  int sms = 0;
  const cudaError_t err = sm_count(&sms);
  if (err != cudaSuccess) return err;
  // More shares until there are 1.5 CTAs per SM, as long as all are resident at once (three per SM) and every warp keeps eight steps
  // of k.  1 / 2 / 4 / 8 shares, one row, weights that exceed L2 together: 5120 x 5120 12.3 / 11.5 / 14.7 / 20.2 us, 7168 x 5120 14.0 /
  // 18.6 / 20.4 / 25.5, 2048 x 2048 4.2 / 3.9 / 4.4 / 7.0, 512 x 16384 20.3 / 12.2 / 8.2 / 6.6, 1024 x 1024 3.1 / 3.3 / 3.3 / 3.6.
  const int tiles = (g.N + kRows - 1) / kRows, steps = (g.K + 31) / 32;
  a.shares = 1;
  while (a.shares < 8 && 2 * tiles * a.shares <= 3 * sms && steps >= 8 * kWarps * 2 * a.shares) a.shares *= 2;
  const cudaError_t r = g.M <= 8 ? launch_few<1, 7>(a, s) : g.M <= 16 ? launch_few<2, 6>(a, s) : launch_few<4, 4>(a, s);
  count_launch();
  return r;
}

}  // namespace nvfp4

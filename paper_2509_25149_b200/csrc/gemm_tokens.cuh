// BF16 product of some tens of rows (tokens of many sequences in generation) with a weight, and its epilogue:  z = A B^T + bias,
// D = act(z) + residual, for up to kTokenRows rows of A.  Bound by the bytes of the weight B [N x K]: what counts is that every SM has loads
// of B in flight from the first moment to the last.  The pair kernels have tiles of 256 rows of A, mostly of rows that are not there, and too few
// tiles for the chip; with mma.sync (gemm_few.cu) every 32 rows of B fetch A again.  Here the sides change places: a tile of the tensor core has
// 128 rows of B and as many columns as A has rows (MT, rounded up), D^T = B A^T, one tile to a CTA, and the CTAs of a cluster share k, so that the
// whole chip streams.
// A CTA lives for one tile: one warp fetches (TMA into a ring of k-blocks of 64), one issues, then all four take their 32 rows of B: a
// tensor-memory lane is a column of D.  With shares, row m of the sums goes to the shared memory of rank m mod shares (stores, which nobody waits
// for; read from there by the one that adds them up, 5120 x 5120 and 32 rows took 15.9 us, not 12.9), which adds up its rows in the order of the
// shares, the same bits in every run, and finishes them.
// Two CTAs to an SM with rings of 96 to 100 KB: 20480 x 5120 (160 tiles), 64 rows 40.6 us; one with a ring of 192 KB 57.2.
// 64 rows: 20480 x 5120 40.6 us (5.2 TB/s, 79 % of the copy rate), 5120 x 20480 39.0, 5120 x 5120 14.7 (3.6 TB/s: 4 us are launch, first trip to memory
// and exchange); pair kernels 59.3, 88, 25.3.
// Included by gemm.cu only.
#pragma once

#include "few.cuh"
#include "tc_ptx.cuh"

namespace nvfp4 {
namespace tokens {

constexpr int kThreads = 128, kCols = 128;  // columns of D: rows of B

__device__ __forceinline__ void tc_ld8(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
}

template <int MT, int ST>
struct Cfg {
  static constexpr int kStage = (kCols + MT) * 128;  // 64 k of bf16
  static constexpr int kBytes = ST * kStage + 1024 /*alignment*/ + 256 /*barriers*/;
  static_assert((MT + 7) * kCols * 4 <= ST * kStage, "the sums reuse the ring");
  static_assert(kBytes <= 232448, "shared memory budget");
  static_assert(2 * ST + 2 <= 30, "barriers");
  static_assert(MT >= 32 && (MT & (MT - 1)) == 0, "columns of tensor memory");
};

__device__ __forceinline__ void mma_bf16(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// Accumulators of a CTA, all that two to an SM leave room for.
template <int MT>
constexpr int kAccs = 256 / MT;

// ACCS: a CTA's k-blocks go to several accumulators, g.chain blocks to each, and what these hold is added rounded to nearest (for codes of 8 bits, see
// code_share in gemm.h): nothing waits, since each is written in one run and read at the end.  16 x 8192 x 4096 (16 draws): 11 codes a step off for 18 of
// products in binary32 (with one accumulator 85), 64 x 5120 x 20480 87 for 159.  64 x 5120 x 5120 16.8 / 16.9 us (one / several), 16 rows 13.1 / 13.6; longer
// contractions, which one accumulator was too short for, 64 x 5120 x 20480 95 (pair kernel) / 41.8, 32 rows 59.6 (gemm_few.cu) / 38.4.
template <int MT, int ST, bool ACCS>
__global__ void __launch_bounds__(kThreads) tokens_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
                                                          const __grid_constant__ FewArgs g) {
  using C = Cfg<MT, ST>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* const base_ptr = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t bar_base = base + ST * C::kStage;
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (ST + s); };
  const uint32_t acc_bar = bar_base + 8u * (2 * ST);
  volatile uint32_t* const tmem_slot = reinterpret_cast<volatile uint32_t*>(base_ptr + ST * C::kStage + 8 * (2 * ST + 1));
  volatile uint32_t* const abort_flag = tmem_slot + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = g.shares > 1 ? (int)cluster_rank() : 0;
  const int n0 = (int)(blockIdx.x / (unsigned)g.shares) * kCols;
  const int blocks = (g.K + 63) / 64, tiles = (g.N + kCols - 1) / kCols;
  const uint32_t columns = MT * (ACCS ? kAccs<MT> : 1);
  const int k0 = (int)((int64_t)blocks * rank / g.shares), k1 = (int)((int64_t)blocks * (rank + 1) / g.shares);  // (never empty: see the launch)

  if (threadIdx.x == 0) {
    for (int s = 0; s < ST; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    mbar_init(acc_bar, 1);
    *abort_flag = 0;
    fence_mbarrier_init();
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (threadIdx.x == 96) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_w) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_x) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void*)tmem_slot)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  griddep_wait();
  griddep_launch_dependents();

  if (warp == 0 && lane == 0) {
    int stage = 0;
    uint32_t phase = 0;
    // With few rows of A all CTAs would want the same few lines of it from L2 at the same time, so each begins somewhere else: 20480 x 5120, one row
    // 45.2 us without, 35.3 with; 16 rows 35.6 / 36.1.
    int kb = g.M <= 8 ? k0 + (int)((int64_t)(k1 - k0) * (n0 / kCols) / tiles) : k0;
    for (int left = k1 - k0; left > 0; --left) {
      if (!mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag, 0xF00u + stage)) break;
      const uint32_t st = base + stage * C::kStage;
      mbar_expect_tx(full_bar(stage), C::kStage);  // (rows and k that are not there count: they come as zeros)
      tma_load_2d(st, &map_w, kb * 64, n0, full_bar(stage));
      tma_load_2d(st + kCols * 128, &map_x, kb * 64, 0, full_bar(stage));
      if (++kb == k1) kb = k0;
      if (++stage == ST) {
        stage = 0;
        phase ^= 1u;
      }
    }
  } else if (warp == 1 && lane == 0) {
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    const uint32_t w_lo0 = ((base >> 4) & 0x3fffu) | (1u << 16), x_lo0 = (((base + kCols * 128) >> 4) & 0x3fffu) | (1u << 16);
    constexpr uint32_t idesc = dense::instr_desc_bf16(kCols, MT, 0, 0);
    uint32_t d = tmem;
    int left = ACCS ? g.chain : 0;
    bool first = true;
    for (int kb = k0; kb < k1; ++kb) {
      if (ACCS && left-- == 0) {
        left = g.chain - 1;
        first = true;
        d += MT;
      }
      if (!(ok = mbar_wait(full_bar(stage), phase, abort_flag, 0xF20u + stage))) break;
      tc_fence_after();
      const uint32_t at = stage * (C::kStage >> 4);
#pragma unroll
      for (int j = 0; j < 4; ++j)  // 16 k: 32 bytes further inside the 128-byte swizzle span
        mma_bf16(d, make_desc(w_lo0 + at + 2 * j, kDescHiOperand), make_desc(x_lo0 + at + 2 * j, kDescHiOperand), idesc,
                 !first || j > 0 ? 1u : 0u);
      first = false;
      tc_commit(empty_bar(stage));
      if (++stage == ST) {
        stage = 0;
        phase ^= 1u;
      }
    }
    if (ok) tc_commit(acc_bar);  // the sums are complete, and the ring has been read
  }
  __syncwarp();
  const int nw = n0 + 32 * warp;
  constexpr int kOwn = 8;  // rows that a warp finishes at a time
  const float bias = bias_of(g, nw + lane);
  float res[kOwn] = {}, next[kOwn] = {};
  residual_rows(g, res, nw + lane, rank, g.shares);
  bool ok = mbar_wait(acc_bar, 0, abort_flag, 0xF40u);
  ok = __all_sync(0xffffffffu, ok);
  tc_fence_after();
  const uint32_t row = tmem + ((uint32_t)(32 * warp) << 16);
  const int accs = ACCS ? (k1 - k0 + g.chain - 1) / g.chain : 1;
  if (g.shares > 1) {
    // Row m goes to rank m mod shares, as its row m / shares of this share: [share][row][row of B]
    const int own = (g.M + g.shares - 1) / g.shares;
    cluster_sync();  // every ring has been read; the sums take their place
    if (ok) {
      const uint32_t to = base + (uint32_t)((rank * own * kCols + 32 * warp + lane) * 4);
      int owner = 0;
      uint32_t at = to;
#pragma unroll 1
      for (int c = 0; c < g.M; c += 32) {
        uint32_t r[32];
        tc_ld32(row + c, r);
        tc_wait_ld();
        if (ACCS)
#pragma unroll 1
          for (int a = 1; a < accs; ++a) {
            uint32_t more[32];
            tc_ld32(row + a * MT + c, more);
            tc_wait_ld();
#pragma unroll
            for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(__uint_as_float(r[j]) + __uint_as_float(more[j]));
          }
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          if (c + j < g.M) st_of_rank(at, (uint32_t)owner, r[j]);
          if (++owner == g.shares) {
            owner = 0;
            at += kCols * 4;
          }
        }
      }
    }
    cluster_sync();
    if (ok && nw < g.N) {
      const float* const mine = reinterpret_cast<const float*>(base_ptr) + 32 * warp + lane;
      for (int i = 0; rank + i * g.shares < g.M; i += kOwn) {
        float v[kOwn] = {};
        residual_rows(g, next, nw + lane, rank + (i + kOwn) * g.shares, g.shares);
        for (int c = 0; c < g.shares; ++c)
#pragma unroll
          for (int j = 0; j < kOwn; ++j)
            if (i + j < own) v[j] += mine[(c * own + i + j) * kCols];
        finish_rows<kOwn>(g, v, res, bias, nw, rank + i * g.shares, g.shares, lane);
#pragma unroll
        for (int j = 0; j < kOwn; ++j) res[j] = next[j];
      }
    }
  } else if (ok && nw < g.N) {
#pragma unroll 1
    for (int c = 0; c < g.M; c += kOwn) {
      uint32_t r[kOwn];
      tc_ld8(row + c, r);
      residual_rows(g, next, nw + lane, c + kOwn, 1);
      tc_wait_ld();
      float v[kOwn];
#pragma unroll
      for (int j = 0; j < kOwn; ++j) v[j] = __uint_as_float(r[j]);
      if (ACCS)
#pragma unroll 1
        for (int a = 1; a < accs; ++a) {
          tc_ld8(row + a * MT + c, r);
          tc_wait_ld();
#pragma unroll
          for (int j = 0; j < kOwn; ++j) v[j] += __uint_as_float(r[j]);
        }
      finish_rows<kOwn>(g, v, res, bias, nw, c, 1, lane);
#pragma unroll
      for (int j = 0; j < kOwn; ++j) res[j] = next[j];
    }
  }
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    // give copies that may still be in flight time to land before the shared memory is handed back
    for (int i = 0; i < 100; ++i) __nanosleep(1000);
  }
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns) : "memory");
  }
}

}  // namespace tokens
}  // namespace nvfp4

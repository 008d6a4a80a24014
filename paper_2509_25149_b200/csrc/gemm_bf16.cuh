// BF16 GEMM on CTA pairs (tcgen05 cta_group::2, kind::f16) for the linear layers the recipe leaves in higher
// precision (Section 4.1: the most sensitive layers stay in BF16; Appendix D: every layer late in training).
//   D[M x N] = A * B^T, FP32 accumulation in tensor memory, bf16 or fp32 output, optional accumulation into D.
// Same persistent structure as the block-scaled pair kernel (256 x 256 tiles, each CTA holding its 128 rows of A
// and half of the B tile) minus the scale path; the tensor-memory columns the scales would take hold a second
// accumulator, so a tile's epilogue runs entirely under the next tile's main loop.
//
// Operand layouts.  An operand is "K-major" when the contraction index is contiguous in memory (A stored [M][K],
// B stored [N][K]) and "MN-major" when the output index is (A stored [K][M], B stored [K][N]).  The three GEMMs of a
// layer with row-major X [M x K], W [N x K], dY [M x N] need no transposed copies:
//   Fprop  Y  = X  W^T : A = X  K-major,  B = W  K-major
//   Dgrad  dX = dY W   : A = dY K-major,  B = W  MN-major (contraction over N, W's rows)
//   Wgrad  dW = dY^T X : A = dY MN-major, B = X  MN-major (contraction over the tokens, the rows of both)
// Shared-memory tiles per stage (K = 64 elements): K-major  128 rows x 128 bytes, 128-byte swizzle, 8-row groups
// 1024 bytes apart; MN-major two boxes of 64 k-rows x 128 bytes (64 contiguous output indices each), 8 KB apart.
// One instruction covers K = 16: 32 bytes further along a K-major row, two 8-row groups further in an MN-major box.
// Included by gemm.cu only.
#pragma once

#include "act.cuh"
#include "copy8.cuh"
#include "gemm_2cta.cuh"

namespace nvfp4 {
namespace dense {

constexpr int kThreads = 320;       // producer, MMA issuer, 2 x 4 epilogue warps
constexpr int kOperandBytes = 128 * 128;           // 128 rows (or output indices) x 64 bf16
constexpr int kStagingBytes = 2 * 16384;
template <int BN, int SPLIT>
struct Cfg {
  static constexpr int kStages = BN == 512 ? 4 : 6;
  // A, this CTA's half of B.  (32 KB for the narrow tile as well: 24 KB apart, 1024 x 1280 x 4096 takes 24.3 us, not 23.9)
  static constexpr int kStageBytes =
      SPLIT > 1 ? kOperandBytes + BN / 2 * 128 : BN == 512 ? 3 * kOperandBytes : 2 * kOperandBytes;
  static constexpr int kRecvBytes = (SPLIT - 1) * 128 * (BN / SPLIT) * 4;
  static constexpr int kSmemBytes = kStages * kStageBytes + kStagingBytes + 1024 /*alignment*/ + 256 /*barriers*/ + kRecvBytes;
  static_assert(kSmemBytes <= 232448, "shared memory budget");
};
constexpr uint32_t kTmemCols = 512;                // two 256-column accumulators

struct Problem {
  int M, N, K;
  int a_mn, b_mn;  // 1 = the operand is stored with the output index contiguous
  int d_is_fp32, accumulate;
};
// One launch works through the tiles of up to two independent products: Dgrad and Wgrad of a layer fill each other's partial last
// round (4088 x 5128 x 5112: 5 + 6 rounds of 256-wide tiles on 74 pairs become 10).
struct Args {
  Problem p[2];
  int n_tiles0;  // tiles of problem 0, which come first (BN < 512)
  int n_tiles;   // tiles of both problems
  // BN = 512: tiles 512 columns wide of problem 0 and 1, then the tiles 256 wide of both, and where each of these four ends
  int wide_n[2];  // column tiles 512 wide of each problem
  int seg_end[4];
  int share;  // SHARES: k-blocks that an accumulator takes at most
};

// What follows a product: z = A B^T + bias, D = act(z) + residual, z kept in bf16 or as a copy in 8 bits (a launch with one problem)
struct NoEpilogue {
  static constexpr bool kFused = false, kBuffers = false;
  static constexpr int kSmemBytes = 0;
};
struct Epilogue {
  static constexpr bool kFused = true, kBuffers = false;
  static constexpr int kSmemBytes = 2 * 128 * 4;  // the bias of a tile's columns, one half per epilogue group
  CUtensorMap map_r, map_z;  // residual and z: the boxes that D is stored in
  const float* bias;
  uint8_t* z8_codes;
  uint8_t* z8_scales;
  int z8_blocks;  // scale bytes of a row
  int act, has_residual, has_z;
};

// 256 x 256 tiles with a residual: a stage of the main loop's ring makes room for buffers of 16 KB per epilogue group, so that both chunks
// of a tile's residual are fetched while its main loop runs.
struct EpilogueBuffers : Epilogue {
  static constexpr bool kBuffers = true;
  static constexpr int kSmemBytes = Epilogue::kSmemBytes + 2 * 16384;
};

template <int ACT, int COLS>
__device__ __forceinline__ void activate(uint32_t (&r)[COLS]) {
#pragma unroll
  for (int j = 0; j < COLS; ++j) r[j] = __float_as_uint(act_value<ACT>(__uint_as_float(r[j])));
}

// COLS columns of one row as a copy in 8 bits, from the registers: a thread has whole blocks, so their maxima need no exchange.  Columns
// behind N are zeros in r.  Where N is a multiple of 32 a thread stores the 32 bytes of a block, a sector, itself; else the warp turns its 32
// rows round in the staging buffer and stores them row by row.  The whole group calls; buf: the group's staging buffer.
template <int COLS>
__device__ __forceinline__ void store_rows8(const uint32_t (&r)[COLS], const Epilogue& e, int row_in_tile, int row0, int M, int x0, int N,
                                            bool wide, uint32_t buf, int et, int bar_id) {
  const int64_t row = row0 + row_in_tile;
  const bool live = row < M;
  uint32_t bytes = 0;
  uint8_t* const scales = e.z8_scales + row * e.z8_blocks + (x0 >> 5);
  const bool word = COLS == 128 && (e.z8_blocks & 3) == 0;
  constexpr int kUnits = COLS / 16;  // of 16 codes in a staged row
  const uint32_t srow = buf + row_in_tile * COLS;
  if (!wide) {
    if (et == 0) pair::bulk_wait_read<0>();  // the stores before have read the buffer
    asm volatile("bar.sync %0, 128;" ::"r"(bar_id) : "memory");
  }
#pragma unroll
  for (int b = 0; b < COLS / 32; ++b) {
    const int x = x0 + 32 * b;
    if (x >= N) break;
    float m = 0.f;
#pragma unroll
    for (int j = 0; j < 32; j += 2) m = amax3(m, __uint_as_float(r[32 * b + j]), __uint_as_float(r[32 * b + j + 1]));
    const uint32_t byte = scale_byte8(m);
    const float2 scale = both(encode_scale8(byte));
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t* const q = &r[32 * b + 4 * j];
      const float2 lo = mul2(make_float2(__uint_as_float(q[0]), __uint_as_float(q[1])), scale);
      const float2 hi = mul2(make_float2(__uint_as_float(q[2]), __uint_as_float(q[3])), scale);
      w[j] = e4m3x4(lo.x, lo.y, hi.x, hi.y);
    }
    if (wide) {
      if (live)
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(e.z8_codes + row * N + x), "r"(w[0]), "r"(w[1]),
                     "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                     : "memory");
    } else {
#pragma unroll
      for (int u = 0; u < 2; ++u)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(srow + (((2 * b + u) ^ (row_in_tile & (kUnits - 1))) << 4)),
                     "r"(w[4 * u]), "r"(w[4 * u + 1]), "r"(w[4 * u + 2]), "r"(w[4 * u + 3])
                     : "memory");
    }
    if (word)
      bytes |= byte << (8 * b);
    else if (live)
      scales[b] = (uint8_t)byte;
  }
  if (word && live && x0 < N) *reinterpret_cast<uint32_t*>(scales) = bytes;
  if (wide) return;
  __syncwarp();
  constexpr int kPieces = COLS / 8, kRowsAtOnce = 32 / kPieces;  // of eight codes
  const int lane = row_in_tile & 31, first = row_in_tile - lane, p = lane % kPieces;
#pragma unroll
  for (int k = 0; k < 32; k += kRowsAtOnce) {
    const int rr = first + k + lane / kPieces;
    if (row0 + rr < M && x0 + 8 * p < N)
      *reinterpret_cast<uint2*>(e.z8_codes + (int64_t)(row0 + rr) * N + x0 + 8 * p) =
          lds8(buf + rr * COLS + (((p >> 1) ^ (rr & (kUnits - 1))) << 4) + 8 * (p & 1));
  }
  // what comes into the buffer next, by a thread or by TMA, comes behind these reads
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  asm volatile("bar.sync %0, 128;" ::"r"(bar_id) : "memory");
}

// Units of 16 bytes of a staged row, as store_half() has them for bf16
template <int COLS>
constexpr int kStagedUnits = COLS < 64 ? 4 : 8;

// A chunk of the residual into a buffer of the group, once the stores before have read it (one thread)
template <int COLS>
__device__ __forceinline__ void load_residual(const Epilogue& e, uint32_t buf, int x, int row0, uint32_t res_bar) {
  pair::bulk_wait_read<0>();
  mbar_expect_tx(res_bar, 128 * 16 * kStagedUnits<COLS>);
  tma_load_2d(buf, &e.map_r, x, row0, res_bar);
}
// z, or a copy of it that a warp turns round, goes through the staging buffer before the residual may come there
__device__ __forceinline__ bool z_is_staged(const Epilogue& e, bool wide8) { return e.has_z || (e.z8_codes && !wide8); }

// The epilogue of COLS columns of one row per thread.  The residual comes by TMA, chunk c into the staging buffer (BUFFERS: the second into
// res_buf), in the place from which the sum then leaves: a thread reads and writes its own row.  prefetched: the first chunk (BUFFERS: the
// second in any case) is on its way.  false: a wait ran out (all 128 threads agree).
template <int COLS, bool BUFFERS>
__device__ __forceinline__ bool finish_half(uint32_t (&r)[COLS], const Epilogue& e, const float* bias, int M, int N, int et, int bar_id,
                                            int row_in_tile, uint32_t stage_buf, uint32_t res_buf, const CUtensorMap* map_d, int x0,
                                            int row0, uint32_t res_bar, uint32_t& res_phase, bool wide8, bool prefetched,
                                            volatile uint32_t* abort_flag) {
  if (e.bias) {
#pragma unroll
    for (int j = 0; j < COLS; j += 4) {
      const float4 b = *reinterpret_cast<const float4*>(bias + j);
      r[j] = __float_as_uint(__uint_as_float(r[j]) + b.x);
      r[j + 1] = __float_as_uint(__uint_as_float(r[j + 1]) + b.y);
      r[j + 2] = __float_as_uint(__uint_as_float(r[j + 2]) + b.z);
      r[j + 3] = __float_as_uint(__uint_as_float(r[j + 3]) + b.w);
    }
  }
  if (e.z8_codes) store_rows8<COLS>(r, e, row_in_tile, row0, M, x0, N, wide8, stage_buf, et, bar_id);
  if (e.has_z) pair::store_half<false, false, COLS>(r, 1.0f, et, bar_id, row_in_tile, stage_buf, &e.map_z, x0, row0, 0, false);
  switch (e.act) {
    case NVFP4_ACT_RELU2: activate<NVFP4_ACT_RELU2>(r); break;
    case NVFP4_ACT_SILU: activate<NVFP4_ACT_SILU>(r); break;
    case NVFP4_ACT_GELU: activate<NVFP4_ACT_GELU>(r); break;
    default: break;
  }
  if (!e.has_residual) {
    pair::store_half<false, false, COLS>(r, 1.0f, et, bar_id, row_in_tile, stage_buf, map_d, x0, row0, 0, false);
    return true;
  }
  constexpr int kUnits = kStagedUnits<COLS>, kChunkCols = 8 * kUnits;
#pragma unroll
  for (int c = 0; c < COLS / kChunkCols; ++c) {
    const bool second = BUFFERS && c == 1;
    const uint32_t buf = second ? res_buf : stage_buf, bar = res_bar + (second ? 16u : 0u);
    if (et == 0 && !second && !(c == 0 && prefetched)) load_residual<COLS>(e, buf, x0 + c * kChunkCols, row0, bar);
    mbar_wait(bar, (res_phase >> (second ? 1 : 0)) & 1u, abort_flag, 0xE00u);
    res_phase ^= second ? 2u : 1u;
    if (group_gave_up(abort_flag, bar_id, 128)) return false;
    const uint32_t srow = buf + row_in_tile * (16 * kUnits);
    const uint32_t x = kUnits == 4 ? (row_in_tile >> 1) & 3 : row_in_tile & 7;  // (the swizzles of store_half)
#pragma unroll
    for (int j = 0; j < kUnits; ++j) {
      const uint32_t at = srow + ((j ^ x) << 4);
      const uint4 w = pair::lds128(at);
      const uint32_t in[4] = {w.x, w.y, w.z, w.w};
      uint32_t p[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        p[k] = pack2(__uint_as_float(r[c * kChunkCols + 8 * j + 2 * k]) + bf16_lo(in[k]),
                     __uint_as_float(r[c * kChunkCols + 8 * j + 2 * k + 1]) + bf16_hi(in[k]));
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(p[0]), "r"(p[1]), "r"(p[2]), "r"(p[3]) : "memory");
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    asm volatile("bar.sync %0, 128;" ::"r"(bar_id) : "memory");
    if (et == 0) {
      pair::tma_store_2d(map_d, x0 + c * kChunkCols, row0, buf);
      pair::bulk_commit();
    }
  }
  return true;
}

// kind::f16 instruction descriptor: FP32 accumulator (bit 4), BF16 x BF16 (format 1 at bits 7 and 10), operand
// major-ness at bits 15 / 16 (0 = K-major), N >> 3 at bit 17, M >> 4 at bit 24
__host__ __device__ constexpr uint32_t instr_desc_bf16(int m, int n, int a_mn, int b_mn) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) |
         ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

__device__ __forceinline__ void tc2_mma_bf16(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc,
                                             uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// BN: columns of a tile (512, 256 or 128).  BN = 512: two accumulators side by side share the loads of A, 48 KB per k-block and
// CTA instead of 64; what is left of the columns, and what balances the rounds better, is taken in tiles of 256 (bf16_wide_tiles).
// That is for operands whose rows do not all begin on 32 bytes: a 128-byte row of a box that does not takes 1.75 times as long on the
// SM's path to L2 (with rows an odd multiple of 16 bytes apart 1.375 on average), and 256-wide tiles wait for it.
// The two halves of such a tile begin and end apart (kLead): the epilogue drains one while the tensor pipe works on the other.
// SPLIT > 1 (BN = 128): a cluster of SPLIT pairs takes one tile, the only one of its life,
// each pair a share of the k-blocks (the exchange: pair::exchange_columns).
// TWO: the launch has two problems.
// E: Epilogue (EpilogueBuffers) or NoEpilogue.
// SHARES: an accumulator takes no more than Args::share k-blocks.  Then the issuer goes on in the other one, and the epilogue warps add what it
// holds to sums of their own, rounded to nearest.  The tensor cores cut off what an addition to an accumulator cannot hold, an error that
// grows with every one of them: a weight gradient over 16384 tokens (values of an 8-bit copy) is 8.6e-6 off in the mean square, 3.1e-5 where all
// terms have one sign; in shares of 8 / 16 k-blocks 1.9e-7 / 2.3e-7 and 3.9e-7 / 6.3e-7.  Weight gradients take shares of kShare, 1024 products;
// codes of 8 bits want shorter ones where the contraction is short (code_share in gemm.h).  What it costs is waiting for the epilogue of the tile
// before, and the power of reading the accumulators more often: 8192 x 20480 x 5120 with codes of 8 bits, in a loop at the power limit, 1326 us in one
// sum, in shares of 8 / 12 / 16 1365 / 1302 / 1288 (on another GPU 1410 / 1360 / 1340); x 2048 591 / 560 / 552; x 1024 333 / 328 / 315 (one share); x 512
// 237 in one share, 252 in shares of 4.
// Not for 512-wide tiles, whose halves need both accumulators.
constexpr int kShare = 16;
template <int BN, int SPLIT = 1, bool TWO = true, class E = NoEpilogue, bool SHARES = false>
__global__ void __cluster_dims__(2 * SPLIT, 1, 1) __launch_bounds__(kThreads, 1)
    gemm_bf16_pair_kernel(const __grid_constant__ CUtensorMap map_a0, const __grid_constant__ CUtensorMap map_b0,
                          const __grid_constant__ CUtensorMap map_d0, const __grid_constant__ CUtensorMap map_a1,
                          const __grid_constant__ CUtensorMap map_b1, const __grid_constant__ CUtensorMap map_d1,
                          const __grid_constant__ Args g, const __grid_constant__ E e) {
  static_assert(!E::kFused || !TWO, "an epilogue belongs to one product");
  static_assert(!SHARES || BN < 512, "two accumulators in turn");
  using namespace pair;
  static_assert(!E::kBuffers || (BN == 256 && SPLIT == 1), "two chunks to a group");
  constexpr int S = dense::Cfg<BN, SPLIT>::kStages - (E::kBuffers ? 1 : 0), kStageBytes = dense::Cfg<BN, SPLIT>::kStageBytes;
  constexpr bool kDouble = BN == 512;        // two 256-column halves
  constexpr int HN = kDouble ? 256 : BN;     // columns of an accumulator
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* base_ptr = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t staging = base + S * kStageBytes;
  constexpr int kBarOffset = S * kStageBytes + dense::kStagingBytes + (E::kBuffers ? 32768 : 0);
  const uint32_t bar_base = base + kBarOffset;
  auto full_bar = [&](int s) { return bar_base + 8u * s; };              // leader only: both CTAs' operands landed
  auto empty_bar = [&](int s) { return bar_base + 8u * (S + s); };       // one per CTA
  auto accf_bar = [&](int b) { return bar_base + 8u * (2 * S + b); };    // one per CTA and accumulator
  auto acce_bar = [&](int b) { return bar_base + 8u * (2 * S + 2 + b); };  // leader only, 16 arrivals
  const uint32_t done_bar = bar_base + 8u * (2 * S + 4);
  const uint32_t recv_bar = done_bar + 16;                               // SPLIT > 1: all shares are here
  auto res_bar = [&](int group) { return done_bar + 24u + 8u * group; };  // E: a chunk of the residual is here (kBuffers: the second, + 16)
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(
      base_ptr + kBarOffset + 8 * (2 * S + 5));
  volatile uint32_t* abort_flag = tmem_slot + 1;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t cta = cluster_ctarank();
  const uint32_t rank = SPLIT > 1 ? cta & 1u : cta;          // in the pair, 0 = leader
  const uint32_t leader_cta = SPLIT > 1 ? cta & ~1u : 0u;    // the leader's rank in the cluster
  const uint16_t pair_mask = (uint16_t)(3u << leader_cta);   // both CTAs of the pair
  const int split = SPLIT > 1 ? (int)(cta >> 1) : 0;         // which share of the contraction
  const bool leader = rank == 0;
  const int pair_id = blockIdx.x / (2 * SPLIT), n_pairs = gridDim.x / (2 * SPLIT);  // (SPLIT > 1: clusters)
  // ragged edges: loads beyond the operands read zeros, stores beyond D are clipped (both by the tensor maps)
  const int n_tiles = g.n_tiles;
  auto prob_of = [&](int tile) {
    if (kDouble) return TWO ? ((tile >= g.seg_end[0] && tile < g.seg_end[1]) || tile >= g.seg_end[2] ? 1 : 0) : 0;
    return TWO && tile >= g.n_tiles0 ? 1 : 0;
  };
  auto halves_of = [&](int tile) { return kDouble && tile < g.seg_end[1] ? 2 : 1; };
  auto k_begin = [&](int tile, int s) {  // first k-block of share s
    const int n = (g.p[prob_of(tile)].K + 63) / 64;
    return SPLIT > 1 ? n * s / SPLIT : n * s;
  };
  // rounds of the pairs; kDouble: odd ones in reverse order, which evens out tiles of different cost
  auto next_tile = [&](int rnd) { return rnd * n_pairs + (kDouble && (rnd & 1) ? n_pairs - 1 - pair_id : pair_id); };
  // groups of eight row-blocks sweep all column-blocks before the next group starts (L2 reuse of A and B);
  // n_blk: the tile's first column in units of HN
  constexpr int kGroupM = 8;
  auto tile_coords = [&](int tile, int& prob, int& m_blk, int& n_blk) {
    prob = prob_of(tile);
    int tiles_n = (g.p[prob].N + HN - 1) / HN, n_first = 0, n_step = 1;
    if constexpr (kDouble) {
      const int seg = (tile >= g.seg_end[0]) + (tile >= g.seg_end[1]) + (tile >= g.seg_end[2]);
      if (seg) tile -= g.seg_end[seg - 1];
      if (seg < 2) {
        tiles_n = g.wide_n[prob];
        n_step = 2;
      } else {
        n_first = 2 * g.wide_n[prob];
        tiles_n -= n_first;
      }
    } else if (prob) {
      tile -= g.n_tiles0;
    }
    const int tiles_m = (g.p[prob].M + 255) / 256;
    const int per_group = kGroupM * tiles_n;
    const int grp = tile / per_group, in_grp = tile - grp * per_group;
    const int m0 = grp * kGroupM;
    const int gm = (tiles_m - m0 < kGroupM) ? (tiles_m - m0) : kGroupM;
    m_blk = m0 + in_grp % gm;
    n_blk = n_first + n_step * (in_grp / gm);
  };

  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(full_bar(s), 2);  // one arrive.expect_tx from each CTA's producer
      mbar_init(empty_bar(s), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(accf_bar(b), 1);
      mbar_init(acce_bar(b), 16);  // eight epilogue warps in each CTA
    }
    mbar_init(done_bar, 2 * SPLIT - 1);
    if (SPLIT > 1) mbar_init(recv_bar, 1);
    if (E::kFused)
      for (int b = 0; b < 4; ++b) mbar_init(res_bar(b), 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    if (SPLIT > 1) mbar_expect_tx(recv_bar, dense::Cfg<BN, SPLIT>::kRecvBytes);
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void*)tmem_slot)),
                 "r"(dense::kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // both CTAs' barriers are initialised before any remote signal
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  griddep_wait();  // the set-up above ran beside the previous kernel; from here on its output is touched
  griddep_launch_dependents();

  if (warp == 0) {
    // ------------------------------------------------------------------ producer ----
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int rnd = 0, tile = pair_id; tile < n_tiles && ok; tile = next_tile(++rnd)) {
        int prob, m_blk, n_blk;
        tile_coords(tile, prob, m_blk, n_blk);
        const int row_a = m_blk * 256 + (int)rank * 128;  // this CTA's rows of A
        const int row_b = n_blk * HN + (int)rank * (HN / 2);  // this CTA's half of the B tile (of its first 256 columns)
        const int halves = halves_of(tile);
        const int k_end = k_begin(tile, split + 1);
        // One copy of the loop for each problem of the launch, with its tensor maps and layouts at fixed places of the parameter
        // bank: with the maps picked by pointer the loads of a stage were issued so late that a pair could not go faster even
        // when it had L2 to itself (last rounds): forward of 3632 x 1552 x 3136 41.0 us, now 35.4, backward 67.6, now 63.4.
        auto load_tile = [&](const CUtensorMap* map_a, const CUtensorMap* map_b, const Problem& pr) {
          for (int kb = k_begin(tile, split); kb < k_end; ++kb) {
            if (!(ok = mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag, 0x900u + stage))) break;
            const uint32_t st = base + stage * kStageBytes;
            const uint32_t bar = map_to_cta(full_bar(stage), leader_cta);  // the leader's barrier counts both CTAs' operands
            mbar_expect_tx_cluster(bar, dense::kOperandBytes + (kDouble ? halves * dense::kOperandBytes : BN / 2 * 128));
            if (pr.a_mn) {
              tma_load_2d_pair(st, map_a, row_a, kb * 64, bar);
              tma_load_2d_pair(st + 8192, map_a, row_a + 64, kb * 64, bar);
            } else {
              tma_load_2d_pair(st, map_a, kb * 64, row_a, bar);
            }
#pragma unroll
            for (int h = 0; h < (kDouble ? 2 : 1); ++h) {
              if (h >= halves) break;
              const uint32_t st_b = st + (1 + h) * dense::kOperandBytes;
              if (pr.b_mn) {
                tma_load_2d_pair(st_b, map_b, row_b + 256 * h, kb * 64, bar);
                if (HN == 256) tma_load_2d_pair(st_b + 8192, map_b, row_b + 256 * h + 64, kb * 64, bar);
              } else {
                tma_load_2d_pair(st_b, map_b, kb * 64, row_b + 256 * h, bar);
              }
            }
            if (++stage == S) {
              stage = 0;
              phase ^= 1u;
            }
          }
        };
        if (!TWO || prob == 0)
          load_tile(&map_a0, &map_b0, g.p[0]);
        else
          load_tile(&map_a1, &map_b1, g.p[1]);
      }
    }
  } else if (warp == 1) {
    // ---------------------------------------------------------------- MMA issuer (leader) ----
    if (leader && lane == 0) {
      int stage = 0;
      uint32_t phase = 0, acc_phase = 0;  // bit b: phase of accumulator b's barrier
      bool ok = true;
      // descriptor halves: start address and leading byte offset (low word), stride byte offset / version /
      // 128-byte swizzle (high word).  K-major: 8-row groups 1024 bytes apart, leading offset unused.  MN-major:
      // 64-index boxes 8192 bytes apart (leading), 8-row k groups 1024 bytes apart (stride).
      const uint32_t a_lo_base = (base >> 4) & 0x3fffu, b_lo_base = ((base + dense::kOperandBytes) >> 4) & 0x3fffu;
      int buf = 0;
      auto acc_free = [&](int b) {
        return mbar_wait_cluster(acce_bar(b), ((acc_phase >> b) & 1u) ^ 1u, abort_flag, 0xB00u + b);
      };
      for (int rnd = 0, tile = pair_id; tile < n_tiles && ok; tile = next_tile(++rnd)) {
        const bool both = halves_of(tile) == 2;
        if (both) buf = 0;
        if (!(ok = acc_free(buf))) break;
        tc_fence_after();
        const int k_blocks = k_begin(tile, split + 1) - k_begin(tile, split);
        // (one copy of the loop for each problem, as in the producer)
        auto main_loop = [&](const Problem& pr) {
          const uint32_t idesc = instr_desc_bf16(256, HN, pr.a_mn, pr.b_mn);
          const uint32_t a_lo0 = a_lo_base | ((pr.a_mn ? (8192u >> 4) : 1u) << 16);
          const uint32_t b_lo0 = b_lo_base | ((pr.b_mn ? (8192u >> 4) : 1u) << 16);
          const uint32_t a_step = pr.a_mn ? (2048u >> 4) : (32u >> 4);  // one K = 16 instruction further
          const uint32_t b_step = pr.b_mn ? (2048u >> 4) : (32u >> 4);
          auto mma = [&](int st, int half, int acc, bool first) {  // a k-block of one half
            const uint32_t a_lo = a_lo0 + st * (kStageBytes >> 4);
            const uint32_t b_lo = b_lo0 + st * (kStageBytes >> 4) + half * (dense::kOperandBytes >> 4);
#pragma unroll
            for (int j = 0; j < 4; ++j)
              tc2_mma_bf16(tmem + acc * 256, make_desc(a_lo + j * a_step, kDescHiOperand),
                           make_desc(b_lo + j * b_step, kDescHiOperand), idesc, (!first || j > 0) ? 1u : 0u);
          };
          auto landed = [&](int st, uint32_t ph) {
            if (!(ok = mbar_wait_cluster(full_bar(st), ph, abort_flag, 0xA00u + st))) return false;
            tc_fence_after();
            return true;
          };
          auto release = [&] {
            tc2_commit_both(empty_bar(stage), pair_mask);  // both CTAs' stages are free once these MMAs have read them
            if (++stage == S) {
              stage = 0;
              phase ^= 1u;
            }
          };
          if constexpr (kDouble) {
            if (both) {
              // runs of up to kLead k-blocks of the first half and then of the second at either end of the tile, half by
              // half in between
              constexpr int kLead = 3;
              for (int kb = 0; kb < k_blocks;) {
                const int left = k_blocks - kb;
                const int run = kb == 0 || left <= kLead ? min(left, kLead) : 1;
                for (int i = 0; i < run; ++i) {
                  const int st = stage + i < S ? stage + i : stage + i - S;
                  if (!landed(st, phase ^ (stage + i < S ? 0u : 1u))) return;
                  mma(st, 0, 0, kb + i == 0);
                }
                if (kb + run == k_blocks) tc2_commit_both(accf_bar(0), pair_mask);  // the first accumulator is complete
                if (kb == 0) {
                  if (!(ok = acc_free(1))) return;
                  tc_fence_after();
                }
                for (int i = 0; i < run; ++i) {
                  mma(stage, 1, 1, kb + i == 0);
                  release();
                }
                kb += run;
              }
              return;
            }
          }
          int left = SHARES ? g.share : 0;  // k-blocks of this share
          bool first = true;
          for (int kb = 0; kb < k_blocks; ++kb) {
            if (SHARES && left-- == 0) {  // this share is complete; on in the other accumulator
              left = g.share - 1;
              first = true;
              tc2_commit_both(accf_bar(buf), pair_mask);
              acc_phase ^= 1u << buf;
              buf ^= 1;
              if (!(ok = acc_free(buf))) return;
              tc_fence_after();
            }
            if (!landed(stage, phase)) return;
            mma(stage, 0, buf, SHARES ? first : kb == 0);
            first = false;
            release();
          }
        };
        if (!TWO || prob_of(tile) == 0)
          main_loop(g.p[0]);
        else
          main_loop(g.p[1]);
        if (!ok) break;
        if (both) {
          tc2_commit_both(accf_bar(1), pair_mask);
          acc_phase ^= 3u;
        } else {
          tc2_commit_both(accf_bar(buf), pair_mask);  // this accumulator is complete in both CTAs
          acc_phase ^= 1u << buf;
          buf ^= 1;
        }
      }
    }
  } else {
    // ------------------------------------------------------------------ epilogue (warps 2-9) ----
    const int quad = warp & 3;              // tensor-memory lanes this warp may read
    const int half = (warp - 2) >> 2;       // column half / epilogue group
    const int et = (threadIdx.x - 64) & 127;  // 0..127 inside the group
    const int bar_id = 1 + half;
    uint32_t acc_phase = 0;
    const int row_in_tile = quad * 32 + lane;
    const uint32_t stage_buf = staging + half * 16384;
    int buf = 0, last_prob = 0, halves = 1;
    [[maybe_unused]] uint32_t res_phase = 0;  // bit c: phase of chunk c's barrier
    [[maybe_unused]] bool wide8 = false, early = false;
    if constexpr (E::kFused) {
      wide8 = (g.p[0].N & 31) == 0 && (reinterpret_cast<uintptr_t>(e.z8_codes) & 31) == 0;
      early = SPLIT == 1 && !z_is_staged(e, wide8);
    }
    [[maybe_unused]] float* const bias_s = reinterpret_cast<float*>(
        base_ptr + kBarOffset + 256 + dense::Cfg<BN, SPLIT>::kRecvBytes) + half * 128;
    [[maybe_unused]] const uint32_t res_buf = staging + dense::kStagingBytes + half * 16384;  // (kBuffers)
    // (kDouble: a tile comes up once for each of its halves, the second time without a step of the walk)
    for (int rnd = 0, half_no = 0, tile = pair_id; tile < n_tiles; tile = half_no ? tile : next_tile(++rnd)) {
      int prob, m_blk, n_blk;
      tile_coords(tile, prob, m_blk, n_blk);
      if constexpr (kDouble) {
        halves = halves_of(tile);
        if (halves == 2) {
          buf = half_no;
          n_blk += half_no;
        }
      }
      const CUtensorMap* map_d = prob ? &map_d1 : &map_d0;
      const bool drain = prob != last_prob;  // the problems of a launch may have different output types
      last_prob = prob;
      if constexpr (E::kFused) {  // what can be fetched while the tile's main loop runs
        constexpr int kCols = SPLIT > 1 ? BN / SPLIT : HN / 2;  // columns that this group finishes (SPLIT > 1: if it finishes any)
        const int x0 = SPLIT > 1 ? n_blk * BN + split * kCols : n_blk * HN + half * kCols;
        // (the threads are behind the barriers of the tile before, and so behind their reads of its bias)
        if (e.bias && et < kCols) bias_s[et] = x0 + et < g.p[0].N ? e.bias[x0 + et] : 0.f;
        if (et == 0 && e.has_residual) {
          const int row0 = m_blk * 256 + (int)rank * 128;
          if (early) load_residual<kCols>(e, stage_buf, x0, row0, res_bar(half));
          if (E::kBuffers) load_residual<kCols>(e, res_buf, x0 + kCols / 2, row0, res_bar(half) + 16);
        }
      }
      const int row0 = m_blk * 256 + (int)rank * 128;
      uint32_t r[HN / 2];
      if constexpr (SHARES) {
        const int shares = (k_begin(tile, split + 1) - k_begin(tile, split) + g.share - 1) / g.share;
        bool gave_up = false;
#pragma unroll
        for (int j = 0; j < HN / 2; ++j) r[j] = 0u;
        for (int share = 0; share < shares; ++share) {
          mbar_wait_cluster(accf_bar(buf), (acc_phase >> buf) & 1u, abort_flag, 0xC00u + buf);
          if ((gave_up = group_gave_up(abort_flag, bar_id, 128))) break;
          tc_fence_after();
          const uint32_t t_row = tmem + ((uint32_t)(quad * 32) << 16) + buf * 256 + half * (HN / 2);
#pragma unroll
          for (int q = 0; q < HN / 32; ++q) {
            uint32_t t[16];  // (with 32 at a time the registers did not suffice)
            tc_ld16(t_row + q * 16, t);
            tc_wait_ld();
#pragma unroll
            for (int j = 0; j < 16; ++j) r[q * 16 + j] = __float_as_uint(__uint_as_float(r[q * 16 + j]) + __uint_as_float(t[j]));
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(map_to_cta(acce_bar(buf), leader_cta));
          if (share + 1 < shares) {  // (the last share's is turned over behind the tile)
            acc_phase ^= 1u << buf;
            buf ^= 1;
          }
        }
        if (gave_up) break;
      } else {
        mbar_wait_cluster(accf_bar(buf), (acc_phase >> buf) & 1u, abort_flag, 0xC00u + buf);
        // agree on giving up: a warp that timed out still joins this barrier, and all 128 threads take ONE decision
        if (group_gave_up(abort_flag, bar_id, 128)) break;
        tc_fence_after();
        const uint32_t t_row = tmem + ((uint32_t)(quad * 32) << 16) + buf * 256 + half * (HN / 2);
#pragma unroll
        for (int q = 0; q < HN / 32; ++q) tc_ld16(t_row + q * 16, *reinterpret_cast<uint32_t(*)[16]>(&r[q * 16]));
        tc_wait_ld();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(map_to_cta(acce_bar(buf), leader_cta));
      }
      if constexpr (SPLIT > 1) {
        constexpr int kCols = BN / SPLIT;
        uint32_t v[kCols];
        if (!exchange_columns<SPLIT>(r, v, half, split, rank, staging + dense::kStagingBytes + 256, recv_bar, row_in_tile,
                                     abort_flag, bar_id))
          break;
        const int xs = n_blk * BN + split * kCols;
        if constexpr (E::kFused) {
          if (!finish_half<kCols, false>(v, e, bias_s, g.p[0].M, g.p[0].N, et, bar_id, row_in_tile, stage_buf, 0, map_d, xs, row0,
                                         res_bar(half), res_phase, wide8, false, abort_flag))
            break;
        } else if (g.p[prob].d_is_fp32)
          store_half<true, false, kCols>(v, 1.0f, et, bar_id, row_in_tile, stage_buf, map_d, xs, row0, g.p[prob].accumulate, drain);
        else
          store_half<false, false, kCols>(v, 1.0f, et, bar_id, row_in_tile, stage_buf, map_d, xs, row0, g.p[prob].accumulate, drain);
      } else if constexpr (E::kFused) {
        if (!finish_half<HN / 2, E::kBuffers>(r, e, bias_s, g.p[0].M, g.p[0].N, et, bar_id, row_in_tile, stage_buf, res_buf, map_d,
                                              n_blk * HN + half * (HN / 2), row0, res_bar(half), res_phase, wide8, early, abort_flag))
          break;
      } else if (g.p[prob].d_is_fp32)
        store_half<true, false, HN / 2>(r, 1.0f, et, bar_id, row_in_tile, stage_buf, map_d, n_blk * HN + half * (HN / 2),
                                        row0, g.p[prob].accumulate, drain);
      else
        store_half<false, false, HN / 2>(r, 1.0f, et, bar_id, row_in_tile, stage_buf, map_d, n_blk * HN + half * (HN / 2),
                                         row0, g.p[prob].accumulate, drain);
      acc_phase ^= 1u << buf;
      buf = halves == 2 ? 0 : buf ^ 1;
      if (kDouble) half_no = halves == 2 ? half_no ^ 1 : 0;
    }
    if (et == 0) bulk_wait_all<0>();  // all stores have left shared memory and are visible
  }

  // ------------------------------------------------------------------ teardown ----
  tc_fence_before();
  leave_cluster<2 * SPLIT>(done_bar, cta, abort_flag, 0xD00u);
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(dense::kTmemCols) : "memory");
  }
}

}  // namespace dense
}  // namespace nvfp4

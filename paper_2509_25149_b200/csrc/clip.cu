// The norm over the gradients of many tensors, and clipping.
//   sum = sum of g^2;   factor = norm > max_norm ? max_norm / norm : 1, norm = sqrt(sum);   out = g factor
// Bound by HBM: everything is read for the sum and once more to be scaled, since the factor needs the whole sum first (the second pass goes backwards, so
// that what the first one read last is still in L2).  The list of tensors travels in the kernel's parameters, so that a captured graph holds it
// and nothing is copied to the device.  Tensors are cut into tiles, which the CTAs take in turn.
// 770 million binary32 numbers to bf16: 452 us for the sum (104 % of the copy rate), 670 to scale (105 %: some of it from L2).
#include <algorithm>
#include <climits>

#include "around.h"
#include "copy8.cuh"
#include "ends.h"

namespace nvfp4 {

namespace {

constexpr int kThreads = 256, kMaxCtas = 148 * 8, kAhead = 4;
constexpr int kTile = kThreads * kAhead * 8, kSmallTile = kThreads * 8;  // elements of a tile: four chunks of eight a thread, or one where few tiles are too few for the GPU
constexpr int kList = 600, kShortList = 64;  // tensors of a launch: 32 bytes each and 4 for the tiles before them, of 32764 bytes of parameters

struct Tensor {
  const void* data;
  void* out;
  int64_t count;
  int32_t head;   // elements before the first whole chunk (data is aligned to its elements only): tiles begin behind them, the first tile takes them too
  uint8_t fp32, out_fp32, vector, pad;  // vector: out's chunks are aligned as data's are
};
template <int N>
struct List {
  static constexpr int kMost = N;
  int32_t n, tiles, tile;  // tile: elements
  int32_t first[N];        // tiles before the tensor
  Tensor t[N];
};

// the tensor that has the tile
template <class L>
__device__ __forceinline__ int find(const L& l, int tile) {
  int lo = 0, hi = l.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (l.first[mid] <= tile) lo = mid; else hi = mid - 1;
  }
  return lo;
}
__device__ __forceinline__ float element(const Tensor& t, int64_t i) {
  return t.fp32 ? static_cast<const float*>(t.data)[i] : bf16_lo(static_cast<const uint16_t*>(t.data)[i]);
}
__device__ __forceinline__ double square(float v) { return (double)v * (double)v; }

// Squares of eight neighbours in binary32, unless they leave its range: then in 64 bits.  Sums of eight below 2^-90 may have lost what they rounded off,
// zeros take the way of 64 bits too, which costs nothing beside the memory.
__device__ __forceinline__ double squares8(const float (&v)[8]) {
  float2 s = make_float2(v[0] * v[0], v[1] * v[1]);
#pragma unroll
  for (int j = 2; j < 8; j += 2) s = fma2(make_float2(v[j], v[j + 1]), make_float2(v[j], v[j + 1]), s);
  const float sum = s.x + s.y;
  if (__builtin_expect(sum >= 0x1p-90f && sum <= 3.402823466e38f, 1)) return (double)sum;
  double d = 0.;
#pragma unroll
  for (int j = 0; j < 8; ++j) d += square(v[j]);
  return d;
}

template <bool F32>
__device__ __forceinline__ double tile_squares(const Tensor& t, int64_t first, int64_t end) {
  double sum = 0.;
  Raw8<F32> raw[kAhead];
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    const int64_t i = first + ((int64_t)u * kThreads + threadIdx.x) * 8;
    if (i + 8 <= end) raw[u].load(t.data, i);
  }
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    const int64_t i = first + ((int64_t)u * kThreads + threadIdx.x) * 8;
    if (i + 8 <= end) {
      float v[8];
      raw[u].values(v);
      sum += squares8(v);
    } else {
      for (int64_t j = i; j < end; ++j) sum += square(element(t, j));
    }
  }
  return sum;
}

__device__ __forceinline__ double block_sum(double v, double* part) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  double s = 0.;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) s += part[w];
  return s;
}

template <class L>
__global__ void __launch_bounds__(kThreads) sq_norm_kernel(const __grid_constant__ L l, double* partial) {
  __shared__ double part[kThreads / 32];
  griddep_wait();
  griddep_launch_dependents();
  double sum = 0.;
  for (int tile = blockIdx.x; tile < l.tiles; tile += gridDim.x) {
    const int at = find(l, tile), k = tile - l.first[at];
    const Tensor& t = l.t[at];
    const int64_t first = t.head + (int64_t)k * l.tile, end = min(first + l.tile, t.count);
    if (k == 0 && threadIdx.x < t.head) sum += square(element(t, threadIdx.x));
    sum += t.fp32 ? tile_squares<true>(t, first, end) : tile_squares<false>(t, first, end);
  }
  const double s = block_sum(sum, part);
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}
__global__ void __launch_bounds__(kThreads) sq_norm_total_kernel(const double* partial, int parts, double* sum, int accumulate) {
  __shared__ double part[kThreads / 32];
  griddep_wait();
  griddep_launch_dependents();
  double v = 0.;
  for (int i = threadIdx.x; i < parts; i += kThreads) v += partial[i];
  const double s = block_sum(v, part);
  if (threadIdx.x == 0) *sum = accumulate ? *sum + s : s;
}

template <bool F32, bool OUT32>
__device__ __forceinline__ void scale_tile(const Tensor& t, int64_t first, int64_t end, float factor) {
  auto scaled = [&](float v) { return factor == 0.f ? 0.f : v * factor; };
  auto put = [&](int64_t i, float v) {
    if (OUT32)
      static_cast<float*>(t.out)[i] = v;
    else
      static_cast<__nv_bfloat16*>(t.out)[i] = __float2bfloat16_rn(v);
  };
  if (!t.vector) {  // neighbouring threads take neighbouring elements
    for (int64_t i = first + threadIdx.x; i < end; i += 8 * kThreads) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = i + j * kThreads < end ? element(t, i + j * kThreads) : 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (i + j * kThreads < end) put(i + j * kThreads, scaled(v[j]));
    }
    return;
  }
  Raw8<F32> raw[kAhead];
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    const int64_t i = first + ((int64_t)u * kThreads + threadIdx.x) * 8;
    if (i + 8 <= end) raw[u].load(t.data, i);
  }
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    const int64_t i = first + ((int64_t)u * kThreads + threadIdx.x) * 8;
    if (i + 8 <= end) {
      float v[8];
      raw[u].values(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = scaled(v[j]);
      store8_first_out<OUT32>(t.out, i, v);  // (770 million elements 1175 -> 1130 us with the norm: more of what that read last is still there)
    } else {
      for (int64_t j = i; j < end; ++j) put(j, scaled(element(t, j)));
    }
  }
}

template <class L>
__global__ void __launch_bounds__(kThreads) clip_kernel(const __grid_constant__ L l, const double* sum, float max_norm, float* stats) {
  griddep_wait();
  griddep_launch_dependents();
  const double norm = sqrt(*sum);
  const bool finite = norm <= 1.7976931348623157e308;
  const float factor = !finite ? 0.f : norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.f;
  if (stats && blockIdx.x == 0 && threadIdx.x == 0) {
    stats[0] = (float)norm;
    stats[1] = factor;
  }
  for (int tile = l.tiles - 1 - (int)blockIdx.x; tile >= 0; tile -= gridDim.x) {
    const int at = find(l, tile), k = tile - l.first[at];
    const Tensor& t = l.t[at];
    if (t.out == t.data && factor == 1.f) continue;
    const int64_t first = t.head + (int64_t)k * l.tile, end = min(first + l.tile, t.count), from = k == 0 ? 0 : first;
    if (from < first) {  // (at most seven)
      if (threadIdx.x < first) {
        const float v = factor == 0.f ? 0.f : element(t, threadIdx.x) * factor;
        if (t.out_fp32)
          static_cast<float*>(t.out)[threadIdx.x] = v;
        else
          static_cast<__nv_bfloat16*>(t.out)[threadIdx.x] = __float2bfloat16_rn(v);
      }
    }
    if (t.fp32) {
      if (t.out_fp32) scale_tile<true, true>(t, first, end, factor); else scale_tile<true, false>(t, first, end, factor);
    } else {
      if (t.out_fp32) scale_tile<false, true>(t, first, end, factor); else scale_tile<false, false>(t, first, end, factor);
    }
  }
}

// The next tensors of a list, as many as a launch holds; returns how many of the list's it took
template <class L>
int fill(L& l, const nvfp4_grad* grads, int n) {
  int64_t all = 0;
  for (int i = 0; i < n; ++i) all += grads[i].count;
  l.tile = all < (int64_t)kMaxCtas * kTile ? kSmallTile : kTile;
  l.n = 0;
  int64_t tiles = 0;
  int i = 0;
  for (; i < n && l.n < L::kMost; ++i) {
    const nvfp4_grad& g = grads[i];
    if (g.count == 0) continue;
    const uintptr_t size = g.is_fp32 ? 4 : 2, at = reinterpret_cast<uintptr_t>(g.data);
    const int64_t head = std::min<int64_t>((int64_t)((16 - at % 16) % 16 / size), g.count);
    const int64_t of_tensor = std::max<int64_t>((g.count - head + l.tile - 1) / l.tile, 1);
    if (tiles + of_tensor > INT_MAX) break;
    Tensor& t = l.t[l.n];
    t.data = g.data;
    t.out = g.out ? g.out : g.data;
    t.count = g.count;
    t.head = (int32_t)head;
    t.fp32 = g.is_fp32 != 0;
    t.out_fp32 = g.out ? g.out_is_fp32 != 0 : t.fp32;
    t.vector = (reinterpret_cast<uintptr_t>(t.out) + (uintptr_t)head * (t.out_fp32 ? 4 : 2)) % 16 == 0;
    t.pad = 0;
    l.first[l.n++] = (int32_t)tiles;
    tiles += of_tensor;
  }
  l.tiles = (int32_t)tiles;
  return i;
}
template <class L>
unsigned ctas_of(const L& l) { return (unsigned)std::min(l.tiles, kMaxCtas); }

template <int N>
cudaError_t sq_norm(const nvfp4_grad* grads, int n, double* sum, bool accumulate, double* workspace, cudaStream_t s) {
  List<N> l;
  for (int done = 0; done < n;) {
    done += fill(l, grads + done, n - done);
    if (l.tiles == 0 && done < n) continue;
    cudaError_t e;
    if (l.tiles > 0) {
      e = launch_divided(kStreamingCarveout, sq_norm_kernel<List<N>>, dim3(ctas_of(l)), dim3(kThreads), 0, s, l, workspace);
      count_launch();
      if (e != cudaSuccess) return e;
    }
    e = launch_divided(kStreamingCarveout, sq_norm_total_kernel, dim3(1), dim3(kThreads), 0, s, workspace, (int)ctas_of(l), sum, (int)accumulate);
    count_launch();
    if (e != cudaSuccess) return e;
    accumulate = true;
  }
  return cudaSuccess;
}
template <int N>
cudaError_t clip(const nvfp4_grad* grads, int n, const double* sum, float max_norm, float* stats, cudaStream_t s) {
  List<N> l;
  for (int done = 0; done < n;) {
    done += fill(l, grads + done, n - done);
    const unsigned grid = std::max(1u, ctas_of(l));  // (without an element too: stats)
    const cudaError_t e = launch_divided(kStreamingCarveout, clip_kernel<List<N>>, dim3(grid), dim3(kThreads), 0, s, l, sum, max_norm, stats);
    count_launch();
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace

size_t grad_sq_norm_workspace() { return kMaxCtas * sizeof(double); }

// (21 KB of parameters cost the host some microseconds more than 2 KB)
cudaError_t launch_grad_sq_norm(const nvfp4_grad* grads, int n, double* sum, bool accumulate, double* workspace, cudaStream_t s) {
  return n <= kShortList ? sq_norm<kShortList>(grads, n, sum, accumulate, workspace, s) : sq_norm<kList>(grads, n, sum, accumulate, workspace, s);
}
cudaError_t launch_grad_clip(const nvfp4_grad* grads, int n, const double* sum, float max_norm, float* stats, cudaStream_t s) {
  return n <= kShortList ? clip<kShortList>(grads, n, sum, max_norm, stats, s) : clip<kList>(grads, n, sum, max_norm, stats, s);
}

}  // namespace nvfp4

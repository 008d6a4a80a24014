// Copies in 8 bits (NVFP4_FORMAT_MXFP8): E4M3 codes and one power-of-two scale byte per 32 elements of a row.
//   E = the smallest whole number >= -127 with amax_b <= 448 * 2^E,  byte = E + 127,  code = e4m3(x * 2^-E)
// Nothing saturates (E is rounded up), and both multiplications are exact: the only rounding is the one to E4M3, to nearest.
// A scale of amax / 448 would use the top of the range fully, at the price of a rounding of the product in either direction.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "async_ptx.cuh"
#include "common.cuh"
#include "quantize_common.cuh"

namespace nvfp4 {

inline int64_t blocks8(int64_t cols) { return (cols + 31) / 32; }  // scale bytes of a row

// A copy as a kernel sees it (codes == NULL: none)
struct Copy8 {
  uint8_t* codes;   // rows x cols
  uint8_t* scales;  // rows x blocks
  int64_t blocks;   // scale bytes of a row
};

// 448 = 1.75 * 2^8: the exponent goes up by one where the mantissa is above 1.75
__device__ __forceinline__ uint32_t scale_byte8(float amax) {
  const uint32_t e = (__float_as_uint(amax) + 0x1FFFFFu) >> 23;
  return e > 8u ? e - 8u : 0u;
}
__device__ __forceinline__ float encode_scale8(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }  // 2^-E
__device__ __forceinline__ float decode_scale8(uint32_t byte) {                                                 // 2^E
  return byte == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(byte << 23);
}

__device__ __forceinline__ float amax8(const float (&v)[8]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; i += 2) m = amax3(m, v[i], v[i + 1]);
  return m;
}
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {  // a in the lowest byte
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\t"
      "mov.b32 %0, {lo, hi};\n\t}"
      : "=r"(r)
      : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}
__device__ __forceinline__ uint2 encode8(const float (&v)[8], float scale) {
  float s[8];
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const float2 p = mul2(make_float2(v[i], v[i + 1]), make_float2(scale, scale));
    s[i] = p.x;
    s[i + 1] = p.y;
  }
  return make_uint2(e4m3x4(s[0], s[1], s[2], s[3]), e4m3x4(s[4], s[5], s[6], s[7]));
}
// four codes -> their values before the scale
__device__ __forceinline__ void decode4(uint32_t w, float (&v)[4]) {
  uint32_t lo, hi;
  asm("{\n\t.reg .b16 a, b;\n\t"
      "mov.b32 {a, b}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, a;\n\t"
      "cvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(w));
  const float2 x = __half22float2(*reinterpret_cast<__half2*>(&lo)), y = __half22float2(*reinterpret_cast<__half2*>(&hi));
  v[0] = x.x; v[1] = x.y; v[2] = y.x; v[3] = y.y;
}
__device__ __forceinline__ void decode8(uint2 w, float scale, float (&v)[8]) {
  float a[4], b[4];
  decode4(w.x, a);
  decode4(w.y, b);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = a[i] * scale;
    v[4 + i] = b[i] * scale;
  }
}

// the same in pairs, for two binary32 operations an instruction
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("{.reg .b64 ra, rb, rc, rd; mov.b64 ra, {%2, %3}; mov.b64 rb, {%4, %5}; mov.b64 rc, {%6, %7}; "
      "fma.rn.f32x2 rd, ra, rb, rc; mov.b64 {%0, %1}, rd;}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return r;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
__device__ __forceinline__ void decode8(uint2 w, float scale, float2 (&v)[4]) {
  float a[4], b[4];
  decode4(w.x, a);
  decode4(w.y, b);
  v[0] = mul2(make_float2(a[0], a[1]), both(scale));
  v[1] = mul2(make_float2(a[2], a[3]), both(scale));
  v[2] = mul2(make_float2(b[0], b[1]), both(scale));
  v[3] = mul2(make_float2(b[2], b[3]), both(scale));
}

// Eight neighbouring elements of a row belong to a lane and a block to four lanes (the chunk's index and the lane agree in
// their last two bits).  Every lane of the warp calls; `live`: the chunk exists (values of one that does not are zero).
__device__ __forceinline__ void store_chunk8(const Copy8& q, const float (&v)[8], int64_t row, int64_t chunk, int64_t cols, bool live) {
  float m = amax8(v);
  m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
  m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
  const uint32_t byte = scale_byte8(m);
  const uint2 codes = encode8(v, encode_scale8(byte));
  if (!live) return;
  *reinterpret_cast<uint2*>(q.codes + row * cols + chunk * 8) = codes;
  if ((chunk & 3) == 0) q.scales[row * q.blocks + (chunk >> 2)] = (uint8_t)byte;
}

// ---- eight neighbouring elements (coherent loads: a source may not be complete when the kernel becomes resident) ----
__device__ __forceinline__ uint2 ldg64_stream(const void* p) {
  uint2 r;
  asm volatile("ld.global.L1::no_allocate.v2.b32 {%0,%1}, [%2];" : "=r"(r.x), "=r"(r.y) : "l"(p));
  return r;
}
__device__ __forceinline__ uint32_t ldg8(const uint8_t* p) {
  uint32_t r;
  asm volatile("ld.global.u8 %0, [%1];" : "=r"(r) : "l"(p));
  return r;
}
__device__ __forceinline__ uint4 lds16(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds8(uint32_t at) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at) : "memory");
  return v;
}
// ---- asynchronous copies of a thread into its own places of shared memory (zeros where there is nothing): 16 or 8 bytes ----
template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, bool live) {
  if (BYTES == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(live ? 8 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void unpack8(uint4 a, float (&v)[8]) {
  v[0] = bf16_lo(a.x); v[1] = bf16_hi(a.x); v[2] = bf16_lo(a.y); v[3] = bf16_hi(a.y);
  v[4] = bf16_lo(a.z); v[5] = bf16_hi(a.z); v[6] = bf16_lo(a.w); v[7] = bf16_hi(a.w);
}
__device__ __forceinline__ void unpack8(uint4 a, float2 (&v)[4]) {
  v[0] = make_float2(bf16_lo(a.x), bf16_hi(a.x));
  v[1] = make_float2(bf16_lo(a.y), bf16_hi(a.y));
  v[2] = make_float2(bf16_lo(a.z), bf16_hi(a.z));
  v[3] = make_float2(bf16_lo(a.w), bf16_hi(a.w));
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
  return make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
}
// what a chunk is loaded as
template <bool F32>
struct Raw8 {
  uint4 w[F32 ? 2 : 1];
  __device__ __forceinline__ void load(const void* base, int64_t elem) {
    if (F32) {
      const float* p = static_cast<const float*>(base) + elem;
      w[0] = ldg128_stream(p);
      w[F32 ? 1 : 0] = ldg128_stream(p + 4);
    } else {
      w[0] = ldg128_stream(static_cast<const uint16_t*>(base) + elem);
    }
  }
  __device__ __forceinline__ void zero() {
    w[0] = make_uint4(0u, 0u, 0u, 0u);
    w[F32 ? 1 : 0] = make_uint4(0u, 0u, 0u, 0u);
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
    if (F32) {
      const uint4 a = w[0], b = w[F32 ? 1 : 0];
      v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y); v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w);
      v[4] = __uint_as_float(b.x); v[5] = __uint_as_float(b.y); v[6] = __uint_as_float(b.z); v[7] = __uint_as_float(b.w);
    } else {
      unpack8(w[0], v);
    }
  }
};
template <bool F32>
__device__ __forceinline__ void values2(const Raw8<F32>& r, float2 (&v)[4]) {
  if (F32) {
    const uint4 a = r.w[0], b = r.w[F32 ? 1 : 0];
    v[0] = make_float2(__uint_as_float(a.x), __uint_as_float(a.y));
    v[1] = make_float2(__uint_as_float(a.z), __uint_as_float(a.w));
    v[2] = make_float2(__uint_as_float(b.x), __uint_as_float(b.y));
    v[3] = make_float2(__uint_as_float(b.z), __uint_as_float(b.w));
  } else {
    unpack8(r.w[0], v);
  }
}
template <bool F32>
__device__ __forceinline__ void store8(void* base, int64_t elem, const float2 (&v)[4]) {
  if (F32) {
    float4* p = reinterpret_cast<float4*>(static_cast<float*>(base) + elem);
    p[0] = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
    p[1] = make_float4(v[2].x, v[2].y, v[3].x, v[3].y);
  } else {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(base) + elem) =
        make_uint4(pack2(v[0].x, v[0].y), pack2(v[1].x, v[1].y), pack2(v[2].x, v[2].y), pack2(v[3].x, v[3].y));
  }
}
template <bool F32>
__device__ __forceinline__ void store8(void* base, int64_t elem, const float (&v)[8]) {
  if (F32) {
    float4* p = reinterpret_cast<float4*>(static_cast<float*>(base) + elem);
    p[0] = make_float4(v[0], v[1], v[2], v[3]);
    p[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(base) + elem) = pack8(v);
  }
}
// the same for results that exceed L2 and are not read again by their kernel: first to leave it, so that what is read stays
template <bool F32>
__device__ __forceinline__ void store8_first_out(void* base, int64_t elem, const float (&v)[8]) {
  if (F32) {
    float4* p = reinterpret_cast<float4*>(static_cast<float*>(base) + elem);
    __stcs(p, make_float4(v[0], v[1], v[2], v[3]));
    __stcs(p + 1, make_float4(v[4], v[5], v[6], v[7]));
  } else {
    __stcs(reinterpret_cast<uint4*>(static_cast<uint16_t*>(base) + elem), pack8(v));
  }
}
__device__ __forceinline__ void load_gain(const float* gain, int64_t elem, float (&g)[8]) {
  if (!gain) {
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = 1.f;
    return;
  }
  const float4* p = reinterpret_cast<const float4*>(gain + elem);
  const float4 a = p[0], b = p[1];
  g[0] = a.x; g[1] = a.y; g[2] = a.z; g[3] = a.w; g[4] = b.x; g[5] = b.y; g[6] = b.z; g[7] = b.w;
}

}  // namespace nvfp4

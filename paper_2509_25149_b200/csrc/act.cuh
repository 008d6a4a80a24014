// The activations between two products and their derivatives, in binary32.
//   squared ReLU  max(z, 0)^2                     2 max(z, 0)
//   SiLU          z s,  s = 1 / (1 + e^-z)         s + z s (1 - s)
//   GELU          z s,  s = 1 / (1 + e^-2u)        s + z s (1 - s) 2u'       u = sqrt(2 / pi) (z + 0.044715 z^3)
// (z/2 (1 + tanh u) is z s: the logistic form keeps its relative accuracy where z is far below zero and 1 + tanh u cancels.)
// e^x and the quotient are the fast ones.  The error of e^x grows with the size of its exponent, a unit in the last place of binary32 or so for each
// unit of it: some 2^-16 of the value at 90, where it ends, far below the rounding to bf16 that follows (and zero where 1 + e^-x is above 2^126, where the true quotient is below 2^-126).
#pragma once
#include <cuda_runtime.h>

#include "nvfp4.h"

namespace nvfp4 {

__device__ __forceinline__ float logistic(float x) { return __fdividef(1.f, 1.f + __expf(-x)); }  // (e^-x = inf: 0)
constexpr float kGelu2c = 1.5957691216057308f, kGelu3 = 0.044715f;  // 2 sqrt(2 / pi)

template <int ACT>
__device__ __forceinline__ float act_value(float z) {
  if (ACT == NVFP4_ACT_RELU2) {
    const float p = fmaxf(z, 0.f);
    return p * p;
  }
  if (ACT == NVFP4_ACT_SILU) return z * logistic(z);
  if (ACT == NVFP4_ACT_GELU) return z * logistic(kGelu2c * z * fmaf(kGelu3 * z, z, 1.f));
  return z;
}

// act(z) and act'(z)
template <int ACT>
__device__ __forceinline__ float act_slope(float z, float& value) {
  if (ACT == NVFP4_ACT_RELU2) {
    const float p = fmaxf(z, 0.f);
    value = p * p;
    return 2.f * p;
  }
  if (ACT == NVFP4_ACT_SILU) {
    const float s = logistic(z);
    value = z * s;
    return fmaf(value, 1.f - s, s);
  }
  if (ACT == NVFP4_ACT_GELU) {
    // (beyond |z| = 100 s is 0 or 1 and the second term zero: its factor must not be infinite there)
    const float zz = fminf(z * z, 1e4f);
    const float s = logistic(z * fmaf(kGelu2c * kGelu3, zz, kGelu2c));
    value = z * s;
    return fmaf(value * (1.f - s), fmaf(3.f * kGelu2c * kGelu3, zz, kGelu2c), s);
  }
  value = z;
  return 1.f;
}

}  // namespace nvfp4

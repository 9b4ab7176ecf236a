// Activations and their slopes on the device.
//
//   relu z -> max(0, z), slope 1 where z > 0;  gelu z -> z Phi(z), slope Phi(z) + z phi(z);  silu z -> z p, slope p (1 + z (1 - p)),
//   p = 1 / (1 + e^-z)
// (Phi, phi: the normal distribution and its density.)  NaN stays NaN; the ends of the line give their limits.
//
// For results of 8 mantissa bits Phi is taken from Abramowitz and Stegun, Handbook of Mathematical Functions, 7.1.26: with t = 1 / (1 + 0.3275911 u)
// erfc(u) = t (a1 + t (a2 + t (a3 + t (a4 + t a5)))) e^(-u^2), off by at most 1.5e-7, and exponentials and reciprocals are the hardware's:
// the error is 1e-7 of |z| before the rounding of up to 2^-8 of the result.  It shares its exponential with the slope's density.  fp32
// results take the library's functions.
#pragma once

#include "dev_common.hpp"
#include "detag.h"

namespace detag {

template <class T>
__device__ __forceinline__ void normal_parts(float z, float &upto, float &density) {
  if constexpr (sizeof(T) == 2) {
    const float t = __builtin_amdgcn_rcpf(1.f + 0.3275911f * 0.70710678f * fabsf(z));
    const float e = __builtin_amdgcn_exp2f(-0.72134752f * z * z);  // e^(-z^2 / 2)
    // half of the sum: a1 / 2 and so on
    const float tail = e * (t * (0.127414796f + t * (-0.142248368f + t * (0.7107068705f + t * (-0.7265760135f + t * 0.5307027145f)))));
    upto = z > 0.f ? 1.f - tail : tail;
    density = 0.39894228f * e;
  } else {
    upto = 0.5f * erfcf(-0.70710678f * z);
    density = 0.39894228f * expf(-0.5f * z * z);
  }
}

template <class T>
__device__ __forceinline__ float logistic(float z) {
  if constexpr (sizeof(T) == 2) return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * z));
  else return 1.f / (1.f + expf(-z));
}

// What a factor that has become zero is multiplied with: finite, and z as far as that matters.  (Of NaN it makes a number, but then the other
// factor is none.)
__device__ __forceinline__ float finite_of(float z, float most) { return __builtin_amdgcn_fmed3f(z, -most, most); }

// T: the type whose accuracy the result is to have.
template <class T>
__device__ __forceinline__ float act_value(float z, int act) {
  if (act == DETAG_ACT_RELU) return z <= 0.f ? 0.f : z;
  if (act == DETAG_ACT_GELU) {
    float upto, density;
    normal_parts<T>(z, upto, density);
    return (z < 0.f ? finite_of(z, 40.f) : z) * upto;
  }
  if (act == DETAG_ACT_SILU) {
    return (z < 0.f ? finite_of(z, 200.f) : z) * logistic<T>(z);
  }
  return z;
}

template <class T>
__device__ __forceinline__ float act_slope(float z, int act) {
  if (act == DETAG_ACT_RELU) return z > 0.f ? 1.f : 0.f;
  if (act == DETAG_ACT_GELU) {
    float upto, density;
    normal_parts<T>(z, upto, density);
    return upto + finite_of(z, 40.f) * density;
  }
  if (act == DETAG_ACT_SILU) {
    const float p = logistic<T>(z);
    return p * (1.f + finite_of(z, 200.f) * (1.f - p));
  }
  return 1.f;
}

}  // namespace detag

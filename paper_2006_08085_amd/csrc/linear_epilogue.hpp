// What a layer's product does with its sums before they are stored: bias, activation and residual, or the slope of an activation.
#pragma once

#include "act_dev.hpp"
#include "linear_common.hpp"

namespace detag {

// Four neighbouring biases of a worker's layer, zeros past the last or without any.
template <class T>
__device__ __forceinline__ f32x4 bias_of(const LinearArgs &a, int worker, int c) {
  if (!a.bias) return f32x4{0.f, 0.f, 0.f, 0.f};
  return load4(static_cast<const T *>(a.bias) + int64_t(worker) * a.ld + c, a.out - c);
}

// z -> residual + act(z) for columns c .. c+3 of row r; z itself is kept where it is wanted.
template <class T, class TC>
__device__ __forceinline__ f32x4 finish_output(const LinearArgs &a, f32x4 z, int64_t r, int c) {
  const int inside = a.out - c;
  if (a.pre) store4(static_cast<T *>(a.pre) + r * a.ldz + c, z, inside);
  if (a.act)
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e] = act_value<TC>(z[e], a.act);
  if (a.residual) z += load4(static_cast<const TC *>(a.residual) + r * a.ldr + c, inside);
  return z;
}

// The gradient of an activation's result -> that of what it was taken of.
template <class T>
__device__ __forceinline__ f32x4 finish_input(const LinearArgs &a, f32x4 v, int64_t r, int c) {
  if (!a.act) return v;
  const f32x4 z = load4(static_cast<const T *>(a.rows_b) + r * a.ldb + c, a.in - c);
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] *= act_slope<T>(z[e], a.act);
  return v;
}

}  // namespace detag

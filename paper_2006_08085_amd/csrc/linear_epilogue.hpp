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

// What the epilogue reads for columns c .. c+3 of row r, as it lies there: of the residual, or (not Forward) of what the activation's slope is
// taken of.
template <class T>
struct Four {
  std::conditional_t<sizeof(T) == 2, u32x2, f32x4> bits;
  __device__ __forceinline__ f32x4 floats() const {
    if constexpr (sizeof(T) == 2) return f32x4{__uint_as_float(bits[0] << 16), __uint_as_float(bits[0] & 0xffff0000u), __uint_as_float(bits[1] << 16), __uint_as_float(bits[1] & 0xffff0000u)};
    else return bits;
  }
};
template <class T>
__device__ __forceinline__ Four<T> read_four(const T *p, int inside) {
  Four<T> v;
  if (inside >= 4) {
    if constexpr (sizeof(T) == 2) v.bits = *reinterpret_cast<const u32x2_any *>(p);
    else v.bits = *reinterpret_cast<const f32x4_any *>(p);
  } else {
    uint32_t e[4] = {0, 0, 0, 0};
    using Bits = std::conditional_t<sizeof(T) == 2, uint16_t, uint32_t>;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < inside) e[k] = reinterpret_cast<const Bits *>(p)[k];
    if constexpr (sizeof(T) == 2) v.bits = u32x2{e[0] | e[1] << 16, e[2] | e[3] << 16};
    else v.bits = __builtin_bit_cast(f32x4, (u32x4{e[0], e[1], e[2], e[3]}));
  }
  return v;
}

// f(the activation as a constant): tests of it inside would cut the arithmetic of many values into pieces that wait for themselves.
template <class F>
__device__ __forceinline__ void with_act(int act, F &&f) {
  if (act == DETAG_ACT_GELU) f(std::integral_constant<int, DETAG_ACT_GELU>{});
  else if (act == DETAG_ACT_SILU) f(std::integral_constant<int, DETAG_ACT_SILU>{});
  else if (act == DETAG_ACT_RELU) f(std::integral_constant<int, DETAG_ACT_RELU>{});
  else f(std::integral_constant<int, DETAG_ACT_NONE>{});
}

}  // namespace detag

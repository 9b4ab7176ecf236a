// One AdamW step over all tensors of all workers' rows:
//
//   m <- beta1 m + (1 - beta1) g;   v <- beta2 v + (1 - beta2) g^2
//   x <- x (1 - lr s w) - lr s clamp((m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps), limit)       s, w: of the tensor
//
// with the moments in fp32 or in 8 bits.  A row is a list of tensors, each cut into blocks of 256 columns from its own start; a
// wavefront takes a block at a time, four neighbouring columns a lane, and finds the block's place and numbers in a table that was
// made with the list.  What bounds it is memory: fp32 models and moments 28 bytes an element, 8-bit moments 16.
//
// 8-bit moments.  Of a block's moments (256 columns of one tensor and worker) the largest finite magnitude gives a power of two;
// relative to that m is kept as sign, 4 exponent and 3 mantissa bits, v, which has no sign and twice the range, as 5 and 3.  A power
// of two costs no precision in a floating format and makes every kept value exact in bfloat16.  The rounding is stochastic: v moves by
// (1 - beta2) of itself a step, far less than half the spacing of three mantissa bits, so that the nearest value would never
// change.  Random bits: Philox-4x32-10 (noise_dev.hpp), counter (64 * block + lane, 0x41646157, worker, t), key = seed; word j of the
// lane's four is column j's, its lower half rounds m, the upper one v.
//
//   E = biased fp32 exponent of the largest finite magnitude, at least 16
//   y = |m| 2^(134-E) or v 2^(142-E);  least normal number 2^-6 or 2^-14
//   code = ((bits(y) + 16 r) >> 20) - 8 (127 - bias) from there on, below floor(2^9 y + 2^-16 r) or floor(2^17 y + 2^-16 r)
// so the largest magnitude has the last exponent but one, and rounding up needs no clamp.  Infinities and NaN become the code with
// all bits set (127, 255), which is read back as NaN.
//
// The moments' arithmetic is rounded operation by operation (no fused multiply-add), so that it can be restated bit by bit.
#include "dev_common.hpp"
#include "detag_internal.h"
#include "noise_dev.hpp"

namespace detag {
namespace {

constexpr int kBlock = kAdamwBlock, kLaneCols = 4;
constexpr int kThreads = 256, kWaves = kThreads / 64;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32_any __attribute__((aligned(1)));

struct StepArgs {
  void *x;
  const float *g;
  void *m, *v;
  uint8_t *scales;  // n x blocks x 2 exponents
  uint16_t *x16;
  const AdamwBlock *blocks;
  int64_t ld, count;  // pitch, blocks of a row
  int n;
  float lr, beta1, rest1, beta2, rest2, eps, unbias1, unbias2, limit;
  uint32_t t, seed_lo, seed_hi;
};

// Four columns at p; `inside` of them exist, the others read as zero.
__device__ __forceinline__ void read4(const float *p, int inside, float (&v)[4]) {
  if (inside >= 4) {
    const f32x4 r = *reinterpret_cast<const f32x4_any *>(p);
    v[0] = r[0], v[1] = r[1], v[2] = r[2], v[3] = r[3];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = e < inside ? p[e] : 0.f;
  }
}
__device__ __forceinline__ void read4(const bf16_t *p, int inside, float (&v)[4]) {
  if (inside >= 4) {
    const u32x2_any r = *reinterpret_cast<const u32x2_any *>(p);
    v[0] = __uint_as_float(r[0] << 16), v[1] = __uint_as_float(r[0] & 0xffff0000u);
    v[2] = __uint_as_float(r[1] << 16), v[3] = __uint_as_float(r[1] & 0xffff0000u);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = e < inside ? to_f32(p[e]) : 0.f;
  }
}
__device__ __forceinline__ uint32_t read4(const uint8_t *p, int inside) {
  if (inside >= 4) return *reinterpret_cast<const u32_any *>(p);
  uint32_t v = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < inside) v |= uint32_t(p[e]) << 8 * e;
  return v;
}
__device__ __forceinline__ void write4(float *p, int inside, const float (&v)[4]) {
  if (inside >= 4) {
    *reinterpret_cast<f32x4_any *>(p) = f32x4{v[0], v[1], v[2], v[3]};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < inside) p[e] = v[e];
  }
}
__device__ __forceinline__ void write4(bf16_t *p, int inside, const float (&v)[4]) {
  const uint32_t a = uint32_t(bf16_bits_rne(v[0])) | uint32_t(bf16_bits_rne(v[1])) << 16;
  const uint32_t b = uint32_t(bf16_bits_rne(v[2])) | uint32_t(bf16_bits_rne(v[3])) << 16;
  if (inside >= 4) {
    *reinterpret_cast<u32x2_any *>(p) = u32x2_any{a, b};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < inside) p[e].bits = uint16_t((e < 2 ? a : b) >> 16 * (e & 1));
  }
}
__device__ __forceinline__ void write4(uint8_t *p, int inside, uint32_t v) {
  if (inside >= 4) {
    *reinterpret_cast<u32_any *>(p) = v;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < inside) p[e] = uint8_t(v >> 8 * e);
  }
}

// Products and sums that are rounded one by one.
__device__ __forceinline__ float times(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}
__device__ __forceinline__ float plus(float a, float b) {
#pragma clang fp contract(off)
  return a + b;
}

// A power of two from its biased exponent (1..254).
__device__ __forceinline__ float power(int biased) { return __uint_as_float(uint32_t(biased) << 23); }

// BIAS 7: m, BIAS 15: v.
template <int BIAS>
struct Format {
  static constexpr int kTop = BIAS == 7 ? 134 : 142;          // y = magnitude * 2^(kTop - E)
  static constexpr uint32_t kNone = BIAS == 7 ? 127u : 255u;  // infinities and NaN
  static constexpr int kLeastExponent = 16;

  __device__ static __forceinline__ float value(uint32_t code, int E) {
    const uint32_t mag = BIAS == 7 ? code & 127u : code;
    // the code's bits as an fp32 number's are the value times 2^(BIAS - 127), below the normal numbers too
    float y = __uint_as_float(mag << 20) * power(254 - BIAS) * power(E < kLeastExponent ? 127 : E + 127 - kTop);
    y = mag == kNone ? __builtin_nanf("") : y;
    return BIAS == 7 && (code & 128u) ? -y : y;
  }

  // The shared exponent of a wavefront's values: 4 a lane.
  __device__ static __forceinline__ int exponent(const float (&x)[4]) {
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t b = __float_as_uint(x[e]) & 0x7fffffffu;
      top = b < 0x7f800000u && b > top ? b : top;
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const uint32_t other = __shfl_xor(top, d);
      top = other > top ? other : top;
    }
    const int E = int(top >> 23);
    return __builtin_amdgcn_readfirstlane(E < kLeastExponent ? kLeastExponent : E);
  }

  __device__ static __forceinline__ uint32_t code(float x, int E, uint32_t r) {
    const uint32_t bits = __float_as_uint(x), mag = bits & 0x7fffffffu;
    const float y = times(__uint_as_float(mag), power(kTop + 127 - E));
    const uint32_t normal = ((__float_as_uint(y) + 16u * r) >> 20) - 8u * (127 - BIAS);
    const uint32_t below = uint32_t(plus(times(y, power(127 + BIAS + 2)), times(float(r), 0x1p-16f)));
    uint32_t c = y < power(127 + 1 - BIAS) ? below : normal;
    c = mag < 0x7f800000u ? c : kNone;
    return BIAS == 7 ? c | (bits >> 31) << 7 : c;
  }
};

template <class ST, bool Eight, bool Copy>
__global__ __launch_bounds__(kThreads) void adamw_kernel(StepArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t first = int64_t(blockIdx.x) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), stride = int64_t(gridDim.x) * kWaves;
  for (int worker = blockIdx.y; worker < a.n; worker += gridDim.y)
  for (int64_t b = first; b < a.count; b += stride) {
    const AdamwBlock blk = a.blocks[b];
    const int inside = blk.count - kLaneCols * lane;
    const int64_t at = int64_t(worker) * a.ld + blk.start + kLaneCols * lane;
    float g[4], x[4], m[4], v[4];
    read4(a.g + at, inside, g);
    read4(static_cast<const ST *>(a.x) + at, inside, x);
    uint8_t *const scale = a.scales + 2 * (int64_t(worker) * a.count + b);
    if constexpr (Eight) {
      const uint32_t cm = read4(static_cast<const uint8_t *>(a.m) + at, inside), cv = read4(static_cast<const uint8_t *>(a.v) + at, inside);
      const int Em = scale[0], Ev = scale[1];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        m[e] = Format<7>::value((cm >> 8 * e) & 255u, Em);
        v[e] = Format<15>::value((cv >> 8 * e) & 255u, Ev);
      }
    } else {
      read4(static_cast<const float *>(a.m) + at, inside, m);
      read4(static_cast<const float *>(a.v) + at, inside, v);
    }
    const float lr = a.lr * blk.lr_scale, keep = 1.f - lr * blk.decay;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      m[e] = plus(times(m[e], a.beta1), times(g[e], a.rest1));
      v[e] = plus(times(v[e], a.beta2), times(times(g[e], g[e]), a.rest2));
      float step = (m[e] * a.unbias1) / (sqrtf(v[e] * a.unbias2) + a.eps);
      step = step > a.limit ? a.limit : step < -a.limit ? -a.limit : step;  // NaN stays
      x[e] = x[e] * keep - lr * step;
    }
    write4(static_cast<ST *>(a.x) + at, inside, x);
    if constexpr (Copy) write4(reinterpret_cast<bf16_t *>(a.x16) + at, inside, x);
    if constexpr (Eight) {
      const int Em = Format<7>::exponent(m), Ev = Format<15>::exponent(v);
      uint32_t r[4], cm = 0, cv = 0;
      const uint64_t id = uint64_t(b) * 64 + lane;
      philox4x32_10(uint32_t(id), 0x41646157u + uint32_t(id >> 32), worker, a.t, a.seed_lo, a.seed_hi, r);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        cm |= Format<7>::code(m[e], Em, r[e] & 0xffffu) << 8 * e;
        cv |= Format<15>::code(v[e], Ev, r[e] >> 16) << 8 * e;
      }
      write4(static_cast<uint8_t *>(a.m) + at, inside, cm);
      write4(static_cast<uint8_t *>(a.v) + at, inside, cv);
      if (lane == 0) scale[0] = uint8_t(Em), scale[1] = uint8_t(Ev);
    } else {
      write4(static_cast<float *>(a.m) + at, inside, m);
      write4(static_cast<float *>(a.v) + at, inside, v);
    }
  }
}

// What 8-bit moments stand for, as OT (exact in either type).
template <class OT>
__global__ __launch_bounds__(kThreads) void adamw_values_kernel(const uint8_t *m, const uint8_t *v, const uint8_t *scales,
                                                                const AdamwBlock *blocks, int n, int64_t ld, int64_t count, OT *m_out, OT *v_out) {
  const int lane = threadIdx.x & 63;
  const int64_t first = int64_t(blockIdx.x) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), stride = int64_t(gridDim.x) * kWaves;
  for (int worker = blockIdx.y; worker < n; worker += gridDim.y)
  for (int64_t b = first; b < count; b += stride) {
    const AdamwBlock blk = blocks[b];
    const int inside = blk.count - kLaneCols * lane;
    const int64_t at = int64_t(worker) * ld + blk.start + kLaneCols * lane;
    const uint8_t *const scale = scales + 2 * (int64_t(worker) * count + b);
    const uint32_t cm = read4(m + at, inside), cv = read4(v + at, inside);
    const int Em = scale[0], Ev = scale[1];
    float fm[4], fv[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      fm[e] = Format<7>::value((cm >> 8 * e) & 255u, Em);
      fv[e] = Format<15>::value((cv >> 8 * e) & 255u, Ev);
    }
    write4(m_out + at, inside, fm);
    write4(v_out + at, inside, fv);
  }
}

dim3 grid_of(int n, int64_t count) {
  int64_t x = (count + kWaves - 1) / kWaves;
  if (x > 4096) x = 4096;
  return dim3(uint32_t(x < 1 ? 1 : x), uint32_t(n < 32768 ? n : 32768));
}

template <class ST>
int launch_step(const StepArgs &a, int n, bool eight, void *stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const dim3 grid = grid_of(n, a.count);
  if (eight) {
    if (a.x16) adamw_kernel<ST, true, true><<<grid, kThreads, 0, st>>>(a);
    else adamw_kernel<ST, true, false><<<grid, kThreads, 0, st>>>(a);
  } else {
    if (a.x16) adamw_kernel<ST, false, true><<<grid, kThreads, 0, st>>>(a);
    else adamw_kernel<ST, false, false><<<grid, kThreads, 0, st>>>(a);
  }
  return hip_rc(hipGetLastError());
}

}  // namespace

int launch_adamw(const Shape &s, const AdamwBlock *blocks, int64_t count, bool eight, void *X, const float *G, void *M, void *V, uint8_t *S,
                 uint16_t *X16, const AdamwNumbers &h, void *stream) {
  StepArgs a{X, G, M, V, S, X16, blocks, s.ld, count, s.n, h.lr, h.beta1, h.rest1, h.beta2, h.rest2, h.eps, h.unbias1, h.unbias2, h.limit,
             h.t, uint32_t(h.seed), uint32_t(h.seed >> 32)};
  return s.bf16 ? launch_step<bf16_t>(a, s.n, eight, stream) : launch_step<float>(a, s.n, eight, stream);
}

int launch_adamw_values(const Shape &s, const AdamwBlock *blocks, int64_t count, const uint8_t *M, const uint8_t *V, const uint8_t *S,
                        bool bf16, void *M_out, void *V_out, void *stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const dim3 grid = grid_of(s.n, count);
  if (bf16) adamw_values_kernel<<<grid, kThreads, 0, st>>>(M, V, S, blocks, s.n, s.ld, count, static_cast<bf16_t *>(M_out), static_cast<bf16_t *>(V_out));
  else adamw_values_kernel<<<grid, kThreads, 0, st>>>(M, V, S, blocks, s.n, s.ld, count, static_cast<float *>(M_out), static_cast<float *>(V_out));
  return hip_rc(hipGetLastError());
}

}  // namespace detag

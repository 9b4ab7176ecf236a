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
// of two costs no precision in a floating format, and every kept value has four significant bits, which bfloat16 holds too, but for the
// least of v under E < 26 (below 2^-133).  The rounding is stochastic: v moves by (1 - beta2) of itself a step, far less than half the
// spacing of three mantissa bits, so that the nearest value would never change.  Random bits: Philox-4x32-10 (noise_dev.hpp), counter
// (64 * block + lane, 0x41646157, worker, t), key = seed; word j of the lane's four is column j's, its lower half rounds m, the upper one v.
//
//   E = biased fp32 exponent of the largest finite magnitude, at least 16
//   y = |m| 2^(134-E) or v 2^(142-E);  least normal number 2^-6 or 2^-14
//   code = ((bits(y) + 16 r) >> 20) - 8 (127 - bias) from there on, below floor(2^9 y + 2^-16 r) or floor(2^17 y + 2^-16 r)
// so the largest magnitude has the last exponent but one, and rounding up needs no clamp.  Infinities and NaN become the code with
// all bits set (127, 255), which is read back as NaN.
//
// The moments' arithmetic is rounded operation by operation (no fused multiply-add), so that it can be restated bit by bit.
//
// Measured: 64 workers of 11,173,962, fp32 moments 3.5 to 3.9 ms (20.0 GB, 5.2 to 5.8 TB/s); 256 of 1,048,576, 8 bits with the bf16 copy
// 0.99 ms (4.8 GB, 4.9 TB/s); 16 of 272,474, 8 bits 15 us.
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
template <bool Stream, class V>
__device__ __forceinline__ V fetch(const V *p) {
  return Stream ? __builtin_nontemporal_load(p) : *p;
}
template <bool Stream, class V>
__device__ __forceinline__ void put(V *p, V v) {
  if constexpr (Stream) __builtin_nontemporal_store(v, p);
  else *p = v;
}
template <bool Stream>
__device__ __forceinline__ void read4(const float *p, int inside, float (&v)[4]) {
  if (inside >= 4) {
    const f32x4 r = fetch<Stream>(reinterpret_cast<const f32x4_any *>(p));
    v[0] = r[0], v[1] = r[1], v[2] = r[2], v[3] = r[3];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = e < inside ? p[e] : 0.f;
  }
}
template <bool Stream>
__device__ __forceinline__ void read4(const bf16_t *p, int inside, float (&v)[4]) {
  if (inside >= 4) {
    const u32x2_any r = fetch<Stream>(reinterpret_cast<const u32x2_any *>(p));
    v[0] = __uint_as_float(r[0] << 16), v[1] = __uint_as_float(r[0] & 0xffff0000u);
    v[2] = __uint_as_float(r[1] << 16), v[3] = __uint_as_float(r[1] & 0xffff0000u);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = e < inside ? to_f32(p[e]) : 0.f;
  }
}
template <bool Stream>
__device__ __forceinline__ uint32_t read4(const uint8_t *p, int inside) {
  if (inside >= 4) return fetch<Stream>(reinterpret_cast<const u32_any *>(p));
  uint32_t v = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < inside) v |= uint32_t(p[e]) << 8 * e;
  return v;
}
template <bool Stream>
__device__ __forceinline__ void write4(float *p, int inside, const float (&v)[4]) {
  if (inside >= 4) {
    put<Stream>(reinterpret_cast<f32x4_any *>(p), f32x4_any{v[0], v[1], v[2], v[3]});
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < inside) p[e] = v[e];
  }
}
template <bool Stream>
__device__ __forceinline__ void write4(bf16_t *p, int inside, const float (&v)[4]) {
  const uint32_t a = uint32_t(bf16_bits_rne(v[0])) | uint32_t(bf16_bits_rne(v[1])) << 16;
  const uint32_t b = uint32_t(bf16_bits_rne(v[2])) | uint32_t(bf16_bits_rne(v[3])) << 16;
  if (inside >= 4) {
    put<Stream>(reinterpret_cast<u32x2_any *>(p), u32x2_any{a, b});
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < inside) p[e].bits = uint16_t((e < 2 ? a : b) >> 16 * (e & 1));
  }
}
template <bool Stream>
__device__ __forceinline__ void write4(uint8_t *p, int inside, uint32_t v) {
  if (inside >= 4) {
    put<Stream>(reinterpret_cast<u32_any *>(p), u32_any(v));
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

// The largest of 64 lanes' values, as a scalar.
template <int CTRL>
__device__ __forceinline__ uint32_t max_dpp(uint32_t v) {
  const uint32_t o = uint32_t(__builtin_amdgcn_update_dpp(0, int(v), CTRL, 0xf, 0xf, true));
  return o > v ? o : v;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = max_dpp<0x128>(v), v = max_dpp<0x124>(v), v = max_dpp<0x122>(v), v = max_dpp<0x121>(v);  // rotations within 16 lanes
  v = max_dpp<0x142>(v), v = max_dpp<0x143>(v);  // rows of 16 into the next, halves into the next: lane 63 has all
  return uint32_t(__builtin_amdgcn_readlane(int(v), 63));
}

// BIAS 7: m, BIAS 15: v.
template <int BIAS>
struct Format {
  static constexpr int kTop = BIAS == 7 ? 134 : 142;          // y = magnitude * 2^(kTop - E)
  static constexpr uint32_t kNone = BIAS == 7 ? 127u : 255u;  // infinities and NaN
  static constexpr int kLeastExponent = 16;

  // What the four codes of a lane stand for.
  __device__ static __forceinline__ void values(uint32_t codes, int E, float (&v)[4]) {
    E = E < kLeastExponent ? kLeastExponent : E;
    // a code's bits as an fp32 number's are the value times 2^(BIAS - 127), below the normal numbers too
    const float up = power(254 - BIAS), scale = power(E + 127 - kTop);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t mag = (codes >> 8 * e) & (BIAS == 7 ? 127u : 255u);
      float y = __uint_as_float(mag << 20) * up * scale;
      if (BIAS == 7) y = __uint_as_float(__float_as_uint(y) | ((codes << (24 - 8 * e)) & 0x80000000u));
      v[e] = y;
    }
    // a code with all bits set: rare, so looked for in all four at once
    const uint32_t none = BIAS == 7 ? ((codes & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u : codes & ((codes & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
    if (__ballot(none != 0)) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (none >> 8 * e & 0x80u) v[e] = __builtin_nanf("");
    }
  }

  // The codes of a wavefront's values, four a lane, with 16 random bits each (`SHIFT` bits up in r), and their exponent.
  template <int SHIFT>
  __device__ static __forceinline__ uint32_t codes(const float (&x)[4], const uint32_t (&r)[4], int &E) {
    uint32_t mag[4], top = 0, least = 0xffffffffu;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      mag[e] = __float_as_uint(x[e]) & 0x7fffffffu;
      top = mag[e] > top ? mag[e] : top, least = mag[e] < least ? mag[e] : least;
    }
    const uint32_t all = wave_max(top);
    E = int(all >> 23);
    // Nearly always everything is finite, and normal numbers in between: then y 2^(BIAS - 127) has the code as its upper bits.
    if (E >= 30 && E <= 140 && !__ballot(least < uint32_t(E - kTop + 128 - BIAS) << 23)) {
      const float scale = power(kTop + BIAS - E);
      uint32_t c = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t u = __float_as_uint(x[e] * scale) + ((SHIFT ? r[e] >> SHIFT : r[e] & 0xffffu) << 4);
        const uint32_t code = BIAS == 7 ? (u >> 20 & 0x7fu) | (u >> 24 & 0x80u) : u >> 20;
        c |= code << 8 * e;
      }
      return c;
    }
    if (all >= 0x7f800000u) {  // the finite ones count
      top = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) top = mag[e] < 0x7f800000u && mag[e] > top ? mag[e] : top;
      E = int(wave_max(top) >> 23);
    }
    E = E < kLeastExponent ? kLeastExponent : E;
    uint32_t c = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t random = SHIFT ? r[e] >> SHIFT : r[e] & 0xffffu;
      const float y = times(__uint_as_float(mag[e]), power(kTop + 127 - E));
      const uint32_t normal = ((__float_as_uint(y) + 16u * random) >> 20) - 8u * (127 - BIAS);
      const uint32_t below = uint32_t(plus(times(y, power(127 + BIAS + 2)), times(float(random), 0x1p-16f)));
      uint32_t code = y < power(127 + 1 - BIAS) ? below : normal;
      code = mag[e] < 0x7f800000u ? code : kNone;
      c |= (BIAS == 7 ? code | (__float_as_uint(x[e]) >> 31) << 7 : code) << 8 * e;
    }
    return c;
  }
};

// A wavefront takes a block.  (Several at a time, to have more loads under way: 64 workers of 3,000,000, 8 bits with the copy 630 us with
// one, 717 with two, 739 with four; 32 bits 990, 1054, 1010.)
template <class ST, bool Eight, bool Copy, bool Stream>
__global__ __launch_bounds__(kThreads) void adamw_kernel(StepArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t first = int64_t(blockIdx.x) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), stride = int64_t(gridDim.x) * kWaves;
  for (int worker = blockIdx.y; worker < a.n; worker += gridDim.y)
    for (int64_t b = first; b < a.count; b += stride) {
      const AdamwBlock blk = a.blocks[b];
      const int inside = blk.count - kLaneCols * lane;
      const int64_t at = int64_t(worker) * a.ld + blk.start + kLaneCols * lane;
      float g[4], x[4], m[4], v[4];
      read4<Stream>(a.g + at, inside, g);
      read4<Stream>(static_cast<const ST *>(a.x) + at, inside, x);
      uint8_t *const scale = a.scales + 2 * (int64_t(worker) * a.count + b);
      if constexpr (Eight) {
        const uint32_t cm = read4<Stream>(static_cast<const uint8_t *>(a.m) + at, inside), cv = read4<Stream>(static_cast<const uint8_t *>(a.v) + at, inside);
        const int Em = __builtin_amdgcn_readfirstlane(scale[0]), Ev = __builtin_amdgcn_readfirstlane(scale[1]);
        Format<7>::values(cm, Em, m);
        Format<15>::values(cv, Ev, v);
      } else {
        read4<Stream>(static_cast<const float *>(a.m) + at, inside, m);
        read4<Stream>(static_cast<const float *>(a.v) + at, inside, v);
      }
      const float lr = a.lr * blk.lr_scale, keep = 1.f - lr * blk.decay;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        m[e] = plus(times(m[e], a.beta1), times(g[e], a.rest1));
        v[e] = plus(times(v[e], a.beta2), times(times(g[e], g[e]), a.rest2));
        // root and reciprocal of the hardware, within 2^-22 of the step (a v below 2^-126 counts as zero there)
        float step = m[e] * a.unbias1 * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v[e] * a.unbias2) + a.eps);
        step = step > a.limit ? a.limit : step < -a.limit ? -a.limit : step;  // NaN stays
        x[e] = x[e] * keep - lr * step;
      }
      write4<Stream>(static_cast<ST *>(a.x) + at, inside, x);
      if constexpr (Copy) write4<Stream>(reinterpret_cast<bf16_t *>(a.x16) + at, inside, x);
      if constexpr (Eight) {
        uint32_t r[4];
        int Em, Ev;
        const uint64_t id = uint64_t(b) * 64 + lane;
        philox4x32_10(uint32_t(id), 0x41646157u + uint32_t(id >> 32), worker, a.t, a.seed_lo, a.seed_hi, r);
        write4<Stream>(static_cast<uint8_t *>(a.m) + at, inside, Format<7>::codes<0>(m, r, Em));
        write4<Stream>(static_cast<uint8_t *>(a.v) + at, inside, Format<15>::codes<16>(v, r, Ev));
        if (lane == 0) scale[0] = uint8_t(Em), scale[1] = uint8_t(Ev);
      } else {
        write4<Stream>(static_cast<float *>(a.m) + at, inside, m);
        write4<Stream>(static_cast<float *>(a.v) + at, inside, v);
      }
    }
}

// What 8-bit moments stand for, as OT.
template <class OT, int Blocks>
__global__ __launch_bounds__(kThreads) void adamw_values_kernel(const uint8_t *m, const uint8_t *v, const uint8_t *scales,
                                                                const AdamwBlock *blocks, int n, int64_t ld, int64_t count, OT *m_out, OT *v_out) {
  const int lane = threadIdx.x & 63;
  const int64_t first = (int64_t(blockIdx.x) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * Blocks;
  const int64_t stride = int64_t(gridDim.x) * kWaves * Blocks;
  for (int worker = blockIdx.y; worker < n; worker += gridDim.y)
    for (int64_t b0 = first; b0 < count; b0 += stride) {
      int64_t at[Blocks];
      int inside[Blocks];
      uint32_t cm[Blocks], cv[Blocks], E[Blocks];
#pragma unroll
      for (int k = 0; k < Blocks; ++k) {
        const int64_t b = b0 + k < count ? b0 + k : count - 1;
        const AdamwBlock blk = blocks[b];
        inside[k] = b0 + k < count ? blk.count - kLaneCols * lane : 0;
        at[k] = int64_t(worker) * ld + blk.start + kLaneCols * lane;
        const uint8_t *const s = scales + 2 * (int64_t(worker) * count + b);
        cm[k] = read4<false>(m + at[k], inside[k]), cv[k] = read4<false>(v + at[k], inside[k]);
        E[k] = s[0] | uint32_t(s[1]) << 8;
      }
#pragma unroll
      for (int k = 0; k < Blocks; ++k) {
        float fm[4], fv[4];
        Format<7>::values(cm[k], __builtin_amdgcn_readfirstlane(E[k] & 255), fm);
        Format<15>::values(cv[k], __builtin_amdgcn_readfirstlane(E[k] >> 8), fv);
        write4<false>(m_out + at[k], inside[k], fm);
        write4<false>(v_out + at[k], inside[k], fv);
      }
    }
}

dim3 grid_of(int n, int64_t count, int blocks) {
  int64_t x = (count + kWaves * blocks - 1) / (kWaves * blocks);
  if (x > 65536) x = 65536;
  return dim3(uint32_t(x < 1 ? 1 : x), uint32_t(n < 32768 ? n : 32768));
}

template <class ST, bool Eight, bool Copy>
int launch_step(const StepArgs &a, void *stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const dim3 grid = grid_of(a.n, a.count, 1);
  // fp32 moments that the memory-side cache cannot hold stream past it: 64 workers of 11,173,962 3.32 ms (3.56), of 3,000,000 992 us
  // (1047); 8-bit ones gain nothing: 571 us (562)
  if constexpr (!Eight)
    if (int64_t(a.n) * a.count * kBlock * (20 + 2 * int64_t(sizeof(ST))) >= int64_t(256) << 20) {
      adamw_kernel<ST, Eight, Copy, true><<<grid, kThreads, 0, st>>>(a);
      return hip_rc(hipGetLastError());
    }
  adamw_kernel<ST, Eight, Copy, false><<<grid, kThreads, 0, st>>>(a);
  return hip_rc(hipGetLastError());
}
template <class ST>
int launch_step(const StepArgs &a, bool eight, void *stream) {
  if (eight) return a.x16 ? launch_step<ST, true, true>(a, stream) : launch_step<ST, true, false>(a, stream);
  return a.x16 ? launch_step<ST, false, true>(a, stream) : launch_step<ST, false, false>(a, stream);
}

template <class OT>
int launch_values(const uint8_t *M, const uint8_t *V, const uint8_t *S, const AdamwBlock *blocks, int n, int64_t ld, int64_t count, OT *M_out,
                  OT *V_out, hipStream_t st) {
  constexpr int kMany = 4;
  // 64 workers of 3,000,000: 205 us with four blocks a wavefront, 286 with one; 16 of 272,474: 8.1 and 7.0
  if (int64_t(n) * count >= 65536)
    adamw_values_kernel<OT, kMany><<<grid_of(n, count, kMany), kThreads, 0, st>>>(M, V, S, blocks, n, ld, count, M_out, V_out);
  else adamw_values_kernel<OT, 1><<<grid_of(n, count, 1), kThreads, 0, st>>>(M, V, S, blocks, n, ld, count, M_out, V_out);
  return hip_rc(hipGetLastError());
}

}  // namespace

int launch_adamw(const Shape &s, const AdamwBlock *blocks, int64_t count, bool eight, void *X, const float *G, void *M, void *V, uint8_t *S,
                 uint16_t *X16, const AdamwNumbers &h, void *stream) {
  StepArgs a{X, G, M, V, S, X16, blocks, s.ld, count, s.n, h.lr, h.beta1, h.rest1, h.beta2, h.rest2, h.eps, h.unbias1, h.unbias2, h.limit,
             h.t, uint32_t(h.seed), uint32_t(h.seed >> 32)};
  return s.bf16 ? launch_step<bf16_t>(a, eight, stream) : launch_step<float>(a, eight, stream);
}

int launch_adamw_values(const Shape &s, const AdamwBlock *blocks, int64_t count, const uint8_t *M, const uint8_t *V, const uint8_t *S,
                        bool bf16, void *M_out, void *V_out, void *stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (bf16) return launch_values(M, V, S, blocks, s.n, s.ld, count, static_cast<bf16_t *>(M_out), static_cast<bf16_t *>(V_out), st);
  return launch_values(M, V, S, blocks, s.n, s.ld, count, static_cast<float *>(M_out), static_cast<float *>(V_out), st);
}

}  // namespace detag

// What the kernels over row matrices share: pieces of 16 bytes of a row, sums over lanes, and which worker (or sequence) a row or a run
// of rows belongs to.
#pragma once

#include "dev_common.hpp"

namespace detag {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));  // at any address its elements may have

// Elements of a piece as floats.
template <class T>
__device__ __forceinline__ float element(u32x4 v, int e) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(v[e]);
  else return __uint_as_float(e % 2 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16);
}

// The piece at p, of which `inside` elements (they may be none) belong to the row; the others read as zero.
template <class T>
__device__ __forceinline__ u32x4 load_piece(const T *p, int inside) {
  constexpr int kElems = 16 / sizeof(T);
  if (inside >= kElems) return *reinterpret_cast<const u32x4_any *>(p);
  union {
    u32x4 v;
    T e[kElems];
  } u;
  u.v = u32x4{0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < kElems; ++e)
    if (e < inside) u.e[e] = p[e];
  return u.v;
}

// Writes the first `inside` of a piece's values, each rounded once.
template <class T>
__device__ __forceinline__ void store_piece(T *p, const float (&v)[16 / sizeof(T)], int inside) {
  constexpr int kElems = 16 / sizeof(T);
  if (inside >= kElems) {
    u32x4 b;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if constexpr (sizeof(T) == 4) b[w] = __float_as_uint(v[w]);
      else b[w] = bf16_pair(v[2 * w], v[2 * w + 1]);
    }
    *reinterpret_cast<u32x4_any *>(p) = b;
  } else {
#pragma unroll
    for (int e = 0; e < kElems; ++e)
      if (e < inside) p[e] = from_f32<T>(v[e]);
  }
}

// The sum over a wavefront's lanes, in every lane, in an order that is always the same.
__device__ __forceinline__ float wave_sum(float v) {
#define DETAG_ADD_LANES(control, rows) \
  v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), control, rows, 0xf, false))
  DETAG_ADD_LANES(0x111, 0xf);  // the lane 1, 2, 4, 8 below, in rows of 16
  DETAG_ADD_LANES(0x112, 0xf);
  DETAG_ADD_LANES(0x114, 0xf);
  DETAG_ADD_LANES(0x118, 0xf);
  DETAG_ADD_LANES(0x142, 0xa);  // the last of the row before, into every second row
  DETAG_ADD_LANES(0x143, 0xc);  // the last of the lower half
#undef DETAG_ADD_LANES
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

// Sums over the lanes up to each.
__device__ __forceinline__ int wave_scan(int v) {
#define DETAG_ADD_LANES(control, rows) v += __builtin_amdgcn_update_dpp(0, v, control, rows, 0xf, false)
  DETAG_ADD_LANES(0x111, 0xf);
  DETAG_ADD_LANES(0x112, 0xf);
  DETAG_ADD_LANES(0x114, 0xf);
  DETAG_ADD_LANES(0x118, 0xf);
  DETAG_ADD_LANES(0x142, 0xa);
  DETAG_ADD_LANES(0x143, 0xc);
#undef DETAG_ADD_LANES
  return v;
}

// Runs of `high` rows of every part (a worker, a sequence), numbered so that a number tells its part without a sum over those before:
// part i's first run has the number off_i / high + i, which lies past the last of part i - 1, since floor(x) + 1 >= ceil(x).  There are
// fewer than part_runs() numbers; some belong to no run.
struct Run {
  int part, lo, hi;  // part -1: none; the part's rows, within the matrix whatever the offsets say
  int first;         // the run's first row
};
__host__ __device__ inline int64_t part_runs(int64_t rows, int parts, int high) { return rows / high + parts; }

__device__ __forceinline__ int within(int at, int rows) { return at < 0 ? 0 : at > rows ? rows : at; }

// The run of a number (high = 0: a number is a row, and a run is that row).  All lanes of a wavefront ask for the same one: each looks at
// another part, 64 at a time, and where there are more, first at every 64th of them.
__device__ __forceinline__ Run run_of(const int32_t *offsets, int parts, int rows, int high, int number) {
  const int lane = threadIdx.x & 63;
  auto start = [&](int i) {
    const int at = within(offsets[i], rows);
    return high ? at / high + i : at;
  };
  int base = 0, count = parts;
  while (count > 64) {
    const int stride = (count + 63) / 64, upto = (lane + 1) * stride < count ? (lane + 1) * stride : count;
    const unsigned long long holds = __ballot(start(base + upto) > number);
    if (!holds) return {-1, 0, 0, 0};
    const int before = (__builtin_amdgcn_readfirstlane(__ffsll(holds)) - 1) * stride;
    base += before, count = count - before < stride ? count - before : stride;
  }
  int lo = 0, hi = 0, next = 0, own = 0;
  if (lane < count) {
    lo = within(offsets[base + lane], rows), hi = within(offsets[base + lane + 1], rows);
    own = high ? lo / high + base + lane : lo, next = high ? hi / high + base + lane + 1 : hi;
  }
  const unsigned long long holds = __ballot(lane < count && next > number);
  if (!holds) return {-1, 0, 0, 0};
  const int at = __builtin_amdgcn_readfirstlane(__ffsll(holds)) - 1;
  Run r;
  r.lo = __builtin_amdgcn_readlane(lo, at), r.hi = __builtin_amdgcn_readlane(hi, at);
  const int64_t first = high ? r.lo + int64_t(number - __builtin_amdgcn_readlane(own, at)) * high : number;
  r.part = first >= r.lo && first < r.hi ? base + at : -1, r.first = int(first);
  return r;
}

}  // namespace detag

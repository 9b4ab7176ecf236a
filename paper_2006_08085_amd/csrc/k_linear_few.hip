// Products of a layer in calls of few tiles.  A tile of k_linear.hip walks the whole contraction step by step, and few tiles leave most
// compute units without one; here the wavefronts of a block share the contraction, each requests a stretch of its own, and the block
// adds up the parts at the end.  What bounds calls of few rows is the weights, which are read once, and how many of those bytes are
// on their way at a time; calls of more rows and the weight gradient, the length of a wavefront's stretch.
//
//   linear_few           forward: a block computes 16 outputs of 16 rows.  Weights and rows go straight from memory to the matrix cores,
//                        16 bytes a lane along the contraction.
//   linear_shared        forward or input gradient: a block computes 64 columns of 16 or 64 rows.  Every wavefront has LDS buffers of its
//                        own, filled past the registers, and needs no barrier until the parts are added up.
//   linear_weight_split  weight gradient: 64 x 64 weights in the same way, the wavefronts share the worker's rows.
// Further rows of a worker are further passes over the same weights, which the caches hold by then, by blocks of their own.
#include "dev_common.hpp"
#include "detag_internal.h"
#include "linear_common.hpp"

namespace detag {
namespace {

constexpr int kOuts = 16;       // outputs of a forward block
constexpr int kAhead = 8;       // loads of a lane under way

// 16 bytes at p, of which `inside` elements belong to the row; the others as zero.
template <class T>
__device__ __forceinline__ u32x4 load16(const T *p, int inside) {
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

// grid (ceil(out / 16), n, passes).  8 workers of one row, 1024 -> 1024 bf16 (16.8 MB) 5.0 us; 1 row, 4096 -> 4096 (33.6 MB) 7.6 us.
template <class T, class TC, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void linear_few_kernel(LinearArgs a) {
  constexpr int kElems = 16 / sizeof(T), kStep = 4 * kElems;  // contracted elements of a load: four lanes of a row
  __shared__ f32x4 parts[WAVES][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, lane = threadIdx.x & 63, p = lane & 15, q = lane >> 4;
  const int out0 = blockIdx.x * kOuts;
  const int steps = (a.in + kStep - 1) / kStep;
  for (int worker = blockIdx.y; worker < a.n; worker += gridDim.y) {
    int lo, hi;
    worker_rows(a, worker, lo, hi);
    const int o = out0 + p < a.out ? out0 + p : a.out - 1;  // rows past the end repeat the last and are not stored
    const T *w = static_cast<const T *>(a.w) + int64_t(worker) * a.ld + int64_t(o) * a.in + q * kElems;
    for (int r0 = lo + int(blockIdx.z) * 16; r0 < hi; r0 += int(gridDim.z) * 16) {
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
      const T *row = static_cast<const T *>(a.rows_a) + int64_t(r0 + p < hi ? r0 + p : hi - 1) * a.lda + q * kElems;  // likewise
      // wavefronts take pairs of steps (a cache line of bf16) in turn
      for (int s0 = 2 * wave; s0 < steps; s0 += kAhead * waves) {
        u32x4 x[kAhead], y[kAhead];
        auto at = [&](int u) { return (s0 + u / 2 * 2 * waves + u % 2) * kStep; };
        if (at(kAhead - 1) + kStep <= a.in) {  // uniform: all whole
#pragma unroll
          for (int u = 0; u < kAhead; ++u) x[u] = *reinterpret_cast<const u32x4_any *>(w + at(u));
#pragma unroll
          for (int u = 0; u < kAhead; ++u) y[u] = *reinterpret_cast<const u32x4_any *>(row + at(u));
        } else {
#pragma unroll
          for (int u = 0; u < kAhead; ++u) x[u] = load16(w + at(u), a.in - at(u) - q * kElems);
#pragma unroll
          for (int u = 0; u < kAhead; ++u) y[u] = load16(row + at(u), a.in - at(u) - q * kElems);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) acc = multiply<T>(x[u], y[u], acc);
      }
      __syncthreads();
      parts[wave][lane] = acc;
      __syncthreads();
      const int r = r0 + p;
      if (wave == 0 && r < hi) {
        f32x4 v = parts[0][lane];
        for (int k = 1; k < waves; ++k) v += parts[k][lane];
        if (a.flag)
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = v[e] <= 0.f ? 0.f : v[e];  // NaN stays
        store4(static_cast<TC *>(a.c) + int64_t(r) * a.ldc + out0 + 4 * q, v, a.out - out0 - 4 * q);
      }
    }
  }
}

constexpr int kSharedCols = 64;  // columns of a block

// grid (ceil(columns / 64), n, passes).  1 row, 4096 -> 4096 bf16, input gradient 10.5 us; 128 rows forward 16.9 us, input gradient 19.5 us.
template <bool Forward, class T, class TC, int GROUPS, int WAVES, bool Direct>
__global__ __launch_bounds__(64 * WAVES) void linear_shared_kernel(LinearArgs a) {
  using Rows = Operand<T, kAlong, 16 * GROUPS, 1, 64, false, Direct>;
  using Cols = Operand<T, Forward ? kAlong : kAcross, kSharedCols, 1, 64, false, Direct>;
  constexpr int kBuffer = Rows::kTileBytes + Cols::kTileBytes, kLoads = Rows::kLoads + Cols::kLoads, kFn = kSharedCols / 16;
  __shared__ __attribute__((aligned(1024))) char lds_[WAVES * 2 * kBuffer];
  static_assert(2 * kBuffer >= GROUPS * kFn * 64 * 16, "a wavefront's part of the results fits its buffers");
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, p = lane & 15, q = lane >> 4;
  const uint32_t lds = uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)lds_)), own = lds + wave * 2 * kBuffer;
  const int columns = Forward ? a.out : a.in, contracted = Forward ? a.in : a.out;
  const int column = blockIdx.x * kSharedCols, width = columns - column < kSharedCols ? columns - column : kSharedCols;
  const typename Rows::Bases row_bases = Rows::template bases<GROUPS>(0);
  const typename Cols::Bases col_bases = Cols::template bases<kFn>(0);
  const int steps = (contracted + Rows::kSteps - 1) / Rows::kSteps, mine = (steps - wave + WAVES - 1) / WAVES;  // in turn
  const int rest = contracted - (steps - 1) * Rows::kSteps;  // of the last
  for (int worker = blockIdx.y; worker < a.n; worker += gridDim.y) {
    int lo, hi;
    worker_rows(a, worker, lo, hi);
    lo = __builtin_amdgcn_readfirstlane(lo), hi = __builtin_amdgcn_readfirstlane(hi);
    const T *w = static_cast<const T *>(a.w) + int64_t(worker) * a.ld + (Forward ? int64_t(column) * a.in : column);
    for (int r0 = lo + int(blockIdx.z) * 16 * GROUPS; r0 < hi; r0 += int(gridDim.z) * 16 * GROUPS) {
      const int count = hi - r0 < 16 * GROUPS ? hi - r0 : 16 * GROUPS;
      f32x4 acc[GROUPS][kFn];
#pragma unroll
      for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        for (int j = 0; j < kFn; ++j) acc[g][j] = f32x4{0.f, 0.f, 0.f, 0.f};
      Rows rows;
      Cols cols;
      rows.init(static_cast<const T *>(a.rows_a) + int64_t(r0) * a.lda, a.lda, count, contracted), rows.advance(wave);
      cols.init(w, a.in, width, contracted), cols.advance(wave);
      auto request = [&](uint32_t buffer) {
#pragma unroll
        for (int it = 0; it < Cols::kLoads; ++it) cols.request(it, buffer + Rows::kTileBytes);
#pragma unroll
        for (int it = 0; it < Rows::kLoads; ++it) rows.request(it, buffer);
        rows.advance(WAVES), cols.advance(WAVES);
      };
      auto deliver = [&](uint32_t buffer) { rows.deliver(buffer, WAVES), cols.deliver(buffer + Rows::kTileBytes, WAVES); };
      if (mine > 0) request(own), deliver(own);
      for (int t = 0; t < mine; ++t) {
        const uint32_t here = own + (t & 1) * kBuffer, other = own + (~t & 1) * kBuffer;
        request(other);  // (zeros after the last)
        if constexpr (Direct) wait_loads<kLoads>();
        asm volatile("" ::: "memory");
        if (Direct && wave + t * WAVES + 1 == steps && rest % Rows::kElems) rows.trim(here, rest), cols.trim(here + Rows::kTileBytes, rest), wait_lds();
#pragma unroll
        for (int s = 0; s < kParts; ++s) {
          u32x4 x[kFn], y[GROUPS];
#pragma unroll
          for (int j = 0; j < kFn; ++j) x[j] = Cols::fragment(col_bases, here + Rows::kTileBytes, j, s);
#pragma unroll
          for (int g = 0; g < GROUPS; ++g) y[g] = Rows::fragment(row_bases, here, g, s);
#pragma unroll
          for (int g = 0; g < GROUPS; ++g)
#pragma unroll
            for (int j = 0; j < kFn; ++j) acc[g][j] = multiply<T>(x[j], y[g], acc[g][j]);
        }
        // the buffer that was read is filled again by the next request
        wait_lds();
        deliver(other);
      }
      wait_all();
#pragma unroll
      for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        for (int j = 0; j < kFn; ++j) *reinterpret_cast<__attribute__((address_space(3))) f32x4 *>(own + ((g * kFn + j) * 64 + lane) * 16) = acc[g][j];
      __syncthreads();
      for (int k = threadIdx.x; k < GROUPS * kFn * 64; k += 64 * WAVES) {  // k = (g * kFn + j) * 64 + a lane's number
        f32x4 v = read_lds<f32x4>(lds + k * 16);
#pragma unroll
        for (int s = 1; s < WAVES; ++s) v += read_lds<f32x4>(lds + s * 2 * kBuffer + k * 16);
        const int r = k / (kFn * 64) * 16 + (k & 15), c = column + k / 64 % kFn * 16 + (k >> 4 & 3) * 4, inside = columns - c;
        if (r >= count || inside <= 0) continue;
        if (Forward && a.flag)
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = v[e] <= 0.f ? 0.f : v[e];  // NaN stays
        if (!Forward && a.rows_b) {
          const f32x4 h = load4(static_cast<const T *>(a.rows_b) + int64_t(r0 + r) * a.ldb + c, inside);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = h[e] > 0.f ? v[e] : 0.f;
        }
        store4(static_cast<TC *>(a.c) + int64_t(r0 + r) * a.ldc + c, v, inside);
      }
      __syncthreads();
    }
  }
}

// grid (tiles of 64 x 64, n).  1 worker of 4096 rows, 256 -> 4096 bf16 25.3 us.
constexpr int kSplitTile = 64, kSplitWaves = 4;
template <class T>
__global__ __launch_bounds__(64 * kSplitWaves) void linear_weight_split_kernel(LinearArgs a) {
  using Part = Operand<T, kAcross, kSplitTile, 1, 64, false, true>;
  constexpr int kBuffer = 2 * Part::kTileBytes, kLoads = 2 * Part::kLoads, kF = kSplitTile / 16;
  __shared__ __attribute__((aligned(1024))) char lds_[kSplitWaves * 2 * kBuffer];
  static_assert(2 * kBuffer >= kSplitTile * kSplitTile * 4, "a wavefront's part of the results fits its buffers");
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const uint32_t lds = uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)lds_)), own = lds + wave * 2 * kBuffer;
  const int across = (a.in + kSplitTile - 1) / kSplitTile, row = blockIdx.x / across * kSplitTile, column = blockIdx.x % across * kSplitTile;
  const int height = a.out - row < kSplitTile ? a.out - row : kSplitTile, width = a.in - column < kSplitTile ? a.in - column : kSplitTile;
  const typename Part::Bases bases = Part::template bases<kF>(0);
  for (int worker = blockIdx.y; worker < a.n; worker += gridDim.y) {
    int lo, hi;
    worker_rows(a, worker, lo, hi);
    lo = __builtin_amdgcn_readfirstlane(lo), hi = __builtin_amdgcn_readfirstlane(hi);
    const int steps = (hi - lo + Part::kSteps - 1) / Part::kSteps, mine = (steps - wave + kSplitWaves - 1) / kSplitWaves;  // in turn
    f32x4 acc[kF][kF];
#pragma unroll
    for (int i = 0; i < kF; ++i)
#pragma unroll
      for (int j = 0; j < kF; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    Part rows, cols;
    rows.init(static_cast<const T *>(a.rows_a) + int64_t(lo) * a.lda + row, a.lda, height, hi - lo), rows.advance(wave);
    cols.init(static_cast<const T *>(a.rows_b) + int64_t(lo) * a.ldb + column, a.ldb, width, hi - lo), cols.advance(wave);
    auto request = [&](uint32_t buffer) {
#pragma unroll
      for (int it = 0; it < Part::kLoads; ++it) rows.request(it, buffer), cols.request(it, buffer + Part::kTileBytes);
      rows.advance(kSplitWaves), cols.advance(kSplitWaves);
    };
    if (mine > 0) request(own);
    for (int t = 0; t < mine; ++t) {
      const uint32_t here = own + (t & 1) * kBuffer, other = own + (~t & 1) * kBuffer;
      request(other);  // (zeros after the last)
      wait_loads<kLoads>();
      asm volatile("" ::: "memory");
#pragma unroll
      for (int s = 0; s < kParts; ++s) {
        u32x4 x[kF], y[kF];
#pragma unroll
        for (int j = 0; j < kF; ++j) x[j] = Part::fragment(bases, here + Part::kTileBytes, j, s), y[j] = Part::fragment(bases, here, j, s);
#pragma unroll
        for (int i = 0; i < kF; ++i)
#pragma unroll
          for (int j = 0; j < kF; ++j) acc[i][j] = multiply<T>(x[j], y[i], acc[i][j]);
      }
      wait_lds();  // the buffer that was read is filled again by the next request
    }
    wait_all();
#pragma unroll
    for (int i = 0; i < kF; ++i)
#pragma unroll
      for (int j = 0; j < kF; ++j) *reinterpret_cast<__attribute__((address_space(3))) f32x4 *>(own + ((i * kF + j) * 64 + lane) * 16) = acc[i][j];
    __syncthreads();
    for (int k = threadIdx.x; k < kF * kF * 64; k += 64 * kSplitWaves) {  // k = (i * kF + j) * 64 + a lane's number
      f32x4 v = read_lds<f32x4>(lds + k * 16);
#pragma unroll
      for (int s = 1; s < kSplitWaves; ++s) v += read_lds<f32x4>(lds + s * 2 * kBuffer + k * 16);
      const int r = k / (kF * 64) * 16 + (k & 15), c = column + k / 64 % kF * 16 + (k >> 4 & 3) * 4, inside = a.in - c;
      if (r >= height || inside <= 0) continue;
      float *const g = static_cast<float *>(a.c) + int64_t(worker) * a.ld + int64_t(row + r) * a.in + c;
      if (a.flag) v += load4(g, inside);
      store4(g, v, inside);
    }
    __syncthreads();
  }
}

// As many wavefronts as fill the chip, while each has a stretch of its own.
int waves_for(int64_t blocks, int stretches, int most) {
  int waves = 4;
  while (waves < most && blocks * waves < 2048 && waves < stretches) waves *= 2;
  return waves;
}
// Blocks for `passes` over a worker's rows at once, as far as that comes to `most` blocks: those that find no rows cost time too.
dim3 grid_of(int64_t x, int n, int passes = 1, int most = 1) {
  const int64_t fill = most / (x * n);
  return dim3(uint32_t(x), uint32_t(n < 32768 ? n : 32768), uint32_t(fill < 1 ? 1 : fill < passes ? fill : passes));
}

}  // namespace

template <bool Forward, class T, class TC>
int launch_linear_few(const LinearArgs &a, bool direct, bool small, void *stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  // passes side by side: all of one worker's, four times the average of several (who has more takes them one after the other)
  const int height = small ? 16 : 64, all = ceil_div_i64(a.rows, height), share = 4 * ceil_div_i64(ceil_div_i64(a.rows, a.n), height);
  const int passes = all < share ? all : share;
  if (Forward && small) {
    const int64_t x = ceil_div_i64(a.out, kOuts);
    const dim3 grid = grid_of(x, a.n, passes, 4096);
    linear_few_kernel<T, TC, 16><<<grid, 64 * waves_for(x * a.n * grid.z, ceil_div_i64(a.in, kStepBytes / int(sizeof(T))), 16), 0, st>>>(a);
    return hip_rc(hipGetLastError());
  }
  const dim3 grid = grid_of(ceil_div_i64(Forward ? a.out : a.in, kSharedCols), a.n, passes, 512);
  if (!small) linear_shared_kernel<Forward, T, TC, 4, 4, true><<<grid, 64 * 4, 0, st>>>(a);  // direct only
  else if constexpr (!Forward) {
    if (direct) linear_shared_kernel<Forward, T, TC, 1, 8, true><<<grid, 64 * 8, 0, st>>>(a);
    else linear_shared_kernel<Forward, T, TC, 1, 8, false><<<grid, 64 * 8, 0, st>>>(a);
  }
  return hip_rc(hipGetLastError());
}
template int launch_linear_few<true, float, float>(const LinearArgs &, bool, bool, void *);
template int launch_linear_few<true, bf16_t, float>(const LinearArgs &, bool, bool, void *);
template int launch_linear_few<true, bf16_t, bf16_t>(const LinearArgs &, bool, bool, void *);
template int launch_linear_few<false, float, float>(const LinearArgs &, bool, bool, void *);
template int launch_linear_few<false, bf16_t, bf16_t>(const LinearArgs &, bool, bool, void *);

template <class T>
int launch_linear_weight_split(const LinearArgs &a, void *stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const dim3 grid = grid_of(int64_t(ceil_div_i64(a.out, kSplitTile)) * ceil_div_i64(a.in, kSplitTile), a.n);
  linear_weight_split_kernel<T><<<grid, 64 * kSplitWaves, 0, st>>>(a);
  return hip_rc(hipGetLastError());
}
template int launch_linear_weight_split<float>(const LinearArgs &, void *);
template int launch_linear_weight_split<bf16_t>(const LinearArgs &, void *);

}  // namespace detag

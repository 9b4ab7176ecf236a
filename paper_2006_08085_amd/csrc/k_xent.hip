// Softmax cross-entropy of every worker's rows and its gradient with respect to the logits.
//
//   valid row r of worker i: 0 <= label < C;  c_i = number of worker i's valid rows
//   l_r  = log sum_c exp z_rc - z_r,label      loss_i = sum_r l_r / c_i   (0 where c_i = 0)
//   dz_r = (softmax(z_r) - e_label) / c_i      (0 for rows that are not valid, whatever their logits)
//
// What bounds it is memory: a row is read once and written once.  A row stays in the registers of the lanes that share it, as it
// was read; each lane takes the largest of its values and the sum of their exponentials relative to that, the pairs are joined
// once, and the exponentials are taken a second time for the store.  Sums and exponents are fp32; the gradient is rounded once.
//
// Three launches: rows' weights (1/c_i, 0, or -1 for a row that no worker owns), rows (more than 2^31 threads in several), the workers'
// losses; one launch where a row is a few pieces and rows are few.  All sums are taken in an order that depends on the sizes only.
// Measured: 8192 x 32000 bf16 190 to 206 us (1.05 GB, 5.1 to 5.5 TB/s), 1500 x 50001 fp32 134 us (4.5 TB/s), 32 workers of 128 rows, 10
// classes 5 us (one launch).
#include <algorithm>

#include "dev_common.hpp"
#include "detag_internal.h"

namespace detag {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

constexpr int kWeightThreads = 1024;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct XentArgs {
  const void *logits;
  void *grad;
  const int32_t *labels;
  const float *weight;  // per row
  float *row_loss;
  int64_t ldl, ldg;
  int rows, classes;
  int64_t first = 0;  // row of the launch's first block
};

__device__ __forceinline__ void worker_rows(const int32_t *offsets, int rows, int i, int &lo, int &hi) {
  lo = offsets[i], hi = offsets[i + 1];
  lo = lo < 0 ? 0 : lo > rows ? rows : lo;
  hi = hi < lo ? lo : hi > rows ? rows : hi;
}

template <int THREADS>
__device__ __forceinline__ int block_sum(int v, int *part) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) v += part[w];
  return v;
}

// f(r) for the worker's rows of this thread, four loads under way at a time.  Row numbers stay below 2^31, and as unsigned ones may
// go a block's stride further.
template <int THREADS, class F>
__device__ __forceinline__ void each_row(int lo, int hi, F &&f) {
  const uint32_t end = uint32_t(hi);
  uint32_t r = uint32_t(lo) + threadIdx.x;
  for (; r + 3 * THREADS < end; r += 4 * THREADS) f(r), f(r + THREADS), f(r + 2 * THREADS), f(r + 3 * THREADS);
  for (; r < end; r += THREADS) f(r);
}

// grid (n, slices): every block counts all of a worker's labels and writes the weights of its slice of the rows.  One worker with
// 16384 rows: 16 slices 3 us, one 30.
__global__ __launch_bounds__(kWeightThreads) void xent_weight_kernel(const int32_t *offsets, const int32_t *labels, int n, int rows,
                                                                     int classes, float *weight) {
  __shared__ int part[kWeightThreads / 64];
  const int i = blockIdx.x;
  int lo, hi;
  worker_rows(offsets, rows, i, lo, hi);
  int count = 0;
  each_row<kWeightThreads>(lo, hi, [&](uint32_t r) { count += uint32_t(labels[r]) < uint32_t(classes); });
  count = block_sum<kWeightThreads>(count, part);
  const float each = 1.f / float(count > 0 ? count : 1);
  const uint32_t step = kWeightThreads * gridDim.y;
  for (uint32_t r = uint32_t(lo) + threadIdx.x + kWeightThreads * blockIdx.y; r < uint32_t(hi); r += step) weight[r] = uint32_t(labels[r]) < uint32_t(classes) ? each : 0.f;
  if (i == 0 && blockIdx.y == 0)
    for (uint32_t r = threadIdx.x; r < uint32_t(lo); r += kWeightThreads) weight[r] = -1.f;
  if (i == n - 1 && blockIdx.y == 0)
    for (uint32_t r = uint32_t(hi) + threadIdx.x; r < uint32_t(rows); r += kWeightThreads) weight[r] = -1.f;
}

// The losses of a worker's rows that count, weighted, in the order of the rows' numbers modulo the block's width.  A thread adds a
// thousandth of the rows one after the other, and holds that sum in 64 bits: equal losses, as those of a model that knows nothing yet,
// are rounded the same way every time (2^24 rows: off by up to 2^-12 in 32 bits).
__global__ __launch_bounds__(kWeightThreads) void xent_loss_kernel(const int32_t *offsets, int rows, const float *weight,
                                                                   const float *row_loss, float *loss) {
  __shared__ float sums[kWeightThreads / 64], weights[kWeightThreads / 64];
  const int i = blockIdx.x;
  int lo, hi;
  worker_rows(offsets, rows, i, lo, hi);
  double own = 0.0;
  float each = 0.f;
  each_row<kWeightThreads>(lo, hi, [&](uint32_t r) {
    const float w = weight[r], l = row_loss[r];
    if (w > 0.f) own += double(l), each = w;
  });
  float sum = float(own);
#pragma unroll
  for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d), each = fmaxf(each, __shfl_xor(each, d));
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum, weights[threadIdx.x >> 6] = each;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWeightThreads / 64; ++w) sum += sums[w], each = fmaxf(each, weights[w]);
    loss[i] = sum * each;
  }
}

template <class T>
struct Piece {
  static constexpr int kElems = 16 / sizeof(T);
  u32x4 raw;
  __device__ __forceinline__ float operator[](int e) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(raw[e]);
    else return __uint_as_float(e % 2 ? raw[e / 2] & 0xffff0000u : raw[e / 2] << 16);
  }
  __device__ __forceinline__ void set(int e, float v) {
    if constexpr (sizeof(T) == 4) raw[e] = __float_as_uint(v);
    else raw[e / 2] = e % 2 ? (raw[e / 2] & 0xffffu) | uint32_t(bf16_bits_rne(v)) << 16 : (raw[e / 2] & 0xffff0000u) | bf16_bits_rne(v);
  }
  // `inside` elements from p on; the others as -inf
  template <bool Stream>
  __device__ __forceinline__ void load(const T *p, int inside) {
    if (inside >= kElems) {
      raw = Stream ? __builtin_nontemporal_load(reinterpret_cast<const u32x4_any *>(p)) : *reinterpret_cast<const u32x4_any *>(p);
    } else {
#pragma unroll
      for (int e = 0; e < kElems; ++e) set(e, e < inside ? to_f32(p[e]) : -INFINITY);
    }
  }
  template <bool Stream>
  __device__ __forceinline__ void store(T *p, int inside) const {
    if (inside >= kElems) {
      if constexpr (Stream) __builtin_nontemporal_store(raw, reinterpret_cast<u32x4_any *>(p));
      else *reinterpret_cast<u32x4_any *>(p) = raw;
    } else {
#pragma unroll
      for (int e = 0; e < kElems; ++e)
        if (e < inside) p[e] = from_f32<T>((*this)[e]);
    }
  }
};

// The larger of two, NaN if either is.
__device__ __forceinline__ float larger(float a, float b) { return a > b || a != a ? a : b; }

// (largest, sum of exp relative to it) of two sets as one.  Sets without a value above -inf count as empty, sum 0.
__device__ __forceinline__ void join(float &m, float &s, float m2, float s2) {
  const float top = larger(m, m2), ref = top == -INFINITY ? 0.f : top;
  s = s * __builtin_amdgcn_exp2f((m - ref) * kLog2e) + s2 * __builtin_amdgcn_exp2f((m2 - ref) * kLog2e);
  m = top;
}

// LANES lanes share a row (a part of a wavefront, or all of several).  PIECES > 0: a row is at most PIECES pieces of 16 bytes a
// lane, which are kept; 0: any width, read twice.
template <class T, int LANES, int PIECES, bool Stream>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void xent_rows_kernel(XentArgs a) {
  constexpr int kThreads = LANES < 256 ? 256 : LANES, kRowsPerBlock = kThreads / LANES, kElems = Piece<T>::kElems;
  __shared__ float parts[2][kThreads / 64];
  const int lane = threadIdx.x % LANES;
  const int64_t r = a.first + int64_t(blockIdx.x) * kRowsPerBlock + threadIdx.x / LANES;
  const bool exists = r < a.rows;
  const float weight = exists ? a.weight[r] : -1.f;
  const int label = exists ? a.labels[r] : -1;
  const T *z = static_cast<const T *>(a.logits) + r * a.ldl;
  T *g = static_cast<T *>(a.grad) + r * a.ldg;
  const bool valid = weight > 0.f;
  constexpr int kStride = LANES * kElems;
  Piece<T> held[PIECES ? PIECES : 1];
  float m = -INFINITY, s = 0.f;
  auto take = [&](const Piece<T> &p) {
    float top = p[0];
#pragma unroll
    for (int e = 1; e < kElems; ++e) top = larger(top, p[e]);
    const float ref0 = larger(m, top), ref = ref0 == -INFINITY ? 0.f : ref0;
    s *= __builtin_amdgcn_exp2f((m - ref) * kLog2e);
#pragma unroll
    for (int e = 0; e < kElems; ++e) s += __builtin_amdgcn_exp2f((p[e] - ref) * kLog2e);
    m = ref0;
  };
  float at_label = 0.f;
  if (valid) {
    at_label = to_f32(z[label]);
    if constexpr (PIECES > 0) {
#pragma unroll
      for (int k = 0; k < PIECES; ++k) {
        const int c = k * kStride + lane * kElems;
        held[k].template load<Stream>(z + c, a.classes - c);
      }
#pragma unroll
      for (int k = 0; k < PIECES; ++k) take(held[k]);
    } else {
      for (int64_t c = lane * kElems; c < a.classes; c += kStride) {
        held[0].template load<false>(z + c, a.classes - c);
        take(held[0]);
      }
    }
  }
#pragma unroll
  for (int d = 1; d < (LANES < 64 ? LANES : 64); d *= 2) join(m, s, __shfl_xor(m, d), __shfl_xor(s, d));
  if constexpr (LANES > 64) {
    if ((threadIdx.x & 63) == 0) parts[0][threadIdx.x >> 6] = m, parts[1][threadIdx.x >> 6] = s;
    __syncthreads();
    m = parts[0][0], s = parts[1][0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) join(m, s, parts[0][w], parts[1][w]);
  }
  if (weight < 0.f) return;
  if (valid && lane == 0 && a.row_loss) a.row_loss[r] = (m - at_label) + __builtin_amdgcn_logf(s) * kLn2;
  const float scale = valid ? weight / s : 0.f;
  auto finish = [&](Piece<T> &p, auto c) {
#pragma unroll
    for (int e = 0; e < kElems; ++e) {
      float v = 0.f;
      if (valid) v = __builtin_amdgcn_exp2f((p[e] - m) * kLog2e) * scale - (c + e == label ? weight : 0.f);
      p.set(e, v);
    }
    p.template store<Stream>(g + c, a.classes - c);
  };
  if constexpr (PIECES > 0) {
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
      const int c = k * kStride + lane * kElems;
      if (c < a.classes) finish(held[k], c);
    }
  } else {
    for (int64_t c = lane * kElems; c < a.classes; c += kStride) {
      if (valid) held[0].template load<false>(z + c, a.classes - c);
      finish(held[0], c);
    }
  }
}

// Everything in one launch, a block per worker, 16 lanes a row: what a few classes and few rows take is the launches (64 workers of 64 rows,
// 10 classes 4.6 us, in three launches 9.6).  A block takes a worker's rows a stretch at a time, and the host does not know whose they are.
// Even ones gain up to 256 rows a worker (16 workers of 256 7.0 us, 9.5, of 512 11.1, 9.4); one worker that holds all of them costs 16 us
// for every 1024 rows, whatever the average (4096 rows 67.5 us, 9.6, 8192 133, 11.1, 16384 263, 15.8).  So both are bounded, the second
// at seven times the three launches, and even calls of more rows go without (64 workers of 128 5.0 us, 9.6).
constexpr int kSmallAverage = 256, kSmallMost = 4096;  // rows of a worker, of a call
constexpr int kSmallThreads = 1024, kSmallLanes = 16, kSmallRows = kSmallThreads / kSmallLanes, kSmallAhead = 2;
template <class T>
__global__ __launch_bounds__(kSmallThreads) void xent_small_kernel(XentArgs a, const int32_t *offsets, float *loss) {
  constexpr int kElems = Piece<T>::kElems;
  __shared__ int counts[kSmallThreads / 64];
  __shared__ float losses[kSmallRows];
  const int i = blockIdx.x, lane = threadIdx.x % kSmallLanes, slot = threadIdx.x / kSmallLanes, c = lane * kElems;
  int lo, hi;
  worker_rows(offsets, a.rows, i, lo, hi);
  int count = 0;
  for (int r = lo + threadIdx.x; r < hi; r += kSmallThreads) count += uint32_t(a.labels[r]) < uint32_t(a.classes);
  Piece<T> held[kSmallAhead];
  int label[kSmallAhead];
  auto request = [&](int r0) {
#pragma unroll
    for (int u = 0; u < kSmallAhead; ++u) {
      const int64_t r = r0 + u * kSmallRows + slot;
      label[u] = -1;
      if (r < hi) label[u] = a.labels[r], held[u].template load<false>(static_cast<const T *>(a.logits) + r * a.ldl + c, a.classes - c);
    }
  };
  request(lo);
  count = block_sum<kSmallThreads>(count, counts);
  const float weight = 1.f / float(count > 0 ? count : 1);
  float sum = 0.f;
  for (int r0 = lo; r0 < hi; r0 += kSmallAhead * kSmallRows) {
#pragma unroll
    for (int u = 0; u < kSmallAhead; ++u) {
      const int64_t r = r0 + u * kSmallRows + slot;
      const bool valid = r < hi && uint32_t(label[u]) < uint32_t(a.classes);
      Piece<T> &p = held[u];
      float m = p[0], s = 0.f, z = 0.f;
#pragma unroll
      for (int e = 1; e < kElems; ++e) m = larger(m, p[e]);
#pragma unroll
      for (int d = 1; d < kSmallLanes; d *= 2) m = larger(m, __shfl_xor(m, d));
      const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int e = 0; e < kElems; ++e) {
        s += __builtin_amdgcn_exp2f((p[e] - ref) * kLog2e);
        if (c + e == label[u]) z = p[e];
      }
#pragma unroll
      for (int d = 1; d < kSmallLanes; d *= 2) s += __shfl_xor(s, d);
      if (valid && uint32_t(label[u] - c) < uint32_t(kElems)) sum += (m - z) + __builtin_amdgcn_logf(s) * kLn2;  // the label's lane
      const float scale = weight / s;
#pragma unroll
      for (int e = 0; e < kElems; ++e) {
        const float v = __builtin_amdgcn_exp2f((p[e] - m) * kLog2e) * scale - (c + e == label[u] ? weight : 0.f);
        p.set(e, valid ? v : 0.f);
      }
      if (r < hi && c < a.classes) p.template store<false>(static_cast<T *>(a.grad) + r * a.ldg + c, a.classes - c);
    }
    if (r0 + kSmallAhead * kSmallRows < hi) request(r0 + kSmallAhead * kSmallRows);
  }
  if (!loss) return;
#pragma unroll
  for (int d = 1; d < kSmallLanes; d *= 2) sum += __shfl_xor(sum, d);
  if (lane == 0) losses[slot] = sum;
  __syncthreads();
  if (threadIdx.x < 64) {
    sum = losses[threadIdx.x];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    if (threadIdx.x == 0) loss[i] = sum * weight;
  }
}

template <class T, int LANES, int PIECES>
int launch_rows(XentArgs a, void *stream) {
  constexpr int kThreads = LANES < 256 ? 256 : LANES;
  constexpr int64_t kPiece = kThreadsPerLaunch / LANES;    // rows
  constexpr bool kMayStream = LANES < 1024 || PIECES != 4;  // that form is for at most 512 rows of 64 KiB
  const hipStream_t st = static_cast<hipStream_t>(stream);
  // what the memory-side cache cannot hold anyway streams past it: 8192 x 32000 bf16 202 us (216), 500 x 131072 fp32 117 (155), but
  // 4096 x 5000 fp32 36 (34)
  const bool streams = kMayStream && 2 * int64_t(a.rows) * a.classes * int64_t(sizeof(T)) >= int64_t(256) << 20;
  for (; a.first < a.rows; a.first += kPiece) {
    const dim3 grid(uint32_t(ceil_div_i64(std::min(a.rows - a.first, kPiece), kThreads / LANES)));
    if (streams) xent_rows_kernel<T, LANES, PIECES, kMayStream><<<grid, kThreads, 0, st>>>(a);
    else xent_rows_kernel<T, LANES, PIECES, false><<<grid, kThreads, 0, st>>>(a);
    if (int rc = hip_rc(hipGetLastError())) return rc;
  }
  return 0;
}

// As few lanes as hold a row in 16 pieces each: several blocks share a compute unit, so that one reads while another writes.  Where
// there are fewer rows than that takes, more lanes a row: 100 rows of 32000 bf16 14.6 us (19.0).
template <class T>
int launch_rows(const XentArgs &a, void *stream) {
  const int pieces = ceil_div_i64(a.classes, Piece<T>::kElems);
  if (a.rows <= 512) {
    if (pieces > 256 && pieces <= 1024) return launch_rows<T, 256, 4>(a, stream);
    if (pieces > 1024 && pieces <= 4096) return launch_rows<T, 1024, 4>(a, stream);
  }
  if (pieces <= 16) return launch_rows<T, 16, 1>(a, stream);
  if (pieces <= 64) return launch_rows<T, 64, 1>(a, stream);
  if (pieces <= 128) return launch_rows<T, 64, 2>(a, stream);
  if (pieces <= 256) return launch_rows<T, 64, 4>(a, stream);
  if (pieces <= 512) return launch_rows<T, 256, 2>(a, stream);
  if (pieces <= 1024) return launch_rows<T, 256, 4>(a, stream);
  if (pieces <= 2048) return launch_rows<T, 256, 8>(a, stream);
  if (pieces <= 4096) return launch_rows<T, 256, 16>(a, stream);
  if (pieces <= 8192) return launch_rows<T, 512, 16>(a, stream);
  if (pieces <= 16384) return launch_rows<T, 1024, 16>(a, stream);
  return launch_rows<T, 1024, 0>(a, stream);
}

}  // namespace

int64_t xent_scratch_floats(int rows) { return 2 * int64_t(rows); }

int launch_cross_entropy(int n, const void *logits, int64_t ldl, bool bf16, const int32_t *labels, const int32_t *rows, int M, int C,
                         void *grad, int64_t ldg, float *scratch, float *loss, void *stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  XentArgs a{logits, grad, labels, scratch, scratch + M, ldl, ldg, M, C};
  if (C <= kSmallLanes * (bf16 ? 8 : 4) && M <= kSmallMost && M <= kSmallAverage * int64_t(n)) {
    if (bf16) xent_small_kernel<bf16_t><<<dim3(uint32_t(n)), kSmallThreads, 0, st>>>(a, rows, loss);
    else xent_small_kernel<float><<<dim3(uint32_t(n)), kSmallThreads, 0, st>>>(a, rows, loss);
    return hip_rc(hipGetLastError());
  }
  const int slices = M < kWeightThreads ? 1 : M < 16 * kWeightThreads ? M / kWeightThreads : 16;
  xent_weight_kernel<<<dim3(uint32_t(n), uint32_t(slices)), kWeightThreads, 0, st>>>(rows, labels, n, M, C, scratch);
  if (int rc = hip_rc(hipGetLastError())) return rc;
  if (M > 0)
    if (int rc = bf16 ? launch_rows<bf16_t>(a, stream) : launch_rows<float>(a, stream)) return rc;
  if (!loss) return 0;
  xent_loss_kernel<<<dim3(uint32_t(n)), kWeightThreads, 0, st>>>(rows, M, scratch, scratch + M, loss);
  return hip_rc(hipGetLastError());
}

}  // namespace detag

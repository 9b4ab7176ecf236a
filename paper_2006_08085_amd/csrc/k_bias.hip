// The gradient of a layer's epilogue: dZ = dY act'(Z), and the bias's, the sum of dZ over every worker's rows.
//
// What bounds it is memory: dY and Z are read once, dZ is written once.  A block takes a strip of columns of a run of one worker's rows;
// a lane has the same eight (fp32: four) columns in all of them, keeps their sums in fp32, and writes them to scratch once.  A second
// launch adds up a worker's runs, in their order, into its row of G: the result depends on the sizes only.  What is summed is dZ before
// it is rounded.  8192 rows of 1024 bf16 of 16 uneven workers, no activation: 5.8 us (17 MB) and 6.0 for the runs.
#include "act_dev.hpp"
#include "dev_common.hpp"
#include "detag_internal.h"
#include "rows_common.hpp"

namespace detag {
namespace {

struct BiasArgs {
  const void *dy, *z;
  void *dz;  // null: no activation, dY is dZ
  float *parts;
  const int32_t *offsets;
  int64_t ldy, ldz, ldd;
  int n, rows, columns, high, act;
};

constexpr int kThreads = 256, kRowsAhead = 4;

// grid (strips, runs)
template <class T, bool Act>
__global__ __launch_bounds__(kThreads) void bias_grad_kernel(BiasArgs a) {
  constexpr int kElems = 16 / sizeof(T);
  const int number = blockIdx.y + gridDim.y * blockIdx.z;
  const Run run = run_of(a.offsets, a.n, a.rows, a.high, number);
  if (run.part < 0) return;
  const int last = run.hi - run.first < a.high ? run.hi : run.first + a.high;
  const int64_t c = (int64_t(blockIdx.x) * kThreads + threadIdx.x) * kElems;
  if (c >= a.columns) return;
  const int inside = a.columns - int(c);
  float sum[kElems];
#pragma unroll
  for (int e = 0; e < kElems; ++e) sum[e] = 0.f;
  for (int64_t r0 = run.first; r0 < last; r0 += kRowsAhead) {
    u32x4 dy[kRowsAhead], z[Act ? kRowsAhead : 1];
#pragma unroll
    for (int k = 0; k < kRowsAhead; ++k) {
      const int here = r0 + k < last ? inside : 0;
      dy[k] = load_piece(static_cast<const T *>(a.dy) + (r0 + k) * a.ldy + c, here);
      if constexpr (Act) z[k] = load_piece(static_cast<const T *>(a.z) + (r0 + k) * a.ldz + c, here);
    }
#pragma unroll
    for (int k = 0; k < kRowsAhead; ++k) {
      if (r0 + k >= last) break;
      float v[kElems];
#pragma unroll
      for (int e = 0; e < kElems; ++e) {
        v[e] = element<T>(dy[k], e);
        if constexpr (Act) v[e] *= act_slope<T>(element<T>(z[k], e), a.act);
        sum[e] += v[e];
      }
      if constexpr (Act) store_piece(static_cast<T *>(a.dz) + (r0 + k) * a.ldd + c, v, inside);
    }
  }
  float *const part = a.parts + int64_t(number) * a.columns + c;
#pragma unroll
  for (int e = 0; e < kElems; e += 4) {
    const float four[4] = {sum[e], sum[e + 1], sum[e + 2], sum[e + 3]};
    store_piece(part + e, four, inside - e);
  }
}

struct JoinArgs {
  const float *parts;
  const int32_t *offsets;
  float *g;
  int64_t ld, first, second;  // columns of G; second < 0: one vector
  int n, rows, columns, high, accumulate;
};

// grid (ceil(columns / 64), vectors, n): a block's GROUPS wavefronts take the runs of a worker in turn, 64 columns of them.
template <int GROUPS>
__global__ __launch_bounds__(64 * GROUPS) void join_runs_kernel(JoinArgs a) {
  __shared__ float parts[GROUPS][64];
  const int group = threadIdx.x >> 6, lane = threadIdx.x & 63, vectors = gridDim.y;
  const int64_t c = int64_t(blockIdx.x) * 64 + lane;
  for (int i = blockIdx.z; i < a.n; i += gridDim.z) {
    const int lo = within(a.offsets[i], a.rows), hi = within(a.offsets[i + 1], a.rows);
    const int runs = hi > lo ? (hi - lo - 1) / a.high + 1 : 0;
    const float *p = a.parts + ((int64_t(lo / a.high) + i) * vectors + blockIdx.y) * a.columns + c;
    float sum = 0.f;
    if (c < a.columns)
#pragma unroll 8
      for (int k = group; k < runs; k += GROUPS) sum += p[int64_t(k) * vectors * a.columns];
    __syncthreads();
    parts[group][lane] = sum;
    __syncthreads();
    if (group == 0 && c < a.columns) {
#pragma unroll
      for (int w = 1; w < GROUPS; ++w) sum += parts[w][lane];
      float *g = a.g + i * a.ld + (blockIdx.y ? a.second : a.first) + c;
      *g = a.accumulate ? *g + sum : sum;
    }
  }
}

}  // namespace

// As many runs as there are compute units for four blocks each, which layer norm's gradient fits (16384 x 4096 bf16: 960 runs 120 us, 1024, whose last
// ones start when the first are done, 135); its 8 to 16 bytes of scratch a column and run (written and read) stay little beside the rows'.
// The bias's gradient takes the same runs; joining 910 of them takes as long as its own pass (8192 rows of 1024, 6.0 and 5.8 us).  Of few rows a run has fewer than eight, for what counts then is how long a block takes over its rows.
constexpr int kRuns = 960, kFewRuns = 512;
int layer_run_rows(int rows) {
  if (rows > 8 * kRuns) return ceil_div_i64(rows, kRuns);
  return rows >= 8 * kFewRuns ? 8 : rows > kFewRuns ? ceil_div_i64(rows, kFewRuns) : 1;
}
int64_t layer_gradient_floats(int n, int rows, int columns) { return part_runs(rows, n, layer_run_rows(rows)) * 2 * columns; }
int64_t layer_gradient_floats_upto(int n, int rows, int columns) { return (int64_t(rows < kRuns ? rows : kRuns) + n + 1) * 2 * columns; }

int launch_join_runs(const Shape &s, const float *parts, const int32_t *rows, int M, int columns, float *G, int64_t first, int64_t second,
                     bool accumulate, void *stream) {
  const JoinArgs a{parts, rows, G, s.ld, first, second, s.n, M, columns, layer_run_rows(M), accumulate};
  const dim3 grid(uint32_t(ceil_div_i64(columns, 64)), second < 0 ? 1 : 2, uint32_t(s.n < 32768 ? s.n : 32768));
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (M / a.high > 128 * s.n) join_runs_kernel<16><<<grid, 64 * 16, 0, st>>>(a);
  else join_runs_kernel<4><<<grid, 64 * 4, 0, st>>>(a);
  return hip_rc(hipGetLastError());
}

int launch_bias_grad(const Shape &s, bool bf16, const void *dY, int64_t ldy, int act, const void *Z, int64_t ldz, const int32_t *rows, int M, int columns,
                     void *dZ, int64_t ldd, float *G, int64_t offset, bool accumulate, float *scratch, void *stream) {
  const BiasArgs a{dY, Z, dZ, scratch, rows, ldy, ldz, ldd, s.n, M, columns, layer_run_rows(M), act};
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (M > 0) {
    const int64_t runs = part_runs(M, s.n, a.high);
    const int64_t y = runs < 32768 ? runs : 32768;
    const dim3 grid(uint32_t(ceil_div_i64(columns, kThreads * (bf16 ? 8 : 4))), uint32_t(y), uint32_t(ceil_div_i64(runs, y)));
    if (bf16 && dZ) bias_grad_kernel<bf16_t, true><<<grid, kThreads, 0, st>>>(a);
    else if (bf16) bias_grad_kernel<bf16_t, false><<<grid, kThreads, 0, st>>>(a);
    else if (dZ) bias_grad_kernel<float, true><<<grid, kThreads, 0, st>>>(a);
    else bias_grad_kernel<float, false><<<grid, kThreads, 0, st>>>(a);
    if (const int rc = hip_rc(hipGetLastError())) return rc;
  }
  return launch_join_runs(s, scratch, rows, M, columns, G, offset, -1, accumulate, stream);
}

}  // namespace detag

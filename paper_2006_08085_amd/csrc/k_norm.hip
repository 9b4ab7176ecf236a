// Layer norm of every worker's rows, each worker with its own gain and bias, and its gradient.
//
//   mu = mean x,  s = 1 / sqrt(mean (x - mu)^2 + eps),  xhat = (x - mu) s
//   forward    y = xhat g + b
//   gradient   h = dy g;  dx = s (h - mean h - xhat mean(h xhat)) [+ add];  dg = sum over the worker's rows of dy xhat;  db = sum dy
//
// What bounds both is memory: every row is read once and written once.  A row stays, as it was read, in the registers of the lanes that
// share it (a wavefront, or four or eight of them), so that the mean is known before the squares are summed: no difference of large
// numbers.  The gradient takes four sums of a row in two rounds: x and h, then (x - mu)^2 and h (x - mu).  Nothing of the forward pass has
// to be kept for it: mu and s cost a sum each over values that are in registers anyway.
//
// The gradients of gain and bias: a block takes a run of one worker's rows, its lanes keep the sums of their columns in fp32 registers over
// the run, and write them to scratch once; a second launch adds up the runs of a worker in their order.  The result depends on the
// sizes only.  All statistics and sums are fp32; results are rounded once, at their store.
//
// Measured, back to back: 16384 rows of 4096 bf16 forward 51 us (268 MB, 5.2 TB/s, what a copy reaches), gradient with `add` 128 (540 MB, 118 for
// the rows, 4.6 TB/s, and 8 for the runs: 960 of them leave 30 MB of sums); eight rows of 1024 forward 4.1, a launch.
#include "dev_common.hpp"
#include "detag_internal.h"
#include "rows_common.hpp"

namespace detag {
namespace {

struct NormArgs {
  const void *gain, *bias;  // at their first columns of the n x ld matrix; bias may be null
  const void *x, *dy, *add;  // add may be null
  void *out;
  float *parts;  // gradient: runs x (1 or 2) x columns
  const int32_t *offsets;
  int64_t ld, ldx, ldy, lda, ldo;
  int n, rows, columns, high;  // high: rows of a run
  float eps;
};

// The WAVES wavefronts that share a row; a block holds kTeams of them.
template <int WAVES>
struct Team {
  static constexpr int kLanes = 64 * WAVES, kThreads = kLanes < 256 ? 256 : kLanes, kTeams = kThreads / kLanes;

  // Two sums over a team, in every lane.  `scratch` alternates between two arrays, so that one barrier a round is enough.
  __device__ static __forceinline__ void sum(float &a, float &b, float (*scratch)[2]) {
    a = wave_sum(a), b = wave_sum(b);
    if constexpr (WAVES > 1) {
      if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6][0] = a, scratch[threadIdx.x >> 6][1] = b;
      __syncthreads();
      a = scratch[0][0], b = scratch[0][1];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) a += scratch[w][0], b += scratch[w][1];
    }
  }
};

template <class T, int WAVES, int PIECES>
__global__ __launch_bounds__(Team<WAVES>::kThreads) void norm_kernel(NormArgs a) {
  using Group = Team<WAVES>;
  constexpr int kElems = 16 / sizeof(T);
  __shared__ float scratch[2][WAVES][2];
  const int team = __builtin_amdgcn_readfirstlane(threadIdx.x / Group::kLanes), t = threadIdx.x % Group::kLanes;
  const float columns = float(a.columns);
  for (int64_t r = int64_t(blockIdx.x) * Group::kTeams + team; r < a.rows; r += int64_t(gridDim.x) * Group::kTeams) {
    const T *row = static_cast<const T *>(a.x) + r * a.ldx;
    u32x4 x[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int c = (i * Group::kLanes + t) * kElems;
      x[i] = load_piece(row + c, a.columns - c);
    }
    const Run own = run_of(a.offsets, a.n, a.rows, 0, int(r));
    if (own.part < 0) continue;  // alike in all wavefronts of the team
    float sum = 0.f, none = 0.f;
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
#pragma unroll
      for (int e = 0; e < kElems; ++e) sum += element<T>(x[i], e);
    Group::sum(sum, none, scratch[0]);
    const float mean = sum / columns;
    float squares = 0.f;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int inside = a.columns - (i * Group::kLanes + t) * kElems;
#pragma unroll
      for (int e = 0; e < kElems; ++e) {
        const float d = e < inside ? element<T>(x[i], e) - mean : 0.f;
        squares += d * d;
      }
    }
    Group::sum(squares, none, scratch[1]);
    const float s = 1.f / sqrtf(squares / columns + a.eps);
    const T *gain = static_cast<const T *>(a.gain) + own.part * a.ld, *bias = static_cast<const T *>(a.bias) + own.part * a.ld;
    T *y = static_cast<T *>(a.out) + r * a.ldo;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int c = (i * Group::kLanes + t) * kElems, inside = a.columns - c;
      if (inside <= 0) break;
      const u32x4 g = load_piece(gain + c, inside), b = a.bias ? load_piece(bias + c, inside) : u32x4{0, 0, 0, 0};
      float v[kElems];
#pragma unroll
      for (int e = 0; e < kElems; ++e) v[e] = (element<T>(x[i], e) - mean) * s * element<T>(g, e) + element<T>(b, e);
      store_piece(y + c, v, inside);
    }
  }
}

template <class T, int WAVES, int PIECES, bool Bias>
__global__ __launch_bounds__(Team<WAVES>::kThreads, WAVES < 8 && PIECES * (16 / int(sizeof(T))) <= 16 ? 4 : 2) void norm_grad_kernel(NormArgs a) {
  using Group = Team<WAVES>;
  constexpr int kElems = 16 / sizeof(T), kVectors = Bias ? 2 : 1;
  __shared__ float scratch[2][WAVES][2];
  __shared__ float joined[WAVES == 1 ? (Group::kTeams - 1) * PIECES * 64 * kElems : 1];
  const int team = __builtin_amdgcn_readfirstlane(threadIdx.x / Group::kLanes), t = threadIdx.x % Group::kLanes;
  const float columns = float(a.columns);
  const Run run = run_of(a.offsets, a.n, a.rows, a.high, blockIdx.x);
  if (run.part < 0) return;
  const int last = run.hi - run.first < a.high ? run.hi : run.first + a.high;
  const T *gain = static_cast<const T *>(a.gain) + run.part * a.ld;
  u32x4 g[PIECES];
  float sums[kVectors][PIECES][kElems];  // of the gain's gradient and of the bias's
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const int c = (i * Group::kLanes + t) * kElems;
    g[i] = load_piece(gain + c, a.columns - c);
#pragma unroll
    for (int e = 0; e < kElems; ++e) {
#pragma unroll
      for (int v = 0; v < kVectors; ++v) sums[v][i][e] = 0.f;
    }
  }
  for (int64_t r = run.first + team; r < last; r += Group::kTeams) {
    const T *xr = static_cast<const T *>(a.x) + r * a.ldx, *yr = static_cast<const T *>(a.dy) + r * a.ldy;
    u32x4 x[PIECES], dy[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int c = (i * Group::kLanes + t) * kElems;
      x[i] = load_piece(xr + c, a.columns - c), dy[i] = load_piece(yr + c, a.columns - c);
    }
    float sum = 0.f, hs = 0.f;
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
#pragma unroll
      for (int e = 0; e < kElems; ++e) sum += element<T>(x[i], e), hs += element<T>(dy[i], e) * element<T>(g[i], e);
    Group::sum(sum, hs, scratch[0]);
    const float mean = sum / columns;
    float squares = 0.f, hx = 0.f;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int inside = a.columns - (i * Group::kLanes + t) * kElems;
#pragma unroll
      for (int e = 0; e < kElems; ++e) {
        const float d = e < inside ? element<T>(x[i], e) - mean : 0.f;
        squares += d * d, hx += element<T>(dy[i], e) * element<T>(g[i], e) * d;
      }
    }
    Group::sum(squares, hx, scratch[1]);
    const float s = 1.f / sqrtf(squares / columns + a.eps), level = hs / columns, slope = hx / columns * s * s;
    T *out = static_cast<T *>(a.out) + r * a.ldo;
    const T *add = static_cast<const T *>(a.add) + r * a.lda;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int c = (i * Group::kLanes + t) * kElems, inside = a.columns - c;
      if (inside <= 0) break;
      const u32x4 more = a.add ? load_piece(add + c, inside) : u32x4{0, 0, 0, 0};
      float v[kElems];
#pragma unroll
      for (int e = 0; e < kElems; ++e) {
        const float dye = element<T>(dy[i], e), d = element<T>(x[i], e) - mean;
        sums[0][i][e] += dye * (d * s);
        if constexpr (Bias) sums[1][i][e] += dye;
        v[e] = s * (dye * element<T>(g[i], e) - level - d * slope) + element<T>(more, e);
      }
      store_piece(out + c, v, inside);
    }
  }
  float *const part = a.parts + int64_t(blockIdx.x) * kVectors * a.columns;
#pragma unroll
  for (int v = 0; v < kVectors; ++v) {
    auto &mine = sums[v];
    if constexpr (WAVES == 1) {  // the teams' rows, added up in their order
      __syncthreads();
      if (team > 0)
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
#pragma unroll
          for (int e = 0; e < kElems; ++e) joined[(((team - 1) * PIECES + i) * kElems + e) * 64 + t] = mine[i][e];
      __syncthreads();
      if (team > 0) continue;
#pragma unroll
      for (int w = 1; w < Group::kTeams; ++w)
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
#pragma unroll
          for (int e = 0; e < kElems; ++e) mine[i][e] += joined[(((w - 1) * PIECES + i) * kElems + e) * 64 + t];
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int c = (i * Group::kLanes + t) * kElems;
#pragma unroll
      for (int e = 0; e < kElems; e += 4) {
        const float four[4] = {mine[i][e], mine[i][e + 1], mine[i][e + 2], mine[i][e + 3]};
        store_piece(part + int64_t(v) * a.columns + c + e, four, a.columns - c - e);
      }
    }
  }
}

// f(WAVES, PIECES) as constants, for rows of that many pieces.
template <class T, class F>
int with_team(int pieces, F &&f) {
  using std::integral_constant;
  if (pieces <= 64) return f(integral_constant<int, 1>{}, integral_constant<int, 1>{});
  if (pieces <= 128) return f(integral_constant<int, 1>{}, integral_constant<int, 2>{});
  if (pieces <= 256) return f(integral_constant<int, 1>{}, integral_constant<int, 4>{});
  if (pieces <= 512) return f(integral_constant<int, 4>{}, integral_constant<int, 2>{});
  if (pieces <= 1024) return f(integral_constant<int, 4>{}, integral_constant<int, 4>{});
  if (pieces <= 2048) return f(integral_constant<int, 8>{}, integral_constant<int, 4>{});
  // the longest rows in fp32
  if constexpr (sizeof(T) == 4) return f(integral_constant<int, 8>{}, integral_constant<int, 8>{});
  else return int(hipErrorInvalidValue);
}
static_assert(kNormColumns <= 8 * 8 * 64 * 4, "the longest rows fit a team of eight wavefronts, in fp32 too");

template <class T>
int norm(const NormArgs &a, hipStream_t st) {
  return with_team<T>(ceil_div_i64(a.columns, 16 / sizeof(T)), [&](auto waves, auto pieces) {
    using Group = Team<decltype(waves)::value>;
    int64_t blocks = ceil_div_i64(a.rows, Group::kTeams);
    if (blocks > 1 << 20) blocks = 1 << 20;
    norm_kernel<T, decltype(waves)::value, decltype(pieces)::value><<<dim3(uint32_t(blocks)), Group::kThreads, 0, st>>>(a);
    return hip_rc(hipGetLastError());
  });
}

template <class T>
int norm_grad(const NormArgs &a, hipStream_t st) {
  return with_team<T>(ceil_div_i64(a.columns, 16 / sizeof(T)), [&](auto waves, auto pieces) {
    constexpr int W = decltype(waves)::value, P = decltype(pieces)::value;
    const dim3 grid(uint32_t(part_runs(a.rows, a.n, a.high)));
    if (a.bias) norm_grad_kernel<T, W, P, true><<<grid, Team<W>::kThreads, 0, st>>>(a);
    else norm_grad_kernel<T, W, P, false><<<grid, Team<W>::kThreads, 0, st>>>(a);
    return hip_rc(hipGetLastError());
  });
}

}  // namespace

int launch_norm(const Shape &s, const void *P, int64_t gain, int64_t bias, bool bf16, const void *X, int64_t ldx, const int32_t *rows, int M,
                int columns, float eps, void *Y, int64_t ldy, void *stream) {
  const size_t e = bf16 ? 2 : 4;
  const char *p = static_cast<const char *>(P);
  NormArgs a{};
  a.gain = p + gain * e, a.bias = bias < 0 ? nullptr : p + bias * e, a.x = X, a.out = Y, a.offsets = rows, a.ld = s.ld, a.ldx = ldx, a.ldo = ldy;
  a.n = s.n, a.rows = M, a.columns = columns, a.eps = eps;
  return bf16 ? norm<bf16_t>(a, static_cast<hipStream_t>(stream)) : norm<float>(a, static_cast<hipStream_t>(stream));
}

int launch_norm_grad(const Shape &s, const void *P, int64_t gain, int64_t bias, bool bf16, const void *X, int64_t ldx, const void *dY, int64_t ldy,
                     const int32_t *rows, int M, int columns, float eps, const void *add, int64_t lda, void *dX, int64_t ldd, float *G,
                     bool accumulate, float *scratch, void *stream) {
  const size_t e = bf16 ? 2 : 4;
  const char *p = static_cast<const char *>(P);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  NormArgs a{};
  a.gain = p + gain * e, a.bias = bias < 0 ? nullptr : p + bias * e, a.x = X, a.dy = dY, a.add = add, a.out = dX, a.parts = scratch, a.offsets = rows;
  a.ld = s.ld, a.ldx = ldx, a.ldy = ldy, a.lda = lda, a.ldo = ldd, a.n = s.n, a.rows = M, a.columns = columns, a.high = layer_run_rows(M), a.eps = eps;
  if (M > 0)
    if (const int rc = bf16 ? norm_grad<bf16_t>(a, st) : norm_grad<float>(a, st)) return rc;
  return launch_join_runs(s, scratch, rows, M, columns, G, gain, bias, accumulate, stream);
}

}  // namespace detag

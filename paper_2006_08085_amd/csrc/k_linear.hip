// Products of a layer for all workers at once, every worker with its own weights and its own number of rows.
//
// Worker i holds rows o_i .. o_{i+1}-1 of the row matrices A (inputs) and dY, and the weights W_i (out x in) as a slice of row i of
// an n x ld matrix:
//
//   forward       Y[r,:]  = act(A[r,:] W_i^T)                    contracts the in inputs
//   grad input    dA[r,:] = (dY[r,:] W_i) * [H[r,:] > 0]         contracts the out outputs
//   grad weight   G_i     (+)= sum_r dY[r,:]^T A[r,:]            contracts the worker's rows
//
// One launch serves all workers; the offsets o are read on the GPU, so that a program may make them there.  With bf16 operands the
// products run on v_mfma_f32_16x16x32_bf16, with fp32 operands on v_mfma_f32_16x16x4_f32; sums are fp32, and a result of a
// narrower type is rounded once, at its store.
//
// A block computes a tile of BM x BN results: the contraction is walked in steps of 128 bytes (64 bf16 or 32 fp32), whose tiles of
// both operands lie in LDS, two steps at a time.  An operand comes in one of two layouts, after how it lies in memory:
//
//   kAlong   the contracted index is contiguous (A and W of the forward product, dY of the input gradient): LDS rows of 128 bytes,
//            one per row of the tile; a lane's 16 bytes of a fragment are one read.
//   kAcross  the other index is contiguous (W of the input gradient, both operands of the weight gradient): LDS rows of one
//            contracted index each.  bf16 fragments are read with the transposing LDS read, fp32 ones value by value.
//
// 16-byte pieces of an LDS row lie at a position xor-ed with bits of the row's number, so that the lanes of a read spread over the
// banks.  Where rows start on whole dwords tiles go from memory to LDS without passing registers; the hardware's range check of the
// buffer loads zeroes what lies past a worker's rows, and what a last piece holds past the end of the contraction is zeroed in LDS.
// Otherwise (bf16 rows of odd length or at an odd address) tiles pass registers: 16 workers, 8192 rows, 1001 -> 4003 take 209, 214 and
// 276 us (forward, input gradient, weight gradient), 1024 -> 4096 92, 91 and 111.
//
// What bounds it: the matrix cores, as far as they are fed.  1 worker, 8192 rows, 4096 -> 4096 bf16: 200, 220 and 200 us, 1250 to 1380
// TFLOP/s of the 1400 to 1580 that a large library product reaches on this card; 8 uneven workers, 16384 rows, 4096 -> 8192: 914, 1072
// and 1014 us (1000 to 1200); fp32, 1 worker, 8192 rows, 4096 -> 4096: 2134 us, 129 of 132 to 154.  The rest is a tile's start and end,
// about 11 us for each 256 x 256 tile that a compute unit takes, 4 of them the stores: one block fills a unit's LDS, and nothing else
// runs there meanwhile.  Where workers have few rows, the weights (or the weight gradient) bound it: 16 workers of 16 rows,
// 2048 -> 2048, 134 MB of weights in 21 us (from the memory-side cache), 268 MB of gradient in 66 us.
//
// MFMA operand layout (lane l, p = l % 16, q = l / 16): 16x16x32 bf16 operands hold index p, k = 8q..8q+7; the four 16x16x4 fp32
// products of a piece hold index p, k = 4q+t for product t; the result's register r is (index 4q+r of the first, p of the second).
// The columns of the result are the first operand, so that a lane holds neighbours of a row.
#include "dev_common.hpp"
#include "detag_internal.h"
#include "linear_common.hpp"

namespace detag {
namespace {

enum Product : int { kForward, kGradInput, kGradWeight };

constexpr int kStages = 2;      // steps in LDS
constexpr int kXcds = 8;
constexpr int kUnits = 256;     // compute units
constexpr int kChooseRounds = 4;  // tiles for each up to which the height of 256-row tiles is chosen
constexpr int kGroup = 8;       // row tiles that are walked together, column by column

// Sums over the lanes up to each.
__device__ __forceinline__ int lane_scan(int v) {
#define DETAG_ADD_LANES(control, rows) v += __builtin_amdgcn_update_dpp(0, v, control, rows, 0xf, false)
  DETAG_ADD_LANES(0x111, 0xf);  // the lane 1, 2, 4, 8 below, in rows of 16
  DETAG_ADD_LANES(0x112, 0xf);
  DETAG_ADD_LANES(0x114, 0xf);
  DETAG_ADD_LANES(0x118, 0xf);
  DETAG_ADD_LANES(0x142, 0xa);  // the last of the row before, into every second row
  DETAG_ADD_LANES(0x143, 0xc);  // the last of the lower half
#undef DETAG_ADD_LANES
  return v;
}

// Row tiles, counted worker by worker: which worker a number belongs to, and how many there are in all.  Every wavefront looks for
// itself: 64 workers at a time, a scan over the lanes; the first 64 are kept.  Tiles are BM rows high.  Choose: or fewer,
// where the compute units, which take a tile each at a time, are done sooner with that; the workers' rows are known here only.  Microseconds
// (chosen, always 256): input gradient of 8192 rows, 4096 -> 1024, 16 even workers 76, 98 and uneven ones 91, 98; 4 workers of 1024 rows,
// 2048 -> 2048 forward 40, 49, input gradient 47, 58; 8 uneven workers, 8192 rows 92, 99 and 104, 120.
struct RowTile {
  int worker, first, count;  // first row, rows of the tile (0: no such tile)
};
template <int BM, bool Choose>
struct RowTiles {
  int lo = 0, hi = 0, upto = 0, total = 0, high = BM;

  __device__ __forceinline__ static int tiles_in(int rows, int high) {
    if constexpr (Choose) return high == BM ? (rows + BM - 1) / BM : high == BM / 2 ? (rows + BM / 2 - 1) / (BM / 2) : (rows + BM / 4 * 3 - 1) / (BM / 4 * 3);
    else return (rows + BM - 1) / BM;
  }
  __device__ __forceinline__ static void load(const LinearArgs &a, int base, int &lo, int &hi) {
    const int at = base + int(threadIdx.x & 63);
    lo = hi = 0;
    if (at < a.n) worker_rows(a, at, lo, hi);
  }
  __device__ __forceinline__ int count(const LinearArgs &a, int high) const {
    int sum = tiles_in(hi - lo, high);
    for (int base = 64; base < a.n; base += 64) {
      int l, h;
      load(a, base, l, h);
      sum += tiles_in(h - l, high);
    }
    return __builtin_amdgcn_readlane(lane_scan(sum), 63);
  }
  __device__ __forceinline__ RowTiles(const LinearArgs &a, int col_tiles) {
    load(a, 0, lo, hi);
    if constexpr (Choose) {
      // a tile of three quarters takes about 0.87 of a whole one's time, of half 0.73
      auto rounds = [&](int tiles) { return (tiles * col_tiles + kUnits - 1) / kUnits; };
      total = count(a, BM);
      if (total * col_tiles <= kChooseRounds * kUnits) {
        const int three = count(a, BM / 4 * 3), half = count(a, BM / 2);
        int cost = 100 * rounds(total);
        if (87 * rounds(three) < cost) cost = 87 * rounds(three), high = BM / 4 * 3, total = three;
        if (half * col_tiles <= kUnits && 73 < cost) high = BM / 2, total = half;
      }
    } else {
      total = count(a, BM);
    }
    upto = lane_scan(tiles_in(hi - lo, high));
  }
  __device__ __forceinline__ RowTile find(const LinearArgs &a, int tile) const {
    int before = 0, l = lo, h = hi, u = upto;
    for (int base = 0;;) {
      const unsigned long long holds = __ballot(before + u > tile);
      if (holds) {
        const int src = __builtin_amdgcn_readfirstlane(__ffsll(holds) - 1);
        const int r0 = __builtin_amdgcn_readlane(l, src), r1 = __builtin_amdgcn_readlane(h, src);
        const int own = tiles_in(r1 - r0, high), first = before + __builtin_amdgcn_readlane(u, src) - own;
        const int at = r0 + (tile - first) * high;
        return {base + src, at, r1 - at < high ? r1 - at : high};
      }
      before += __builtin_amdgcn_readlane(u, 63);
      if ((base += 64) >= a.n) return {0, 0, 0};
      load(a, base, l, h);
      u = lane_scan(tiles_in(h - l, high));
    }
  }
};

// The worker with the `rank`-th most rows (of the first 64; their order beyond that): long contractions start first.
__device__ __forceinline__ int worker_by_rows(const LinearArgs &a, int rank) {
  if (rank >= 64 || a.n == 1) return rank;
  const int lane = threadIdx.x & 63, known = a.n < 64 ? a.n : 64;
  int lo = 0, hi = -1;
  if (lane < known) worker_rows(a, lane, lo, hi);
  const int count = hi - lo;
  int before = 0;
  for (int j = 0; j < known; ++j) {
    const int other = __builtin_amdgcn_readlane(count, j);
    before += other > count || (other == count && j < lane);
  }
  const unsigned long long holds = __ballot(lane < known && before == rank);
  return holds ? __builtin_amdgcn_readfirstlane(__ffsll(holds) - 1) : rank;
}

// A barrier that waits for nothing else: loads stay under way.
__device__ __forceinline__ void bare_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <Product P, class T, class TC, int BM, int BN, int WM, int WN, bool Direct>
__global__ __launch_bounds__(64 * WM * WN) void linear_tile_kernel(LinearArgs a) {
  constexpr int kThreads = 64 * WM * WN, kFm = BM / WM / 16, kFn = BN / WN / 16;
  constexpr Layout kRowLayout = P == kGradWeight ? kAcross : kAlong, kColLayout = P == kForward ? kAlong : kAcross;
  constexpr bool kMixed = P == kForward && sizeof(TC) == 2;
  using Rows = Operand<T, kRowLayout, BM, WM, kThreads, false, Direct>;
  using Cols = Operand<T, kColLayout, BN, WN, kThreads, kMixed, Direct>;
  constexpr int kBuffer = Rows::kTileBytes + Cols::kTileBytes, kLoads = Rows::kLoads + Cols::kLoads;
  __shared__ __attribute__((aligned(1024))) char lds_[kStages * kBuffer];
  const uint32_t lds = uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)lds_));
  constexpr bool kDeal = P == kForward && sizeof(T) == 4;

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, p = lane & 15, q = lane >> 4;
  // the 16-row groups of a tile go to the wavefronts in turn, so that a tile with few rows costs each of them less
  const int wave_row = wave / WN, wave_col = wave % WN;
  const int columns = P == kForward ? a.out : a.in, col_tiles = (columns + BN - 1) / BN;
  const int per_worker = (a.out + BM - 1) / BM * col_tiles;  // weight gradient: tiles of a worker
  // (tiles are counted in 32 bits: memory holds fewer)
  for (int at = blockIdx.x;; at += gridDim.x) {
    // (looked up again for every tile: most blocks have one, and it would hold registers through the products)
    const RowTiles<P == kGradWeight ? 1 << 30 : BM, P != kGradWeight && BM == 256> tiles_of(a, col_tiles);
    // Workgroups go to the eight XCDs in turn.  Each XCD takes a run of neighbouring tiles, of every worker where the workers' tiles
    // differ in length.  fp32 forward products are bound by the matrix cores and their tiles differ by the rows they hold: there the
    // XCDs take kGroup tiles in turn (32 uneven workers, 1999 rows, 777 -> 1003 52.1 us, 58.0; bf16 reads more from memory that way:
    // 64 workers, 4096 rows, 512 -> 512 13.1 us, 11.4).
    int share, all;
    if constexpr (P == kGradWeight) share = (per_worker + kXcds - 1) / kXcds, all = share * a.n;
    else if constexpr (kDeal) share = all = (tiles_of.total * col_tiles + kXcds * kGroup - 1) / (kXcds * kGroup) * kGroup;
    else share = all = (tiles_of.total * col_tiles + kXcds - 1) / kXcds;
    if (at >= kXcds * all) break;
    const int xcd = at % kXcds, turn = at / kXcds;
    int worker, first, count, contracted, column, row_start;
    int number = kDeal ? (turn / kGroup * kXcds + xcd) * kGroup + turn % kGroup : xcd * share + turn, row_tiles = tiles_of.total;
    if constexpr (P == kGradWeight) {
      const int rank = turn / share;
      number = xcd * share + (turn - rank * share), row_tiles = (a.out + BM - 1) / BM;
      worker = worker_by_rows(a, rank);
    }
    if (number >= row_tiles * col_tiles) continue;
    const int group = number / (kGroup * col_tiles), inner = number - group * kGroup * col_tiles;
    const int high = row_tiles - group * kGroup < kGroup ? row_tiles - group * kGroup : kGroup;
    const int row_tile = group * kGroup + inner % high;
    column = inner / high * BN;
    if constexpr (P == kGradWeight) {
      first = row_tile * BM, count = a.out - first < BM ? a.out - first : BM;
      int hi;
      worker_rows(a, worker, row_start, hi);
      row_start = __builtin_amdgcn_readfirstlane(row_start), contracted = __builtin_amdgcn_readfirstlane(hi) - row_start;
    } else {
      const RowTile t = tiles_of.find(a, row_tile);
      worker = t.worker, first = t.first, count = t.count, contracted = P == kForward ? a.in : a.out;
      if (count <= 0) continue;
    }
    const int width = columns - column < BN ? columns - column : BN;
    const T *w = static_cast<const T *>(a.w) + int64_t(worker) * a.ld;
    Rows rows;
    Cols cols;
    if constexpr (P == kForward) {
      rows.init(static_cast<const T *>(a.rows_a) + int64_t(first) * a.lda, a.lda, count, contracted);
      cols.init(w + int64_t(column) * a.in, a.in, width, contracted);
    } else if constexpr (P == kGradInput) {
      rows.init(static_cast<const T *>(a.rows_a) + int64_t(first) * a.lda, a.lda, count, contracted);
      cols.init(w + column, a.in, width, contracted);
    } else {
      rows.init(static_cast<const T *>(a.rows_a) + int64_t(row_start) * a.lda + first, a.lda, count, contracted);
      cols.init(static_cast<const T *>(a.rows_b) + int64_t(row_start) * a.ldb + column, a.ldb, width, contracted);
    }

    f32x4 acc[kFm][kFn];
#pragma unroll
    for (int i = 0; i < kFm; ++i)
#pragma unroll
      for (int j = 0; j < kFn; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    const int steps = (contracted + Rows::kSteps - 1) / Rows::kSteps;
    auto request = [&](int it, uint32_t buffer) {
      if (it < Rows::kLoads) rows.request(it, buffer);
      else cols.request(it - Rows::kLoads, buffer + Rows::kTileBytes);
    };
    auto request_all = [&](uint32_t buffer) {
#pragma unroll
      for (int it = 0; it < kLoads; ++it) request(it, buffer);
      rows.advance(), cols.advance();
    };
    auto deliver = [&](uint32_t buffer) { rows.deliver(buffer), cols.deliver(buffer + Rows::kTileBytes); };
    // step kt ends inside a piece
    const int rest = contracted - (steps - 1) * Rows::kSteps;
    auto trim = [&](int kt, uint32_t buffer) {
      if (Direct && kt + 1 == steps && rest % Rows::kElems) rows.trim(buffer, rest), cols.trim(buffer + Rows::kTileBytes, rest);
    };
    // The products of half a step run while the fragments of the next half are read and, from the moment when all have read a
    // step's second half, the step after the next is requested into its buffer.  Reads and requests go between the products, a few
    // at a time: issued in one go they would hold up the matrix cores, since a wavefront issues in order.  Active: 16-row groups of
    // a wavefront that hold rows.
    auto walk = [&](auto active) {
      constexpr int kActive = decltype(active)::value;
      // Row fragments are read kAhead groups before the products that free their registers would allow, into as many spare ones:
      // first halves hold row r in slot r and go upwards, second halves in slot r - kAhead (the first rows: the spare ones) and go
      // downwards, so that the slot of the row that is read next is always free already.
      constexpr int kAhead = kActive < 2 ? kActive : 2, kLoadsEach = (kLoads + kActive - 1) / kActive, kColsEach = (kFn + kActive - 1) / kActive;
      u32x4 x[kParts][kFn], y[kActive + kAhead];
      const typename Rows::Bases row_bases = Rows::template bases<kFm>(wave_row);
      const typename Cols::Bases col_bases = Cols::template bases<kFn>(wave_col);
      auto read_col = [&](int j, uint32_t buffer, int part) { x[part][j] = Cols::fragment(col_bases, buffer + Rows::kTileBytes, j, part); };
      auto slot = [&](int r, int part) { return part == 0 ? r : r < kAhead ? kActive + r : r - kAhead; };
      auto read_row = [&](int r, uint32_t buffer, int part) { y[slot(r, part)] = Rows::fragment(row_bases, buffer, r, part); };
      // Products of a half; fragments of the next, from the buffer `from`; the second half also requests the step after the next into
      // the other buffer.
      auto half = [&](auto part_, uint32_t from, uint32_t into) {
        constexpr int part = decltype(part_)::value;
#pragma unroll
        for (int e = 0; e < kAhead; ++e) read_row(part == 0 ? e : kActive - 1 - e, from, part ^ 1);
#pragma unroll
        for (int g = 0; g < kActive; ++g) {
          const int i = part == 0 ? g : kActive - 1 - g, next = part == 0 ? i + kAhead : i - kAhead;
          if constexpr (part == 1)
#pragma unroll
            for (int it = g * kLoadsEach; it < (g + 1) * kLoadsEach && it < kLoads; ++it) request(it, into);
#pragma unroll
          for (int j = g * kColsEach; j < (g + 1) * kColsEach && j < kFn; ++j) read_col(j, from, part ^ 1);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int j = 0; j < kFn; ++j) acc[i][j] = multiply<T>(x[part][j], y[slot(i, part)], acc[i][j]);
          __builtin_amdgcn_sched_barrier(0);
          if (next >= 0 && next < kActive) read_row(next, from, part ^ 1);
        }
        if constexpr (part == 1) rows.advance(), cols.advance();
      };
      if (steps == 0) return;
      request_all(lds), deliver(lds);
      request_all(lds + kBuffer);
      if (Direct) wait_loads<kLoads>();
      else wait_all();
      trim(0, lds);
      wait_lds();
      bare_barrier();
#pragma unroll
      for (int j = 0; j < kFn; ++j) read_col(j, lds, 0);
#pragma unroll
      for (int r = 0; r < kActive; ++r) read_row(r, lds, 0);
      uint32_t here = lds, other = lds + kBuffer;
      for (int kt = 0; kt < steps; ++kt) {
        half(std::integral_constant<int, 0>{}, here, 0);
        deliver(other);
        wait_all();
        if (kt + 2 == steps) trim(kt + 1, other), wait_lds();
        bare_barrier();  // the next step is there, and all have read this one
        half(std::integral_constant<int, 1>{}, other, here);
        const uint32_t t = here;
        here = other, other = t;
      }
      wait_all();
    };
    __syncthreads();  // the tile before is done with the buffers
    if (kFm >= 4 && count <= BM / 4) walk(std::integral_constant<int, (kFm + 3) / 4>{});
    else if (kFm >= 2 && count <= BM / 2) walk(std::integral_constant<int, (kFm + 1) / 2>{});
    else if (kFm >= (sizeof(T) == 4 ? 4 : 8) && count <= BM / 4 * 3) walk(std::integral_constant<int, (3 * kFm + 3) / 4>{});
    else walk(std::integral_constant<int, kFm>{});

#pragma unroll
    for (int i = 0; i < kFm; ++i) {
      const int r = 16 * (i * WM + wave_row) + p;
      if (r >= count) continue;
      TC *crow = static_cast<TC *>(a.c) + (P == kGradWeight ? int64_t(worker) * a.ld + int64_t(first + r) * a.in : int64_t(first + r) * a.ldc);
      // results of fragment j, four neighbours from column(j) on
      auto column_of = [&](int j) { return column + (kMixed ? wave_col * (BN / WN) + j / 2 * 32 + 8 * q + 4 * (j % 2) : 16 * Cols::group(j, wave_col) + 4 * q); };
      auto result = [&](int j) {
        const int c = column_of(j), inside = columns - c;
        f32x4 v = acc[i][j];
        if constexpr (P == kForward) {
          if (a.flag)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = v[e] <= 0.f ? 0.f : v[e];  // NaN stays
        } else if constexpr (P == kGradInput) {
          if (a.rows_b) {
            const f32x4 h = load4(static_cast<const T *>(a.rows_b) + int64_t(first + r) * a.ldb + c, inside);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = h[e] > 0.f ? v[e] : 0.f;
          }
        } else if (a.flag) {
          v += load4(crow + c, inside);
        }
        return v;
      };
#pragma unroll
      for (int j = 0; j < kFn; j += kMixed ? 2 : 1) {
        const int c = column_of(j), inside = columns - c;
        if constexpr (kMixed) {  // two fragments' fours are 16 bytes
          const f32x4 u = result(j), v = result(j + 1);
          if (inside >= 8) store8(crow + c, u, v);
          else store4(crow + c, u, inside), store4(crow + c + 4, v, inside - 4);
        } else {
          store4(crow + c, result(j), inside);
        }
      }
    }
  }
}

template <Product P, class T, class TC, int BM, int BN, int WM, int WN>
int launch_tiles(const LinearArgs &a, bool direct, void *stream) {
  const int64_t col_tiles = ceil_div_i64(P == kForward ? a.out : a.in, BN);
  // as many as there can be, whatever the offsets
  int64_t blocks = P == kGradWeight ? (int64_t(ceil_div_i64(a.out, BM)) * col_tiles + kXcds - 1) / kXcds * kXcds * a.n
                                    : ((int64_t(a.rows) / BM + (a.n < a.rows ? a.n : a.rows)) * col_tiles + kXcds * kGroup - 1) / (kXcds * kGroup) * (kXcds * kGroup);
  if (P != kGradWeight && BM == 256 && blocks < kUnits) blocks = kUnits;  // lower tiles (or none)
  if (blocks > 1 << 20) blocks = 1 << 20;
  if (blocks == 0) return 0;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if constexpr (BM > 64) linear_tile_kernel<P, T, TC, BM, BN, WM, WN, true><<<dim3(uint32_t(blocks)), 64 * WM * WN, 0, st>>>(a);  // direct only
  else if constexpr (P == kGradWeight && sizeof(T) == 2)  // direct ones have larger tiles or share rows out
    linear_tile_kernel<P, T, TC, BM, BN, WM, WN, false><<<dim3(uint32_t(blocks)), 64 * WM * WN, 0, st>>>(a);
  else if (direct) linear_tile_kernel<P, T, TC, BM, BN, WM, WN, true><<<dim3(uint32_t(blocks)), 64 * WM * WN, 0, st>>>(a);
  else linear_tile_kernel<P, T, TC, BM, BN, WM, WN, false><<<dim3(uint32_t(blocks)), 64 * WM * WN, 0, st>>>(a);
  return hip_rc(hipGetLastError());
}

// Larger tiles read their operands less often, smaller ones leave fewer rows empty and fewer compute units without a tile, and several
// blocks of them share a compute unit, so that one multiplies while another starts or stores.  bf16, aligned, microseconds
// (256 x 256, 128 x 128, 64 x 128, 64 x 64): 16 workers, 8192 rows, 1024 -> 4096 forward 92, 117, 127, 146, input gradient
// 91, 135, 114, 129; 64 workers, 4096 rows, 512 -> 512 forward 19, 15, 12, 13, weight gradient 39, 26, 29, 35; 4 workers, 64 rows,
// 4096 -> 4096 forward 55, 40, 36, 32.  The fp32 matrix cores are so much slower that the empty rows decide: 8 workers, 4096 rows,
// 1024 -> 1024 248, 137, 105, 95; and tiles that pass registers have none to spare: 16 workers, 8192 rows, 1001 -> 4003 321, 245, 204, 220.
template <Product P, class T, class TC>
int launch_product(const LinearArgs &a, bool direct, void *stream) {
  const int columns = P == kForward ? a.out : a.in;
  auto tiles = [&](int m, int n) {
    const int64_t down = P == kGradWeight ? int64_t(ceil_div_i64(a.out, m)) * a.n : a.rows / m + (a.n + 1) / 2;
    return down * ceil_div_i64(columns, n);
  };
  // Few tiles, microseconds (kernels for few tiles with blocks of 16 rows, of 64 rows, tiles), bf16 unless said otherwise.  Forward: 1 row,
  // 4096 -> 4096 7.6, 16.1, 31; 64 rows 30.9, 16.8, 32.4; 128 rows 57.8, 16.9, 32.4; 1000 rows, 2048 -> 64 6.8, 10.3, 15.3; 1024 rows,
  // 1024 -> 1024 82.6, 8.0, 9.9; 4 workers of 512 rows, 256 -> 1024 32, 14.9, 6.9; 64 workers of a row, 512 -> 512 10.6, 10.2, 7.7; fp32,
  // 85 rows, 1320 -> 64 8.0, 29, 35.7.  Input gradient: 1 row, 4096 -> 4096 10.5, 17.3, 31; 128 rows 24.6, 19.5, 34; 1024 rows, 1024 -> 1024
  // 18.9, 9.2, 11.1; 3 uneven workers, 771 rows, 612 -> 446 14.3, 7.4, 7.7; fp32, 2 workers of 64 rows, 2048 -> 2048 18, 44, 56.  Blocks of 64
  // rows pass LDS directly only: through registers they were no faster than tiles.
  if constexpr (P != kGradWeight) {
    // blocks of m x n, workers alike
    auto blocks = [&](int m, int n) { return int64_t(a.n) * ceil_div_i64(ceil_div_i64(a.rows, a.n), m) * ceil_div_i64(columns, n); };
    const bool deep = (P == kForward ? a.in : a.out) >= int(8 * kStepBytes / sizeof(T));
    const bool sixteen = P == kForward ? deep && blocks(16, 16) <= 512 : (direct || deep) && blocks(16, 64) <= 256;
    if (sixteen) return launch_linear_few<P == kForward, T, TC>(a, direct, true, stream);
    if (direct && deep && blocks(64, 64) <= 256) return launch_linear_few<P == kForward, T, TC>(a, direct, false, stream);
  }
  const bool large = tiles(128, 128) >= 256;
  if constexpr (sizeof(T) == 2) {
    const int64_t each = a.rows / a.n;  // rows of a worker
    if (direct && each >= 192 && tiles(256, 256) >= 128) return launch_tiles<P, T, TC, 256, 256, 2, 4>(a, direct, stream);
    if (direct && (P == kGradWeight || each >= 96) && large) return launch_tiles<P, T, TC, 128, 128, 2, 2>(a, direct, stream);
  }
  // fp32 weight gradients of few rows are bound by the result instead (128 x 128, 64 x 64): 16 workers, 256 rows, 2048 -> 2048 96, 110; 64
  // workers, 4096 rows, 512 -> 512 47, 57; 32 workers, 512 rows, 777 -> 1003 46, 53; but with 256 tiles, 4 workers, 512 rows, 1024 -> 1024
  // 18.9, 17.3, and where long workers end last, 8 uneven workers, 4096 rows, 1024 -> 1024 124, 87.
  if constexpr (P == kGradWeight && sizeof(T) == 4)
    if (direct && a.rows <= 128 * int64_t(a.n) && tiles(128, 128) >= 512) return launch_tiles<P, T, TC, 128, 128, 2, 2>(a, direct, stream);
  // Few tiles with a sum over all rows in each, microseconds (rows shared out, one tile after the other): 1 worker of 4096 rows, 64 -> 64
  // 15.7, 25.3 and 256 -> 4096 25.3, 33.5; 4 uneven workers of 2048 rows, 512 -> 512 20.4, 33.7; the same in fp32 98, 111; 4 workers of 64
  // rows 5.0, 4.6; where there are tiles enough, 4 workers of 512 rows, 1024 -> 1024, 21.5, 15.8.  Through registers it was the slower.
  if constexpr (P == kGradWeight)
    if (direct && !large) return launch_linear_weight_split<T>(a, stream);
  if constexpr (sizeof(T) == 2)
    if (tiles(64, 128) >= 256) return launch_tiles<P, T, TC, 64, 128, 2, 2>(a, direct, stream);
  // fp32 rows in sixteens (a wavefront has all rows of 16 columns) and in thirty-twos (half of 32): 8 workers, 4096 uneven rows, 1024 -> 1024
  // forward 93.0, 95.5, input gradient 95.0, 100; 1 worker, 4096 rows, 2048 -> 2048 272, 279 and 281, 292
  if constexpr (P != kGradWeight && sizeof(T) == 4) return launch_tiles<P, T, TC, 64, 64, 1, 4>(a, direct, stream);
  else return launch_tiles<P, T, TC, 64, 64, 2, 2>(a, direct, stream);
}

// Tiles go straight to LDS where rows start on whole dwords and the rows of a step are within a buffer's offsets.
bool on_dwords(const void *p, int64_t pitch, size_t elem) {
  return reinterpret_cast<uintptr_t>(p) % 4 == 0 && pitch * int64_t(elem) % 4 == 0 && 256 * pitch * int64_t(elem) < kBufferMax;
}

}  // namespace

int launch_linear(const Shape &s, const void *W, int64_t offset, bool bf16, const void *A, int64_t lda, const int32_t *rows, int M, int in,
                  int out, bool relu, void *Y, int64_t ldy, bool y_bf16, void *stream) {
  const size_t e = bf16 ? 2 : 4;
  LinearArgs a{static_cast<const char *>(W) + offset * e, A, nullptr, Y, rows, s.ld, lda, 0, ldy, s.n, M, in, out, relu};
  const bool direct = on_dwords(a.w, in, e) && s.ld * e % 4 == 0 && on_dwords(A, lda, e);
  if (!bf16) return launch_product<kForward, float, float>(a, direct, stream);
  return y_bf16 ? launch_product<kForward, bf16_t, bf16_t>(a, direct, stream) : launch_product<kForward, bf16_t, float>(a, direct, stream);
}

int launch_linear_grad_input(const Shape &s, const void *W, int64_t offset, bool bf16, const void *dY, int64_t ldy, const int32_t *rows, int M,
                             int in, int out, const void *H, int64_t ldh, void *dA, int64_t lda, void *stream) {
  const size_t e = bf16 ? 2 : 4;
  LinearArgs a{static_cast<const char *>(W) + offset * e, dY, H, dA, rows, s.ld, ldy, ldh, lda, s.n, M, in, out, 0};
  const bool direct = on_dwords(a.w, in, e) && s.ld * e % 4 == 0 && on_dwords(dY, ldy, e);
  return bf16 ? launch_product<kGradInput, bf16_t, bf16_t>(a, direct, stream) : launch_product<kGradInput, float, float>(a, direct, stream);
}

int launch_linear_grad_weight(const Shape &s, bool bf16, const void *dY, int64_t ldy, const void *A, int64_t lda, const int32_t *rows, int M, int in,
                              int out, float *G, int64_t offset, bool accumulate, void *stream) {
  const size_t e = bf16 ? 2 : 4;
  LinearArgs a{nullptr, dY, A, G + offset, rows, s.ld, ldy, lda, 0, s.n, M, in, out, accumulate};
  const bool direct = on_dwords(dY, ldy, e) && on_dwords(A, lda, e);
  return bf16 ? launch_product<kGradWeight, bf16_t, float>(a, direct, stream) : launch_product<kGradWeight, float, float>(a, direct, stream);
}

}  // namespace detag

// The tile kernel of a layer's products and the choice of tiles (k_linear.hip has the mathematics, the layouts and what was measured).
// Epilogue: what linear_epilogue.hpp adds goes over the sums before they are stored (k_linear_act.hip).
#pragma once

#include "dev_common.hpp"
#include "detag_internal.h"
#include "linear_common.hpp"
#include "linear_epilogue.hpp"
#include "rows_common.hpp"

namespace detag {
namespace {

enum Product : int { kForward, kGradInput, kGradWeight };

constexpr int kStages = 2;      // steps in LDS
constexpr int kXcds = 8;
constexpr int kUnits = 256;     // compute units
constexpr int kChooseRounds = 4;  // tiles for each up to which the height of 256-row tiles is chosen
constexpr int kGroup = 8;       // row tiles that are walked together, column by column

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
    return __builtin_amdgcn_readlane(wave_scan(sum), 63);
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
    upto = wave_scan(tiles_in(hi - lo, high));
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
      u = wave_scan(tiles_in(h - l, high));
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

template <Product P, class T, class TC, int BM, int BN, int WM, int WN, bool Direct, bool Epilogue>
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

    // results of fragment j, four neighbours from column(j) on
    auto column_of = [&](int j) { return column + (kMixed ? wave_col * (BN / WN) + j / 2 * 32 + 8 * q + 4 * (j % 2) : 16 * Cols::group(j, wave_col) + 4 * q); };
    const int64_t row0 = first;
    if constexpr (Epilogue) {
      // The input gradient requests all that it reads for the tile in one go, where its rows start on whole dwords (a.flag): the products' fragments
      // have left registers for that, and a group of rows at a time waits for memory eight times a tile.  8192 uneven rows, 16 workers, 4096 ->
      // 1024, gelu: 147 us, and 133.  The forward product's residual was the slower for it (1024 outputs of 4096: 103, 109), since its biases
      // are held too.
      constexpr bool kFwd = P == kForward;
      using Read = std::conditional_t<kFwd, TC, T>;
      const Read *const reads = static_cast<const Read *>(kFwd ? a.residual : a.rows_b);
      const int64_t ld_reads = kFwd ? a.ldr : a.ldb;
      constexpr int kBatch = sizeof(Read) == 2 || kFm < 2 ? kFm : kFm / 2;
      auto row_of = [&](int i) { return 16 * (i * WM + wave_row) + p; };
      f32x4 bias[kFwd ? kFn : 1];
      auto finish = [&](auto act, auto buffered) {
        constexpr int kAct = decltype(act)::value;
        constexpr bool kBuffered = decltype(buffered)::value;
        Four<Read> read[kBuffered ? kBatch : 1][kFn];
        auto inside_of = [&](int j) { return columns - column_of(j); };
        // What is out of a buffer's range reads as zero; what is past a row's end is not stored.
        auto request_reads = [&](int i) {
          const int above = 16 * (i * WM + wave_row), rows = count - above < 16 ? count - above : 16;
          const int64_t bytes = rows > 0 && reads ? ((rows - 1) * ld_reads + columns - column) * int64_t(sizeof(Read)) : 0;
          const rsrc_t from = make_rsrc(reads + (row0 + above) * ld_reads + column, uint32_t(bytes + 3) & ~3u);  // whole dwords
          const uint32_t off = (uint32_t(p) * uint32_t(ld_reads) + uint32_t(column_of(0) - column)) * uint32_t(sizeof(Read));
#pragma unroll
          for (int j = 0; j < kFn; ++j) {
            const int at = int(off) + (column_of(j) - column_of(0)) * int(sizeof(Read));
            if constexpr (sizeof(Read) == 2) read[i % kBatch][j].bits = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(from, at, 0, 0));
            else read[i % kBatch][j].bits = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from, at, 0, 0));
          }
        };
        if constexpr (kFwd)
#pragma unroll
          for (int j = 0; j < kFn; ++j) bias[j] = bias_of<T>(a, worker, column_of(j));
#pragma unroll
        for (int i = 0; i < kFm; ++i) {
          if constexpr (kBuffered) {
            if (i % kBatch == 0) {
#pragma unroll
              for (int k = i; k < i + kBatch; ++k) request_reads(k);
              __builtin_amdgcn_sched_barrier(0);
            }
          } else if (reads) {
            const int r = row_of(i) < count ? row_of(i) : count - 1;
#pragma unroll
            for (int j = 0; j < kFn; ++j) read[0][j] = read_four(reads + (row0 + r) * ld_reads + column_of(j), columns - column_of(j));
          }
          const int r = row_of(i);
          // two fragments' fours are 16 bytes (Mixed)
          auto put = [&](auto *to) {
            using TO = std::remove_pointer_t<decltype(to)>;
#pragma unroll
            for (int j = 0; j < kFn; j += kMixed ? 2 : 1) {
              const int c = column_of(j), inside = inside_of(j);
              if constexpr (kMixed && sizeof(TO) == 2) {
                if (inside >= 8) store8(to + c, acc[i][j], acc[i][j + 1]);
                else store4(to + c, acc[i][j], inside), store4(to + c + 4, acc[i][j + 1], inside - 4);
              } else {
                store4(to + c, acc[i][j], inside);
                if (kMixed) store4(to + column_of(j + 1), acc[i][j + 1], inside_of(j + 1));
              }
            }
          };
          if constexpr (kFwd) {
#pragma unroll
            for (int j = 0; j < kFn; ++j) acc[i][j] += bias[j];
            if (a.pre && r < count) put(static_cast<T *>(a.pre) + (row0 + r) * a.ldz);
          }
#pragma unroll
          for (int j = 0; j < kFn; ++j) {
            if constexpr (kFwd) {
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[i][j][e] = act_value<TC>(acc[i][j][e], kAct);
            } else if constexpr (kAct != DETAG_ACT_NONE) {
              const f32x4 z = read[kBuffered ? i % kBatch : 0][j].floats();
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[i][j][e] *= act_slope<T>(z[e], kAct);
            }
          }
          if (kFwd && reads)
#pragma unroll
            for (int j = 0; j < kFn; ++j) acc[i][j] += read[kBuffered ? i % kBatch : 0][j].floats();
          if (r < count) put(static_cast<TC *>(a.c) + (row0 + r) * a.ldc);
        }
      };
      with_act(a.act, [&](auto act) {
        if constexpr (kFm * kFn >= 16 && !kFwd) {
          if (a.flag) return finish(act, std::true_type{});
        }
        finish(act, std::false_type{});
      });
      continue;
    }
#pragma unroll
    for (int i = 0; i < kFm; ++i) {
      const int r = 16 * (i * WM + wave_row) + p;
      if (r >= count) continue;
      TC *crow = static_cast<TC *>(a.c) + (P == kGradWeight ? int64_t(worker) * a.ld + int64_t(first + r) * a.in : int64_t(first + r) * a.ldc);
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

template <Product P, class T, class TC, bool Epilogue, int BM, int BN, int WM, int WN>
int launch_tiles(const LinearArgs &a, bool direct, void *stream) {
  const int64_t col_tiles = ceil_div_i64(P == kForward ? a.out : a.in, BN);
  // as many as there can be, whatever the offsets
  int64_t blocks = P == kGradWeight ? (int64_t(ceil_div_i64(a.out, BM)) * col_tiles + kXcds - 1) / kXcds * kXcds * a.n
                                    : ((int64_t(a.rows) / BM + (a.n < a.rows ? a.n : a.rows)) * col_tiles + kXcds * kGroup - 1) / (kXcds * kGroup) * (kXcds * kGroup);
  if (P != kGradWeight && BM == 256 && blocks < kUnits) blocks = kUnits;  // lower tiles (or none)
  if (blocks > 1 << 20) blocks = 1 << 20;
  if (blocks == 0) return 0;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if constexpr (BM > 64) linear_tile_kernel<P, T, TC, BM, BN, WM, WN, true, Epilogue><<<dim3(uint32_t(blocks)), 64 * WM * WN, 0, st>>>(a);  // direct only
  else if constexpr (P == kGradWeight && sizeof(T) == 2)  // direct ones have larger tiles or share rows out
    linear_tile_kernel<P, T, TC, BM, BN, WM, WN, false, Epilogue><<<dim3(uint32_t(blocks)), 64 * WM * WN, 0, st>>>(a);
  else if (direct) linear_tile_kernel<P, T, TC, BM, BN, WM, WN, true, Epilogue><<<dim3(uint32_t(blocks)), 64 * WM * WN, 0, st>>>(a);
  else linear_tile_kernel<P, T, TC, BM, BN, WM, WN, false, Epilogue><<<dim3(uint32_t(blocks)), 64 * WM * WN, 0, st>>>(a);
  return hip_rc(hipGetLastError());
}

// Larger tiles read their operands less often, smaller ones leave fewer rows empty and fewer compute units without a tile, and several
// blocks of them share a compute unit, so that one multiplies while another starts or stores.  bf16, aligned, microseconds
// (256 x 256, 128 x 128, 64 x 128, 64 x 64): 16 workers, 8192 rows, 1024 -> 4096 forward 92, 117, 127, 146, input gradient
// 91, 135, 114, 129; 64 workers, 4096 rows, 512 -> 512 forward 19, 15, 12, 13, weight gradient 39, 26, 29, 35; 4 workers, 64 rows,
// 4096 -> 4096 forward 55, 40, 36, 32.  The fp32 matrix cores are so much slower that the empty rows decide: 8 workers, 4096 rows,
// 1024 -> 1024 248, 137, 105, 95; and tiles that pass registers have none to spare: 16 workers, 8192 rows, 1001 -> 4003 321, 245, 204, 220.
template <Product P, class T, class TC, bool Epilogue = false>
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
    if (sixteen) return launch_linear_few<P == kForward, T, TC, Epilogue>(a, direct, true, stream);
    if (direct && deep && blocks(64, 64) <= 256) return launch_linear_few<P == kForward, T, TC, Epilogue>(a, direct, false, stream);
  }
  const bool large = tiles(128, 128) >= 256;
  if constexpr (sizeof(T) == 2) {
    const int64_t each = a.rows / a.n;  // rows of a worker
    if (direct && each >= 192 && tiles(256, 256) >= 128) return launch_tiles<P, T, TC, Epilogue, 256, 256, 2, 4>(a, direct, stream);
    if (direct && (P == kGradWeight || each >= 96) && large) return launch_tiles<P, T, TC, Epilogue, 128, 128, 2, 2>(a, direct, stream);
  }
  // fp32 weight gradients of few rows are bound by the result instead (128 x 128, 64 x 64): 16 workers, 256 rows, 2048 -> 2048 96, 110; 64
  // workers, 4096 rows, 512 -> 512 47, 57; 32 workers, 512 rows, 777 -> 1003 46, 53; but with 256 tiles, 4 workers, 512 rows, 1024 -> 1024
  // 18.9, 17.3, and where long workers end last, 8 uneven workers, 4096 rows, 1024 -> 1024 124, 87.
  if constexpr (P == kGradWeight && sizeof(T) == 4)
    if (direct && a.rows <= 128 * int64_t(a.n) && tiles(128, 128) >= 512) return launch_tiles<P, T, TC, Epilogue, 128, 128, 2, 2>(a, direct, stream);
  // Few tiles with a sum over all rows in each, microseconds (rows shared out, one tile after the other): 1 worker of 4096 rows, 64 -> 64
  // 15.7, 25.3 and 256 -> 4096 25.3, 33.5; 4 uneven workers of 2048 rows, 512 -> 512 20.4, 33.7; the same in fp32 98, 111; 4 workers of 64
  // rows 5.0, 4.6; where there are tiles enough, 4 workers of 512 rows, 1024 -> 1024, 21.5, 15.8.  Through registers it was the slower.
  if constexpr (P == kGradWeight)
    if (direct && !large) return launch_linear_weight_split<T>(a, stream);
  if constexpr (sizeof(T) == 2)
    if (tiles(64, 128) >= 256) return launch_tiles<P, T, TC, Epilogue, 64, 128, 2, 2>(a, direct, stream);
  // fp32 rows in sixteens (a wavefront has all rows of 16 columns) and in thirty-twos (half of 32): 8 workers, 4096 uneven rows, 1024 -> 1024
  // forward 93.0, 95.5, input gradient 95.0, 100; 1 worker, 4096 rows, 2048 -> 2048 272, 279 and 281, 292
  if constexpr (P != kGradWeight && sizeof(T) == 4) return launch_tiles<P, T, TC, Epilogue, 64, 64, 1, 4>(a, direct, stream);
  else return launch_tiles<P, T, TC, Epilogue, 64, 64, 2, 2>(a, direct, stream);
}

// Whether what an epilogue reads may come through a buffer: rows that start on whole dwords, and 16 of them within its offsets.
inline bool reads_by_buffer(const void *p, int64_t pitch, size_t elem) {
  return reinterpret_cast<uintptr_t>(p) % 4 == 0 && pitch * int64_t(elem) % 4 == 0 && 16 * pitch * int64_t(elem) < kBufferMax;
}

// Tiles go straight to LDS where rows start on whole dwords and the rows of a step are within a buffer's offsets.
bool on_dwords(const void *p, int64_t pitch, size_t elem) {
  return reinterpret_cast<uintptr_t>(p) % 4 == 0 && pitch * int64_t(elem) % 4 == 0 && 256 * pitch * int64_t(elem) < kBufferMax;
}

}  // namespace
}  // namespace detag

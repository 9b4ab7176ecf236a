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
// banks.  Where rows start on 16 bytes (and the contraction is whole pieces) tiles go from memory to LDS without passing registers;
// the hardware's range check of the buffer loads zeroes what lies past a worker's rows or the end of the contraction.  Otherwise
// they pass registers.
//
// MFMA operand layout (lane l, p = l % 16, q = l / 16): 16x16x32 bf16 operands hold index p, k = 8q..8q+7; the four 16x16x4 fp32
// products of a piece hold index p, k = 4q+t for product t; the result's register r is (index 4q+r of the first, p of the second).
// The columns of the result are the first operand, so that a lane holds neighbours of a row.
#include "dev_common.hpp"
#include "detag_internal.h"

namespace detag {
namespace {

enum Product : int { kForward, kGradInput, kGradWeight };
enum Layout : int { kAlong, kAcross };

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// pieces at any address their elements may have
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef __attribute__((address_space(3))) char lds_char;

constexpr int kStepBytes = 128;  // of the contraction, per LDS step: a cache line
constexpr int kPieces = kStepBytes / 16;
constexpr int kParts = 2;       // of a step: one MFMA of bf16, four of fp32 each
constexpr int kStages = 2;      // steps in LDS
constexpr int kXcds = 8;
constexpr int kGroup = 8;       // row tiles that are walked together, column by column
constexpr int64_t kBufferMax = (int64_t(1) << 31) - 1;  // bytes a buffer resource is made for at most

struct LinearArgs {
  const void *w;       // n x ld weights, already at the layer's first column
  const void *rows_a;  // A, or dY for the input gradient
  const void *rows_b;  // weight gradient: A (rows_a is dY); input gradient: H or null
  void *c;             // Y, dA or G at the layer's first column
  const int32_t *offsets;
  int64_t ld, lda, ldb, ldc;  // pitches in elements: of w (and G), rows_a, rows_b, c
  int n, rows, in, out;
  int flag;  // forward: relu; weight gradient: accumulate
};

// A worker's rows, kept inside the row matrices whatever the offsets say.
__device__ __forceinline__ void worker_rows(const LinearArgs &a, int i, int &lo, int &hi) {
  lo = a.offsets[i], hi = a.offsets[i + 1];
  lo = lo < 0 ? 0 : lo > a.rows ? a.rows : lo;
  hi = hi < lo ? lo : hi > a.rows ? a.rows : hi;
}

// Row tiles of BM rows, counted worker by worker: which worker a number belongs to, and how many there are in all.  Every
// wavefront looks for itself: 64 workers at a time, a scan over the lanes; the first 64 are kept.
struct RowTile {
  int worker, first, count;  // first row, rows of the tile (0: no such tile)
};
template <int BM>
struct RowTiles {
  int lo = 0, hi = 0, upto = 0, total = 0;

  __device__ __forceinline__ static int scan(const LinearArgs &a, int base, int &lo, int &hi) {
    const int lane = threadIdx.x & 63;
    lo = hi = 0;
    if (base + lane < a.n) worker_rows(a, base + lane, lo, hi);
    int upto = (hi - lo + BM - 1) / BM;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int v = __shfl_up(upto, d);
      if (lane >= d) upto += v;
    }
    return upto;
  }
  __device__ __forceinline__ explicit RowTiles(const LinearArgs &a) {
    upto = scan(a, 0, lo, hi);
    total = __builtin_amdgcn_readlane(upto, 63);
    for (int base = 64; base < a.n; base += 64) {
      int l, h;
      total += __builtin_amdgcn_readlane(scan(a, base, l, h), 63);
    }
  }
  __device__ __forceinline__ RowTile find(const LinearArgs &a, int tile) const {
    int before = 0, l = lo, h = hi, u = upto;
    for (int base = 0;;) {
      const unsigned long long holds = __ballot(before + u > tile);
      if (holds) {
        const int src = __builtin_amdgcn_readfirstlane(__ffsll(holds) - 1);
        const int r0 = __builtin_amdgcn_readlane(l, src), r1 = __builtin_amdgcn_readlane(h, src);
        const int own = (r1 - r0 + BM - 1) / BM, first = before + __builtin_amdgcn_readlane(u, src) - own;
        const int at = r0 + (tile - first) * BM;
        return {base + src, at, r1 - at < BM ? r1 - at : BM};
      }
      before += __builtin_amdgcn_readlane(u, 63);
      if ((base += 64) >= a.n) return {0, 0, 0};
      u = scan(a, base, l, h);
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

// 16 bytes a lane from a buffer into LDS, the wavefront's 1024 from `lds` on; what is out of the buffer's range arrives as zeros.  As
// an instruction of its own and not the builtin, because behind that the compiler lets every transposing read wait for all loads
// under way, whichever part of LDS they go to; the waits are in the kernel.  It leaves no register written.
__device__ __forceinline__ void load_to_lds(u32x4 resource, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(offset), "s"(resource), "s"(lds) : "memory", "m0");
}

template <class V>
__device__ __forceinline__ V read_lds(uint32_t at) {
  return *reinterpret_cast<const __attribute__((address_space(3))) V *>(at);
}

// One operand of a tile: ROWS of its own index by one step of the contraction, in LDS from `lds` on.
//   kAlong : base at (first row, k = 0); `valid` rows, `contracted` elements in each
//   kAcross: base at (k = 0, first column); `valid` columns
// The operand's index is dealt out to WAVES wavefronts in groups of 16, in turn; Mixed: in runs of 16 * GROUPS.
template <class T, Layout L, int ROWS, int WAVES, int THREADS, bool Mixed, bool Direct>
struct Operand {
  static constexpr int kElems = 16 / sizeof(T);               // elements of a piece
  static constexpr int kSteps = kStepBytes / sizeof(T);       // contracted elements of a step
  static constexpr int kTileBytes = ROWS * kStepBytes;
  static constexpr int kLoads = ROWS * kPieces / THREADS;     // pieces a thread moves per step
  static constexpr int kRowPieces = L == kAlong ? kPieces : ROWS / kElems;
  static constexpr int kRowBytes = 16 * kRowPieces;
  static_assert(kLoads * THREADS == ROWS * kPieces, "the threads share the pieces evenly");

  const char *base;  // the next step's
  int64_t pitch;     // bytes
  int64_t bytes;     // that belong to the operand, from `base` on
  int valid, contracted;  // contracted: from `base` on
  // A thread's pieces of a step lie kRowsApart LDS rows apart.  Where that leaves spread() as it is, one offset serves them all and
  // the distance goes into the buffer's base, which costs no vector registers.
  static constexpr int kRowsApart = THREADS / kRowPieces;
  static constexpr bool kOneOffset = kRowsApart % (L == kAlong ? 32 : 16) == 0;
  uint32_t off[Direct ? (kOneOffset ? 1 : kLoads) : 1];
  uint32_t now;  // the step's
  int left;      // bytes of the buffer that the step's loads use
  u32x4 held[Direct ? 1 : kLoads];

  // Which position of an LDS row a piece is kept at: bits that are xor-ed to the piece's number.
  __device__ static __forceinline__ int spread(int row) {
    if constexpr (L == kAlong) return Mixed ? (row & 3) | ((row >> 4) & 1) << 2 : row & 7;
    else if constexpr (sizeof(T) == 2) return (row & 3) << 1;
    else return (((row >> 2) & 3) << 2) & (kRowPieces - 1);
  }

  __device__ __forceinline__ void place(int it, int &row, int &piece) const {
    const int id = it * THREADS + threadIdx.x;
    row = id / kRowPieces, piece = (id % kRowPieces) ^ spread(row);
  }

  __device__ __forceinline__ void init(const void *b, int64_t pitch_elems, int valid_, int contracted_) {
    base = static_cast<const char *>(b), pitch = pitch_elems * int64_t(sizeof(T)), valid = valid_, contracted = contracted_;
    bytes = L == kAlong ? (valid - 1) * pitch + contracted * int64_t(sizeof(T)) : (contracted - 1) * pitch + valid * int64_t(sizeof(T));
    if constexpr (Direct) {
#pragma unroll
      for (int it = 0; it < (kOneOffset ? 1 : kLoads); ++it) {
        int row, piece;
        place(it, row, piece);
        off[it] = uint32_t(row * pitch) + 16u * piece;
      }
    }
    aim();
  }

  // A step is requested piece by piece (directly into LDS, or into registers), then advance() goes on to the next.  What lies past
  // the end of the contraction arrives as zeros.
  __device__ __forceinline__ void request(int it, uint32_t lds) {
    if constexpr (Direct) {
      const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
      const int away = kOneOffset ? it * kRowsApart * int(pitch) : 0;
      const uint64_t from = reinterpret_cast<uint64_t>(base) + uint32_t(away);
      const u32x4 r = {uint32_t(from), uint32_t(from >> 32), uint32_t(left > away ? left - away : 0), 0x00020000u};
      load_to_lds(r, kOneOffset ? now : off[it], lds + (it * THREADS + wave * 64) * 16);
    } else {
      int row, piece;
      place(it, row, piece);
      const int k = L == kAlong ? piece * kElems : row, x = L == kAlong ? row : piece * kElems;
      const int inside = L == kAlong ? (x < valid ? contracted - k : 0) : (k < contracted ? valid - x : 0);
      const char *p = base + (L == kAlong ? x * pitch + k * int64_t(sizeof(T)) : k * pitch + x * int64_t(sizeof(T)));
      u32x4 v = {0, 0, 0, 0};
      if (inside >= kElems) {
        v = *reinterpret_cast<const u32x4_any *>(p);
      } else if (inside > 0) {
        union {
          u32x4 v;
          T e[kElems];
        } u;
        u.v = v;
#pragma unroll
        for (int e = 0; e < kElems; ++e)
          if (e < inside) u.e[e] = reinterpret_cast<const T *>(p)[e];
        v = u.v;
      }
      held[it] = v;
    }
  }
  __device__ __forceinline__ void advance() {
    const int64_t skip = L == kAlong ? int64_t(kStepBytes) : kSteps * pitch;
    base += skip, bytes -= skip, contracted -= kSteps;
    aim();
  }
  // The next step's range, and (kAlong) which of the thread's pieces are past the contraction's end.
  __device__ __forceinline__ void aim() {
    if constexpr (Direct) {
      // what is left of the operand, as far as a buffer counts (a step's offsets stay below that)
      left = bytes < 0 ? 0 : bytes < kBufferMax ? int(bytes) : int(kBufferMax);
      now = off[0];
      if constexpr (L == kAlong) {
        static_assert(kOneOffset || !Direct, "one piece number for all rows of a thread");
        int row, piece;
        place(0, row, piece);
        if (16 * piece >= contracted * int(sizeof(T))) now = 0xffffff00u;
      }
    }
  }

  // Writes what request() left in registers.
  __device__ __forceinline__ void deliver(uint32_t lds) {
    if constexpr (!Direct) {
#pragma unroll
      for (int it = 0; it < kLoads; ++it)
        *reinterpret_cast<__attribute__((address_space(3))) u32x4 *>(lds + (it * THREADS + threadIdx.x) * 16) = held[it];
    }
  }

  // Where a lane reads: fragment f, part s of a step is at address(wave, ...) plus constants.  kAcross with bf16: a fragment is 32
  // bytes of an LDS row, four of which share 128 bytes and are xor-ed; two wavefronts' fragments alternate in those.
  static constexpr int kBases = L == kAlong ? kParts : sizeof(T) == 2 ? (WAVES % 4 == 0 ? 1 : WAVES == 2 ? 2 : 4) : 4;
  struct Bases {
    uint32_t at[kBases];
  };
  template <int GROUPS>
  __device__ static __forceinline__ Bases bases(int wave) {
    const int lane = threadIdx.x & 63, p = lane & 15, q = lane >> 4;
    Bases b;
    if constexpr (L == kAlong) {
      const int row = Mixed ? 16 * GROUPS * wave + 16 * (p >> 2) + (p & 3) : 16 * wave + p;
#pragma unroll
      for (int s = 0; s < kParts; ++s) b.at[s] = row * kRowBytes + (((4 * s + q) ^ spread(row)) << 4);
    } else if constexpr (sizeof(T) == 2) {
      const int k = 8 * q + (p >> 2);
#pragma unroll
      for (int v = 0; v < kBases; ++v) {
        const int piece = 2 * (v * WAVES + wave) + ((p >> 1) & 1);  // lane's 8 bytes: columns 4 * (p % 4) of the fragment
        b.at[v] = k * kRowBytes + ((piece ^ spread(k)) << 4) + (p & 1) * 8;
      }
    } else {
      const int col = 16 * wave + p;
#pragma unroll
      for (int t = 0; t < 4; ++t) b.at[t] = (4 * q + t) * kRowBytes + (((col >> 2) ^ spread(4 * q + t)) << 4) + (col & 3) * 4;
    }
    return b;
  }

  // Lane's 16 bytes of fragment f.  Mixed: index p of fragment f of a run of 64 stands for 16*(p/4) + 4f + p%4, so that four fragments
  // give a lane 16 neighbours.
  __device__ __forceinline__ static u32x4 fragment(const Bases &b, uint32_t lds, int f, int s) {
    if constexpr (L == kAlong) {
      const int row = Mixed ? f / 4 * 64 + f % 4 * 4 : 16 * WAVES * f;
      return read_lds<u32x4>(b.at[s] + lds + row * kRowBytes);
    } else if constexpr (sizeof(T) == 2) {
      // groups 16 * (WAVES f + wave): the part below four groups is in the base
      const uint32_t at = b.at[f % kBases] + lds + f / kBases * (kBases * WAVES * 32) + 32 * s * kRowBytes;
      auto read = [&](uint32_t a) {
        return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) s16x4 *>(a)));
      };
      const u32x2 lo = read(at), hi = read(at + 4 * kRowBytes);
      return u32x4{lo[0], lo[1], hi[0], hi[1]};
    } else {
      u32x4 v;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        // spread() touches pieces 4 and 8, that is 16 and 32 columns: fragments of 16 columns are xor-ed among four
        const uint32_t at = (b.at[t] ^ (f * WAVES % 4 << 6)) + f * WAVES / 4 * 256;
        v[t] = read_lds<uint32_t>(at + lds + 16 * s * kRowBytes);
      }
      return v;
    }
  }
};

template <class T>
__device__ __forceinline__ f32x4 multiply(u32x4 x, u32x4 y, f32x4 acc) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), acc, 0, 0, 0);
  } else {
#pragma unroll
    for (int t = 0; t < 4; ++t)
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(f32x4, x)[t], __builtin_bit_cast(f32x4, y)[t], acc, 0, 0, 0);
    return acc;
  }
}

// Four neighbouring results, `inside` of them in the matrix.
template <class T>
__device__ __forceinline__ void store4(T *p, f32x4 v, int inside) {
  if (inside >= 4) {
    if constexpr (sizeof(T) == 2) {
      const u32x2 b = {uint32_t(bf16_bits_rne(v[0])) | uint32_t(bf16_bits_rne(v[1])) << 16,
                       uint32_t(bf16_bits_rne(v[2])) | uint32_t(bf16_bits_rne(v[3])) << 16};
      *reinterpret_cast<u32x2_any *>(p) = b;
    } else {
      *reinterpret_cast<f32x4_any *>(p) = v;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < inside) p[e] = from_f32<T>(v[e]);
  }
}

// Four neighbouring elements at p; those that are not in the matrix read as zero.
template <class T>
__device__ __forceinline__ f32x4 load4(const T *p, int inside) {
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (inside >= 4) {
    if constexpr (sizeof(T) == 2) {
      const u32x2 b = *reinterpret_cast<const u32x2_any *>(p);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(e % 2 ? b[e / 2] & 0xffff0000u : b[e / 2] << 16);
    } else {
      v = *reinterpret_cast<const f32x4_any *>(p);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < inside) v[e] = to_f32(p[e]);
  }
  return v;
}

template <int N>
__device__ __forceinline__ void wait_loads() {  // all but the N newest loads have arrived
  __builtin_amdgcn_s_waitcnt((N & 15) | 7 << 4 | 15 << 8 | (N >> 4) << 14);
}
__device__ __forceinline__ void wait_all() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(7 << 4);
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
  constexpr bool kMixed = P == kForward && kFn % 4 == 0;
  using Rows = Operand<T, kRowLayout, BM, WM, kThreads, false, Direct>;
  using Cols = Operand<T, kColLayout, BN, WN, kThreads, kMixed, Direct>;
  constexpr int kBuffer = Rows::kTileBytes + Cols::kTileBytes, kLoads = Rows::kLoads + Cols::kLoads;
  __shared__ __attribute__((aligned(1024))) char lds_[kStages * kBuffer];
  const uint32_t lds = uint32_t(reinterpret_cast<uintptr_t>((lds_char *)lds_));

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, p = lane & 15, q = lane >> 4;
  // the 16-row groups of a tile go to the wavefronts in turn, so that a tile with few rows costs each of them less
  const int wave_row = wave / WN, wave_col = wave % WN;
  const int columns = P == kForward ? a.out : a.in, col_tiles = (columns + BN - 1) / BN;
  const int per_worker = (a.out + BM - 1) / BM * col_tiles;  // weight gradient: tiles of a worker
  for (int64_t at = blockIdx.x;; at += gridDim.x) {
    // (looked up again for every tile: most blocks have one, and it would hold registers through the products)
    const RowTiles<P == kGradWeight ? 1 << 30 : BM> tiles_of(a);
    // Workgroups go to the eight XCDs in turn.  Each XCD takes a run of neighbouring tiles, of every worker where the workers' tiles
    // differ in length.
    int64_t share, all;
    if constexpr (P == kGradWeight) share = (per_worker + kXcds - 1) / kXcds, all = share * a.n;
    else share = all = (int64_t(tiles_of.total) * col_tiles + kXcds - 1) / kXcds;
    if (at >= kXcds * all) break;
    const int xcd = int(at % kXcds);
    int worker, first, count, contracted, column, row_start;
    if constexpr (P == kGradWeight) {
      const int64_t turn = at / kXcds;
      const int number = int(xcd * share + turn % share);
      if (number >= per_worker) continue;
      worker = worker_by_rows(a, int(turn / share));
      const int row_tiles = (a.out + BM - 1) / BM, group = number / (kGroup * col_tiles), rest = number - group * kGroup * col_tiles;
      const int high = row_tiles - group * kGroup < kGroup ? row_tiles - group * kGroup : kGroup;
      first = (group * kGroup + rest % high) * BM, column = rest / high * BN;
      count = a.out - first < BM ? a.out - first : BM;
      int hi;
      worker_rows(a, worker, row_start, hi);
      row_start = __builtin_amdgcn_readfirstlane(row_start), contracted = __builtin_amdgcn_readfirstlane(hi) - row_start;
    } else {
      const int64_t number = xcd * share + at / kXcds;
      if (number >= int64_t(tiles_of.total) * col_tiles) continue;
      const int group = int(number / (kGroup * col_tiles)), rest = int(number - int64_t(group) * kGroup * col_tiles);
      const int high = tiles_of.total - group * kGroup < kGroup ? tiles_of.total - group * kGroup : kGroup;
      const RowTile t = tiles_of.find(a, group * kGroup + rest % high);
      worker = t.worker, first = t.first, count = t.count, contracted = P == kForward ? a.in : a.out, column = rest / high * BN;
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
    else walk(std::integral_constant<int, kFm>{});

#pragma unroll
    for (int i = 0; i < kFm; ++i) {
      const int r = 16 * (i * WM + wave_row) + p;
      if (r >= count) continue;
      TC *crow = static_cast<TC *>(a.c) + (P == kGradWeight ? int64_t(worker) * a.ld + int64_t(first + r) * a.in : int64_t(first + r) * a.ldc);
#pragma unroll
      for (int j = 0; j < kFn; ++j) {
        const int c = column + (kMixed ? wave_col * (BN / WN) + j / 4 * 64 + 16 * q + 4 * (j % 4) : 16 * (j * WN + wave_col) + 4 * q), inside = columns - c;
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
        store4(crow + c, v, inside);
      }
    }
  }
}

template <Product P, class T, class TC, int BM, int BN, int WM, int WN>
int launch_tiles(const LinearArgs &a, bool direct, void *stream) {
  const int64_t col_tiles = ceil_div_i64(P == kForward ? a.out : a.in, BN);
  // as many as there can be, whatever the offsets
  int64_t blocks = P == kGradWeight ? (int64_t(ceil_div_i64(a.out, BM)) * col_tiles + kXcds - 1) / kXcds * kXcds * a.n
                                    : ((int64_t(a.rows) / BM + (a.n < a.rows ? a.n : a.rows)) * col_tiles + kXcds - 1) / kXcds * kXcds;
  if (blocks > 1 << 20) blocks = 1 << 20;
  if (blocks == 0) return 0;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if constexpr (BM > 64) linear_tile_kernel<P, T, TC, BM, BN, WM, WN, true><<<dim3(uint32_t(blocks)), 64 * WM * WN, 0, st>>>(a);  // direct only
  else if (direct) linear_tile_kernel<P, T, TC, BM, BN, WM, WN, true><<<dim3(uint32_t(blocks)), 64 * WM * WN, 0, st>>>(a);
  else linear_tile_kernel<P, T, TC, BM, BN, WM, WN, false><<<dim3(uint32_t(blocks)), 64 * WM * WN, 0, st>>>(a);
  return hip_rc(hipGetLastError());
}

// Larger tiles read their operands less often, smaller ones leave fewer rows empty and fewer compute units without a tile, and several
// blocks of them share a compute unit, so that one multiplies while another starts or stores.  bf16, aligned, microseconds
// (256 x 256, 128 x 128, 64 x 128, 64 x 64): 16 workers, 8192 rows, 1024 -> 4096 forward 104, 122, 127, 146, input gradient
// 94, 129, 114, 129; 64 workers, 4096 rows, 512 -> 512 forward 19, 15, 12, 13, weight gradient 39, 26, 29, 35; 4 workers, 64 rows,
// 4096 -> 4096 forward 55, 40, 36, 32.  The fp32 matrix cores are so much slower that the empty rows decide: 8 workers, 4096 rows,
// 1024 -> 1024 248, 137, 105, 95; and tiles that pass registers have none to spare: 16 workers, 8192 rows, 1001 -> 4003 321, 245, 204, 220.
template <Product P, class T, class TC>
int launch_product(const LinearArgs &a, bool direct, void *stream) {
  const int columns = P == kForward ? a.out : a.in;
  auto tiles = [&](int m, int n) {
    const int64_t down = P == kGradWeight ? int64_t(ceil_div_i64(a.out, m)) * a.n : a.rows / m + (a.n + 1) / 2;
    return down * ceil_div_i64(columns, n);
  };
  if constexpr (sizeof(T) == 2) {
    const int64_t each = a.rows / a.n;  // rows of a worker
    if (direct && each >= 192 && tiles(256, 256) >= 128) return launch_tiles<P, T, TC, 256, 256, 2, 4>(a, direct, stream);
    if (direct && (P == kGradWeight || each >= 96) && tiles(128, 128) >= 256) return launch_tiles<P, T, TC, 128, 128, 2, 2>(a, direct, stream);
    if (tiles(64, 128) >= 256) return launch_tiles<P, T, TC, 64, 128, 2, 2>(a, direct, stream);
  }
  return launch_tiles<P, T, TC, 64, 64, 2, 2>(a, direct, stream);
}

// Tiles go straight to LDS where every 16-byte piece is aligned and the rows of a step are within a buffer's offsets.
bool on_pieces(const void *p, int64_t pitch, size_t elem) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && pitch * int64_t(elem) % 16 == 0 && 256 * pitch * int64_t(elem) < kBufferMax;
}

}  // namespace

int launch_linear(const Shape &s, const void *W, int64_t offset, bool bf16, const void *A, int64_t lda, const int32_t *rows, int M, int in,
                  int out, bool relu, void *Y, int64_t ldy, bool y_bf16, void *stream) {
  const size_t e = bf16 ? 2 : 4;
  LinearArgs a{static_cast<const char *>(W) + offset * e, A, nullptr, Y, rows, s.ld, lda, 0, ldy, s.n, M, in, out, relu};
  const bool direct = on_pieces(a.w, in, e) && s.ld * e % 16 == 0 && on_pieces(A, lda, e);
  if (!bf16) return launch_product<kForward, float, float>(a, direct, stream);
  return y_bf16 ? launch_product<kForward, bf16_t, bf16_t>(a, direct, stream) : launch_product<kForward, bf16_t, float>(a, direct, stream);
}

int launch_linear_grad_input(const Shape &s, const void *W, int64_t offset, bool bf16, const void *dY, int64_t ldy, const int32_t *rows, int M,
                             int in, int out, const void *H, int64_t ldh, void *dA, int64_t lda, void *stream) {
  const size_t e = bf16 ? 2 : 4;
  LinearArgs a{static_cast<const char *>(W) + offset * e, dY, H, dA, rows, s.ld, ldy, ldh, lda, s.n, M, in, out, 0};
  const bool direct = on_pieces(a.w, in, e) && s.ld * e % 16 == 0 && on_pieces(dY, ldy, e) && out * e % 16 == 0;
  return bf16 ? launch_product<kGradInput, bf16_t, bf16_t>(a, direct, stream) : launch_product<kGradInput, float, float>(a, direct, stream);
}

int launch_linear_grad_weight(const Shape &s, bool bf16, const void *dY, int64_t ldy, const void *A, int64_t lda, const int32_t *rows, int M, int in,
                              int out, float *G, int64_t offset, bool accumulate, void *stream) {
  const size_t e = bf16 ? 2 : 4;
  LinearArgs a{nullptr, dY, A, G + offset, rows, s.ld, ldy, lda, 0, s.n, M, in, out, accumulate};
  const bool direct = on_pieces(dY, ldy, e) && on_pieces(A, lda, e);
  return bf16 ? launch_product<kGradWeight, bf16_t, float>(a, direct, stream) : launch_product<kGradWeight, float, float>(a, direct, stream);
}

}  // namespace detag

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

constexpr int kStepBytes = 128;  // of the contraction, per LDS step
constexpr int kPieces = kStepBytes / 16;
constexpr int kXcds = 8;
constexpr int64_t kBufferMax = int64_t(1) << 31;  // bytes a buffer resource is made for at most

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

// Which worker the row tile number `tile` (of BM rows each, counted worker by worker) belongs to, and how many there are in all.
// Every wavefront looks for itself: 64 workers at a time, a scan over the lanes.
struct RowTile {
  int worker, first, count;  // first row, rows of the tile (0: no such tile)
};
template <int BM>
__device__ __forceinline__ int count_row_tiles(const LinearArgs &a) {
  const int lane = threadIdx.x & 63;
  int total = 0;
  for (int base = 0; base < a.n; base += 64) {
    int lo = 0, hi = 0;
    if (base + lane < a.n) worker_rows(a, base + lane, lo, hi);
    int t = (hi - lo + BM - 1) / BM;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) t += __shfl_xor(t, d);
    total += t;
  }
  return total;
}
template <int BM>
__device__ __forceinline__ RowTile find_row_tile(const LinearArgs &a, int tile) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int base = 0; base < a.n; base += 64) {
    int lo = 0, hi = 0;
    if (base + lane < a.n) worker_rows(a, base + lane, lo, hi);
    const int t = (hi - lo + BM - 1) / BM;
    int upto = t;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int v = __shfl_up(upto, d);
      if (lane >= d) upto += v;
    }
    const unsigned long long holds = __ballot(before + upto > tile);
    if (holds) {
      const int src = __ffsll(holds) - 1;
      const int first = before + __shfl(upto, src) - __shfl(t, src);
      const int r0 = __shfl(lo, src) + (tile - first) * BM, left = __shfl(hi, src) - r0;
      return {base + src, __builtin_amdgcn_readfirstlane(r0), __builtin_amdgcn_readfirstlane(left < BM ? left : BM)};
    }
    before += __shfl(upto, 63);
  }
  return {0, 0, 0};
}

// One operand of a tile: ROWS of its own index by one step of the contraction.
//   kAlong : base at (first row, k = 0); `valid` rows, `contracted` elements in each
//   kAcross: base at (k = 0, first column); `valid` columns
template <class T, Layout L, int ROWS, int THREADS, bool Mixed, bool Direct>
struct Operand {
  static constexpr int kElems = 16 / sizeof(T);               // elements of a piece
  static constexpr int kSteps = kStepBytes / sizeof(T);       // contracted elements of a step
  static constexpr int kTileBytes = ROWS * kStepBytes;
  static constexpr int kLoads = ROWS * kPieces / THREADS;     // pieces a thread moves per step
  static constexpr int kRowPieces = L == kAlong ? kPieces : ROWS / kElems;
  static_assert(kLoads * THREADS == ROWS * kPieces, "the threads share the pieces evenly");

  const char *base;
  int64_t pitch;  // bytes
  int valid, contracted;
  uint32_t off[Direct ? kLoads : 1];
  u32x4 held[Direct ? 1 : kLoads];

  // Which position of an LDS row a piece is kept at.
  __device__ static __forceinline__ int spread(int row) {
    if constexpr (L == kAlong) return Mixed ? (row & 3) | ((row >> 4) & 1) << 2 : row & 7;
    else if constexpr (sizeof(T) == 2) return (((row & 3) << 1) | ((row >> 3) & 1) << 3) & (kRowPieces - 1);
    else return (((row >> 2) & 3) << 2) & (kRowPieces - 1);
  }

  __device__ __forceinline__ void place(int it, int &row, int &piece) const {
    const int id = it * THREADS + threadIdx.x;
    row = id / kRowPieces, piece = (id % kRowPieces) ^ spread(row);
  }

  __device__ __forceinline__ void init(const void *b, int64_t pitch_elems, int valid_, int contracted_) {
    base = static_cast<const char *>(b), pitch = pitch_elems * int64_t(sizeof(T)), valid = valid_, contracted = contracted_;
    if constexpr (Direct) {
#pragma unroll
      for (int it = 0; it < kLoads; ++it) {
        int row, piece;
        place(it, row, piece);
        off[it] = uint32_t(row * pitch) + 16u * piece;
      }
    }
  }

  // Bytes from `base` on that belong to the operand.
  __device__ __forceinline__ int64_t extent() const {
    return L == kAlong ? (valid - 1) * pitch + contracted * int64_t(sizeof(T)) : (contracted - 1) * pitch + valid * int64_t(sizeof(T));
  }

  // Requests step `kt` (directly into `lds`, or into registers).
  __device__ __forceinline__ void request(int kt, lds_char *lds) {
    if constexpr (Direct) {
      const int64_t skip = L == kAlong ? int64_t(kt) * kStepBytes : int64_t(kt) * kSteps * pitch;
      const int left = (contracted - kt * kSteps) * int(sizeof(T));  // kAlong: bytes of a row that are left
      // what is left of the operand, as far as a buffer counts (a step's offsets stay below that)
      const int64_t bytes = extent() - skip;
      const rsrc_t r = make_rsrc(base + skip, bytes < kBufferMax ? uint32_t(bytes) : uint32_t(kBufferMax));
      const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
      for (int it = 0; it < kLoads; ++it) {
        uint32_t o = off[it];
        if constexpr (L == kAlong)
          if (left < kStepBytes) {  // uniform: the last step
            int row, piece;
            place(it, row, piece);
            if (16 * piece >= left) o = 0xffffff00u;
          }
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)(lds + (it * THREADS + wave * 64) * 16), 16,
                                                 int(o), 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int it = 0; it < kLoads; ++it) {
        int row, piece;
        place(it, row, piece);
        const int k = kt * kSteps + (L == kAlong ? piece * kElems : row), x = L == kAlong ? row : piece * kElems;
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
  }

  // Writes what request() left in registers.
  __device__ __forceinline__ void deliver(lds_char *lds) {
    if constexpr (!Direct) {
#pragma unroll
      for (int it = 0; it < kLoads; ++it)
        *reinterpret_cast<__attribute__((address_space(3))) u32x4 *>(lds + (it * THREADS + threadIdx.x) * 16) = held[it];
    }
  }

  // Lane's 16 bytes of fragment f (16 of the operand's index from `first` on), part s of a step.  Mixed: index p of fragment f stands
  // for 16*(p/4) + 4f + p%4, so that the four fragments of a wavefront give a lane 16 neighbours.
  __device__ __forceinline__ static u32x4 fragment(const lds_char *lds, int first, int f, int s) {
    const int lane = threadIdx.x & 63, p = lane & 15, q = lane >> 4;
    if constexpr (L == kAlong) {
      const int row = Mixed ? first + 16 * (p >> 2) + 4 * f + (p & 3) : first + 16 * f + p;
      return *reinterpret_cast<const __attribute__((address_space(3))) u32x4 *>(lds + row * kStepBytes + (((4 * s + q) ^ spread(row)) << 4));
    } else if constexpr (sizeof(T) == 2) {
      const int col = first + 16 * f + 4 * (p & 3), k = 32 * s + 8 * q + (p >> 2);
      auto read = [&](int row) {
        return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(
                                             lds + row * (ROWS * 2) + (((col >> 3) ^ spread(row)) << 4) + (col & 4) * 2)));
      };
      const u32x2 a = read(k), b = read(k + 4);
      return u32x4{a[0], a[1], b[0], b[1]};
    } else {
      const int col = first + 16 * f + p;
      u32x4 v;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int k = 16 * s + 4 * q + t;
        v[t] = *reinterpret_cast<const __attribute__((address_space(3))) uint32_t *>(lds + k * (ROWS * 4) + (((col >> 2) ^ spread(k)) << 4) +
                                                                                    (col & 3) * 4);
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

template <Product P, class T, class TC, int BM, int BN, int WM, int WN, bool Direct>
__global__ __launch_bounds__(64 * WM * WN) void linear_tile_kernel(LinearArgs a) {
  constexpr int kThreads = 64 * WM * WN, kFm = BM / WM / 16, kFn = BN / WN / 16;
  constexpr Layout kRowLayout = P == kGradWeight ? kAcross : kAlong, kColLayout = P == kForward ? kAlong : kAcross;
  constexpr bool kMixed = P == kForward && kFn == 4;
  using Rows = Operand<T, kRowLayout, BM, kThreads, false, Direct>;
  using Cols = Operand<T, kColLayout, BN, kThreads, kMixed, Direct>;
  __shared__ __attribute__((aligned(128))) char lds_[2 * (Rows::kTileBytes + Cols::kTileBytes)];
  lds_char *const lds = (lds_char *)lds_;
  constexpr int kBuffer = Rows::kTileBytes + Cols::kTileBytes;

  const int columns = P == kForward ? a.out : a.in, col_tiles = (columns + BN - 1) / BN;
  const int row_tiles = P == kGradWeight ? (a.out + BM - 1) / BM * a.n : count_row_tiles<BM>(a);
  const int64_t tiles = int64_t(row_tiles) * col_tiles;
  // workgroups go to the eight XCDs in turn: each XCD takes a run of neighbouring tiles
  const int64_t share = (tiles + kXcds - 1) / kXcds;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, p = lane & 15, q = lane >> 4;
  const int row0 = wave / WN * (BM / WM), col0 = wave % WN * (BN / WN);

  for (int64_t at = blockIdx.x; at < kXcds * share; at += gridDim.x) {
    const int64_t number = at % kXcds * share + at / kXcds;
    if (at / kXcds >= share || number >= tiles) continue;
    const int row_tile = int(number / col_tiles), column = int(number % col_tiles) * BN;
    int worker, first, count, contracted;
    if constexpr (P == kGradWeight) {
      const int per = (a.out + BM - 1) / BM;
      worker = row_tile / per, first = row_tile % per * BM, count = a.out - first < BM ? a.out - first : BM;
    } else {
      const RowTile t = find_row_tile<BM>(a, row_tile);
      worker = t.worker, first = t.first, count = t.count, contracted = P == kForward ? a.in : a.out;
    }
    if (count <= 0) continue;
    worker = __builtin_amdgcn_readfirstlane(worker);
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
      int lo, hi;
      worker_rows(a, worker, lo, hi);
      lo = __builtin_amdgcn_readfirstlane(lo), contracted = __builtin_amdgcn_readfirstlane(hi) - lo;
      rows.init(static_cast<const T *>(a.rows_a) + int64_t(lo) * a.lda + first, a.lda, count, contracted);
      cols.init(static_cast<const T *>(a.rows_b) + int64_t(lo) * a.ldb + column, a.ldb, width, contracted);
    }

    f32x4 acc[kFm][kFn];
#pragma unroll
    for (int i = 0; i < kFm; ++i)
#pragma unroll
      for (int j = 0; j < kFn; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    const int steps = (contracted + Rows::kSteps - 1) / Rows::kSteps;
    __syncthreads();  // the tile before is done with the buffers
    if (steps > 0) {
      rows.request(0, lds), cols.request(0, lds + Rows::kTileBytes);
      rows.deliver(lds), cols.deliver(lds + Rows::kTileBytes);
    }
    for (int kt = 0; kt < steps; ++kt) {
      lds_char *const now = lds + (kt & 1) * kBuffer, *const next = lds + (~kt & 1) * kBuffer;
      __syncthreads();  // step kt has arrived, and nobody reads `next` any more
      if (kt + 1 < steps) rows.request(kt + 1, next), cols.request(kt + 1, next + Rows::kTileBytes);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        u32x4 x[kFn], y[kFm];
#pragma unroll
        for (int j = 0; j < kFn; ++j) x[j] = Cols::fragment(now + Rows::kTileBytes, col0, j, s);
#pragma unroll
        for (int i = 0; i < kFm; ++i) y[i] = Rows::fragment(now, row0, i, s);
#pragma unroll
        for (int i = 0; i < kFm; ++i)
#pragma unroll
          for (int j = 0; j < kFn; ++j) acc[i][j] = multiply<T>(x[j], y[i], acc[i][j]);
      }
      if (kt + 1 < steps) rows.deliver(next), cols.deliver(next + Rows::kTileBytes);
    }

#pragma unroll
    for (int i = 0; i < kFm; ++i) {
      const int r = row0 + 16 * i + p;
      if (r >= count) continue;
      TC *crow = static_cast<TC *>(a.c) + (P == kGradWeight ? int64_t(worker) * a.ld + int64_t(first + r) * a.in : int64_t(first + r) * a.ldc);
#pragma unroll
      for (int j = 0; j < kFn; ++j) {
        const int c = column + col0 + (kMixed ? 16 * q + 4 * j : 16 * j + 4 * q), inside = columns - c;
        f32x4 v = acc[i][j];
        if constexpr (P == kForward) {
          if (a.flag)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = v[e] <= 0.f ? 0.f : v[e];  // NaN stays
        } else if constexpr (P == kGradInput) {
          if (a.rows_b) {
            const T *h = static_cast<const T *>(a.rows_b) + int64_t(first + r) * a.ldb + c;
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (e < inside) v[e] = to_f32(h[e]) > 0.f ? v[e] : 0.f;
          }
        } else if (a.flag) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e < inside) v[e] += to_f32(crow[c + e]);
        }
        store4(crow + c, v, inside);
      }
    }
  }
}

template <Product P, class T, class TC, int BM, int BN, int WM, int WN>
int launch_tiles(const LinearArgs &a, bool direct, void *stream) {
  const int64_t col_tiles = ceil_div_i64(P == kForward ? a.out : a.in, BN);
  const int64_t row_tiles = P == kGradWeight ? int64_t(ceil_div_i64(a.out, BM)) * a.n : int64_t(a.rows) / BM + (a.n < a.rows ? a.n : a.rows);
  int64_t blocks = (row_tiles * col_tiles + kXcds - 1) / kXcds * kXcds;
  if (blocks > 1 << 20) blocks = 1 << 20;
  if (blocks == 0) return 0;
  if (direct) linear_tile_kernel<P, T, TC, BM, BN, WM, WN, true><<<dim3(uint32_t(blocks)), 64 * WM * WN, 0, static_cast<hipStream_t>(stream)>>>(a);
  else linear_tile_kernel<P, T, TC, BM, BN, WM, WN, false><<<dim3(uint32_t(blocks)), 64 * WM * WN, 0, static_cast<hipStream_t>(stream)>>>(a);
  return hip_rc(hipGetLastError());
}

template <Product P, class T, class TC>
int launch_product(const LinearArgs &a, bool direct, void *stream) {
  return launch_tiles<P, T, TC, 128, 128, 2, 2>(a, direct, stream);
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

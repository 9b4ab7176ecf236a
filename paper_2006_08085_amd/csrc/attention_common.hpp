// What the attention kernels share (k_attention.hip, k_attention_grad.hip): panels of rows in LDS, their fragments, and the order of work.
//
// The matrix products run on v_mfma_f32_32x32x16_bf16 or v_mfma_f32_32x32x2_f32.  Lane l, p = l % 32, h = l / 32: an operand holds
// index p and eight (fp32: one) contracted indices from 8h (h) on; register r of the result is (index 8(r/4) + 4h + r%4 of the first
// operand, p of the second).  The second operand's index is always the one that belongs to the wavefront (its queries, or
// its keys): a lane then holds one of them, with 16 of the panel's rows in its registers, and the statistics of a row of scores need one
// exchange between the two halves.  The products that follow contract the panel's rows: a lane's registers 8g .. 8g+7 are rows
// 16g + 4h + (0..3) and 16g + 8 + 4h + (0..3), which is as good an order of a contraction as any other, so they become an operand as
// they are, and the other one is read from LDS in that order: no value changes its lane.
#pragma once

#include "detag_internal.h"
#include "dev_common.hpp"
#include "linear_common.hpp"
#include "rows_common.hpp"

namespace detag {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kLn2 = 0.6931471805599453f;

// 16 bytes of both operands.
template <class T>
__device__ __forceinline__ f32x16 multiply32(u32x4 x, u32x4 y, f32x16 acc) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), acc, 0, 0, 0);
  } else {
#pragma unroll
    for (int t = 0; t < 4; ++t)
      acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(x[t]), __uint_as_float(y[t]), acc, 0, 0, 0);
    return acc;
  }
}

__device__ __forceinline__ float other_half(float v) {  // the value of the lane 32 away
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(threadIdx.x & 32 ? r[0] : r[1]);
}

// ROWS rows of a matrix, WIDTH columns each (those past the matrix's own are zeros, as are rows past the part's last), in LDS.
template <class T, int WIDTH, int ROWS, int THREADS, bool Direct>
struct Panel {
  static constexpr int kElems = 16 / sizeof(T), kPieces = WIDTH / kElems, kRowBytes = WIDTH * sizeof(T), kBytes = ROWS * kRowBytes;
  static constexpr int kLoads = ROWS * kPieces / THREADS, kRowsApart = THREADS / kPieces;
  static constexpr int kSteps = kPieces / 2;  // of the contraction over columns, 16 bytes a lane each
  static constexpr int kBlocks = WIDTH / 32;  // of columns
  static_assert(kLoads * THREADS == ROWS * kPieces && kRowsApart % 8 == 0, "the threads share the pieces evenly, and spread() repeats");

  const char *base;  // the part's first row
  int64_t pitch;     // bytes
  int width;         // columns of the matrix
  uint32_t off;
  u32x4 held[Direct ? 1 : kLoads];

  // Bits that are xor-ed to a piece's position: eight rows that are read together at one column lie in eight places, and so do
  // the 32 bytes of four rows that a transposing read takes.
  __device__ static __forceinline__ int spread(int row) { return (row & 3) << 1 | (row >> 2 & 1); }

  __device__ __forceinline__ void init(const void *first, int64_t pitch_elems, int width_) {
    base = static_cast<const char *>(first), pitch = pitch_elems * int64_t(sizeof(T)), width = width_;
    const int row = threadIdx.x / kPieces, piece = threadIdx.x % kPieces ^ spread(row);
    off = Direct ? (piece * kElems < width ? uint32_t(row * pitch) + 16u * piece : 0xffffff00u) : 0u;
  }

  // Requests rows `at` .. of the part, which has `rows`; deliver() (not Direct) writes them.
  __device__ __forceinline__ void request(int at, int rows, uint32_t lds) {
    if constexpr (Direct) {
      const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
      for (int it = 0; it < kLoads; ++it) {
        const int first = at + it * kRowsApart;
        const int64_t left = rows > first ? (rows - first - 1) * pitch + width * int64_t(sizeof(T)) : 0;
        const uint64_t from = reinterpret_cast<uint64_t>(base) + first * pitch;
        const u32x4 r = {uint32_t(from), uint32_t(from >> 32), uint32_t(left < kBufferMax ? left : kBufferMax), 0x00020000u};
        load_to_lds(r, off, lds + (it * THREADS + wave * 64) * 16);
      }
    } else {
      const int row = threadIdx.x / kPieces, piece = threadIdx.x % kPieces ^ spread(row);
#pragma unroll
      for (int it = 0; it < kLoads; ++it) {
        const int r = at + it * kRowsApart + row;
        held[it] = load_piece(reinterpret_cast<const T *>(base + r * pitch) + piece * kElems, r < rows ? width - piece * kElems : 0);
      }
    }
  }
  __device__ __forceinline__ void deliver(uint32_t lds) const {
    if constexpr (!Direct) {
#pragma unroll
      for (int it = 0; it < kLoads; ++it)
        *reinterpret_cast<__attribute__((address_space(3))) u32x4 *>(lds + (it * THREADS + threadIdx.x) * 16) = held[it];
    }
  }

  // Where a lane reads.  along: its 16 bytes of row p, contraction step 0; across: see below.
  __device__ static __forceinline__ uint32_t along_base() {
    const int p = threadIdx.x & 31, h = threadIdx.x >> 5 & 1;
    return p * kRowBytes + ((h ^ spread(p)) << 4);
  }
  // Rows 32 * block + p, step s of the columns.
  __device__ static __forceinline__ u32x4 along(uint32_t base, uint32_t lds, int block, int s) {
    return read_lds<u32x4>((base ^ (2 * s % 8) << 4) + lds + block * 32 * kRowBytes + (2 * s / 8) * 128);
  }

  // Columns 32 * block + p as the index, rows as what is contracted, in the order of a result's registers: 16 rows from 16 g on (bf16: one
  // product) or rows 8 g + 4 h + t (fp32: product t of four).
  __device__ static __forceinline__ uint32_t across_base() {
    const int lane = threadIdx.x & 63, h = lane >> 5;
    if constexpr (sizeof(T) == 2) {
      const int i = lane & 15, row = 4 * h + (i >> 2), piece = 2 * (lane >> 4 & 1) + (i >> 1 & 1);
      return row * kRowBytes + ((piece ^ spread(row)) << 4) + (i & 1) * 8;
    } else {
      const int p = lane & 31;
      return 4 * h * kRowBytes + (((p >> 2) ^ spread(4 * h)) << 4) + (p & 3) * 4;
    }
  }
  static constexpr int kGroups = sizeof(T) == 2 ? 2 : 4;  // of the 16 registers of a result
  __device__ static __forceinline__ u32x4 across(uint32_t base, uint32_t lds, int block, int row0, int g) {
    if constexpr (sizeof(T) == 2) {
      const uint32_t at = (base ^ (block & 1) << 6) + lds + (block >> 1) * 128 + (row0 + 16 * g) * kRowBytes;
      auto read = [&](uint32_t a) {
        return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) s16x4 *>(a)));
      };
      const u32x2 lo = read(at), hi = read(at + 8 * kRowBytes);
      return u32x4{lo[0], lo[1], hi[0], hi[1]};
    } else {
      u32x4 v;
#pragma unroll
      for (int t = 0; t < 4; ++t) v[t] = read_lds<uint32_t>((base ^ (t << 1) << 4) + lds + block * 128 + (row0 + 8 * g + t) * kRowBytes);
      return v;
    }
  }
};

// Registers of group g of a result (probabilities, or their gradients) as the second operand of the next product.
template <class T>
__device__ __forceinline__ u32x4 as_operand(const f32x16 &s, int g) {
  u32x4 v;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if constexpr (sizeof(T) == 2) v[w] = uint32_t(bf16_bits_rne(s[8 * g + 2 * w])) | uint32_t(bf16_bits_rne(s[8 * g + 2 * w + 1])) << 16;
    else v[w] = __float_as_uint(s[4 * g + w]);
  }
  return v;
}

// A lane's pieces of row `row` of a matrix as the second operand of a product over columns: step s holds 16 bytes from piece 2s + h on.
// Zeros where the row is not `there`.
template <class T, int STEPS>
__device__ __forceinline__ void load_operand(u32x4 (&x)[STEPS], const T *first, int64_t pitch, int64_t row, bool there, int width) {
  constexpr int kElems = 16 / sizeof(T);
  const int h = threadIdx.x >> 5 & 1;
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    const int c = (2 * s + h) * kElems;
    x[s] = load_piece(first + row * pitch + c, there ? width - c : 0);
  }
}

// Writes a wavefront's result transposed: register r of block b of `acc` is column 32 b + 8 (r/4) + 4 h + r%4 of the lane's row.
template <class T, int BLOCKS>
__device__ __forceinline__ void store_row(T *row, const f32x16 (&acc)[BLOCKS], float factor, int width) {
  const int h = threadIdx.x >> 5 & 1;
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const int c = 32 * b + 2 * r + 4 * h;
      if (c < width) store4(row + c, f32x4{acc[b][r] * factor, acc[b][r + 1] * factor, acc[b][r + 2] * factor, acc[b][r + 3] * factor}, width - c);
    }
}

// Which head and which run of rows a block works on.  Workgroups go to the eight XCDs in turn, each with an L2 of its own: those that
// read the same keys and values (the runs and query heads of a key head) share as few XCDs as divide the key heads evenly, and where
// several XCDs share a key head they take its runs in turn.
struct Work {
  int kv, run, group;  // run: -1: none
};
constexpr int kXcds = 8;
__host__ __device__ inline int xcds_apart(int kv_heads) { return kv_heads % 8 == 0 ? 8 : kv_heads % 4 == 0 ? 4 : kv_heads % 2 == 0 ? 2 : 1; }
// Blocks that work_of() needs: `each` pieces of work of every key head.
__host__ __device__ inline int64_t attention_blocks(int kv_heads, int64_t each) {
  const int apart = xcds_apart(kv_heads), share = kXcds / apart;
  return (each + share - 1) / share * (kv_heads / apart) * kXcds;
}
__device__ __forceinline__ Work work_of(int64_t block, int kv_heads, int64_t runs, int groups) {
  const int apart = xcds_apart(kv_heads), share = kXcds / apart;
  const int64_t each = runs * groups, turns = (each + share - 1) / share;
  const int xcd = int(block % kXcds);
  const int64_t turn = block / kXcds, kv = turn / turns, at = (turn - kv * turns) * share + xcd / apart;
  if (kv >= kv_heads / apart || at >= each) return {0, -1, 0};
  return {int(kv) * apart + xcd % apart, int(at / groups), int(at % groups)};
}

// Whether panels go straight from memory to LDS: whole pieces in rows that start on whole dwords, and offsets that a buffer counts.
inline bool panels_direct(const void *p, int64_t pitch, int width, size_t elem) {
  return reinterpret_cast<uintptr_t>(p) % 4 == 0 && pitch * int64_t(elem) % 4 == 0 && width * int(elem) % 16 == 0 && 64 * pitch * int64_t(elem) < kBufferMax;
}

}  // namespace detag

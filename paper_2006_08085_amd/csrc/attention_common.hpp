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

// ROWS rows of a part of a matrix, WIDTH columns each (those past the matrix's own are zeros, as are rows past the part's last), in LDS.
template <class T, int WIDTH, int ROWS, int THREADS, bool Direct>
struct Panel {
  static constexpr int kElems = 16 / sizeof(T), kPieces = WIDTH / kElems, kRowBytes = WIDTH * sizeof(T), kBytes = ROWS * kRowBytes;
  static constexpr int kLoads = ROWS * kPieces / THREADS, kRowsApart = THREADS / kPieces;
  static constexpr int kSteps = kPieces / 2;  // of the contraction over columns, 16 bytes a lane each
  static constexpr int kBlocks = WIDTH / 32;  // of columns
  static constexpr int kOffsets = kRowsApart % 16 == 0 ? 1 : 16 / kRowsApart;  // spread() repeats after 16 rows
  static_assert(kLoads * THREADS == ROWS * kPieces && (kRowsApart % 16 == 0 || 16 % kRowsApart == 0), "the threads share the pieces evenly");

  // THREADS move a panel's pieces: the block, or a part of its wavefronts.
  __device__ static __forceinline__ int thread() { return threadIdx.x % THREADS; }

  uint64_t from;  // the next panel's first row
  int64_t left;   // bytes of the part from there on
  int64_t pitch;  // bytes
  int width;      // columns of the matrix
  uint32_t off[Direct ? kOffsets : 1];
  u32x4 held[Direct ? 1 : kLoads];

  // Bits that are xor-ed to a piece's position.  LDS has 64 banks, 256 bytes: 16 lanes that read 16 bytes of as many rows at one column
  // find them in 16 places, and so do the 32 lanes of a transposing read, which take 64 bytes of four rows.  Rows of 128 bytes
  // share 256 in pairs.
  __device__ static __forceinline__ int spread(int row) {
    return kRowBytes == 128 ? (row >> 1 & 1) << 2 | (row >> 2 & 3) : (row & 3) << 2 | (row >> 2 & 3);
  }

  // first: the part's first row, of `rows`
  __device__ __forceinline__ void init(const T *first, int64_t pitch_elems, int width_, int rows) {
    pitch = pitch_elems * int64_t(sizeof(T)), width = width_;
    from = reinterpret_cast<uint64_t>(first), left = (rows - 1) * pitch + width * int64_t(sizeof(T));
    if constexpr (Direct) {
#pragma unroll
      for (int k = 0; k < kOffsets; ++k) {
        const int row = thread() / kPieces, piece = thread() % kPieces ^ spread(row + k * kRowsApart);
        off[k] = piece * kElems < width ? uint32_t(row * pitch) + 16u * piece : 0xffffff00u;
      }
    }
  }
  __device__ __forceinline__ void skip(int rows) { from += rows * pitch, left -= rows * pitch; }

  // Requests the next panel; deliver() (not Direct) writes it.
  __device__ __forceinline__ void request(uint32_t lds) {
    if constexpr (Direct) {
      const int wave = __builtin_amdgcn_readfirstlane(thread() >> 6), apart = kRowsApart * int(pitch);
      int now = left < 0 ? 0 : left < kBufferMax ? int(left) : int(kBufferMax);
      uint64_t at = from;
#pragma unroll
      for (int it = 0; it < kLoads; ++it) {
        const u32x4 r = {uint32_t(at), uint32_t(at >> 32), uint32_t(now), 0x00020000u};
        load_to_lds(r, off[it % kOffsets], lds + (it * THREADS + wave * 64) * 16);
        at += uint32_t(apart), now = now > apart ? now - apart : 0;
      }
    } else {
#pragma unroll
      for (int it = 0; it < kLoads; ++it) {
        const int row = it * kRowsApart + thread() / kPieces, piece = thread() % kPieces ^ spread(row);
        held[it] = load_piece(reinterpret_cast<const T *>(from + row * pitch) + piece * kElems, row * pitch < left ? width - piece * kElems : 0);
      }
    }
    skip(ROWS);
  }
  __device__ __forceinline__ void deliver(uint32_t lds) const {
    if constexpr (!Direct) {
#pragma unroll
      for (int it = 0; it < kLoads; ++it)
        *reinterpret_cast<__attribute__((address_space(3))) u32x4 *>(lds + (it * THREADS + thread()) * 16) = held[it];
    }
  }

  // Where a lane reads.  along: its 16 bytes of row p, contraction step 0; across: see below.
  __device__ static __forceinline__ uint32_t along_base() {
    const int p = threadIdx.x & 31, h = threadIdx.x >> 5 & 1;
    return p * kRowBytes + ((h ^ spread(p)) << 4);
  }
  // Rows 32 * block + p, step s of the columns.
  __device__ static __forceinline__ u32x4 along(uint32_t base, uint32_t lds, int block, int s) {
    return read_lds<u32x4>((base ^ (2 * s % 16) << 4) + lds + block * 32 * kRowBytes + 2 * s / 16 * 256);
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
      auto read = [&](uint32_t a) {
        return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) s16x4 *>(a)));
      };
      // eight rows further on the third bit of the row has turned
      const uint32_t at = base ^ block << 6, rows = lds + (row0 + 16 * g) * kRowBytes;
      const u32x2 lo = read(at + rows), hi = read((at ^ 32) + rows + 8 * kRowBytes);
      return u32x4{lo[0], lo[1], hi[0], hi[1]};
    } else {
      u32x4 v;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const uint32_t at = base ^ (t << 2 | (g & 1) << 1) << 4 ^ (block & 1) << 7;
        v[t] = read_lds<uint32_t>(at + lds + block / 2 * 256 + (row0 + 8 * g + t) * kRowBytes);
      }
      return v;
    }
  }
};

// A float for every lane from a buffer into LDS, the wavefront's 256 bytes from `lds` on; zeros out of the buffer's range.
__device__ __forceinline__ void load_floats_to_lds(u32x4 resource, uint32_t lds) {
  const uint32_t offset = (threadIdx.x & 63) * 4;
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(offset), "s"(resource), "s"(lds) : "memory", "m0");
}

// Registers of group g of a result (probabilities, or their gradients) as the second operand of the next product.
template <class T>
__device__ __forceinline__ u32x4 as_operand(const f32x16 &s, int g) {
  u32x4 v;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if constexpr (sizeof(T) == 2) v[w] = bf16_pair(s[8 * g + 2 * w], s[8 * g + 2 * w + 1]);
    else v[w] = __float_as_uint(s[4 * g + w]);
  }
  return v;
}

// A lane's pieces of row `row`, counted from `first` on, of a matrix as the second operand of a product over columns: step s holds 16 bytes from
// piece 2s + h on.  Zeros where the row is not `there`.  Whole: panels_direct() of the matrix, and row < 256; no branches then.
template <class T, bool Whole, int STEPS>
__device__ __forceinline__ void load_operand(u32x4 (&x)[STEPS], const T *first, int64_t pitch, int row, bool there, int width) {
  constexpr int kElems = 16 / sizeof(T);
  constexpr uint32_t kNowhere = 0xf0000000u;
  const int h = threadIdx.x >> 5 & 1;
  if constexpr (Whole) {
    asm volatile("" : "+v"(row));  // (as in store_rows)
    const auto from = make_rsrc(first, uint32_t(kBufferMax));
    const uint32_t at = uint32_t(row) * uint32_t(pitch * int64_t(sizeof(T)));
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int c = (2 * s + h) * kElems;
      x[s] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(from, int(there && c < width ? at + c * uint32_t(sizeof(T)) : kNowhere), 0, 0));
    }
  } else {
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int c = (2 * s + h) * kElems;
      x[s] = load_piece(first + row * pitch + c, there ? width - c : 0);
    }
  }
}

// Writes a wavefront's result transposed: register r of block b of `acc` is column 32 b + 8 (r/4) + 4 h + r%4 of the lane's row.
template <class T, int BLOCKS>
__device__ __forceinline__ void store_row(T *row, const f32x16 (&acc)[BLOCKS], float factor, int width) {
  const int h = threadIdx.x >> 5 & 1;
  asm volatile("" : "+s"(width));  // what follows is not to be worked out ahead, where it would hold registers
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const int c = 32 * b + 2 * r + 4 * h;
      if (c < width) store4(row + c, f32x4{acc[b][r] * factor, acc[b][r + 1] * factor, acc[b][r + 2] * factor, acc[b][r + 3] * factor}, width - c);
    }
}

// The same for a matrix of whole pieces: the wavefront's rows pass through 32 rows of LDS of its own (of nobody else's until all are
// done), so that whole rows are written.  first: of the wavefront's rows, `rows` of which are there.
template <class T, int BLOCKS>
__device__ __forceinline__ void store_rows(T *first, int64_t pitch, int rows, uint32_t lds, const f32x16 (&acc)[BLOCKS], float factor, int width) {
  using Rows = Panel<T, 32 * BLOCKS, 32, 64, true>;
  constexpr int kElems = Rows::kElems;
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));  // what follows is not to be worked out ahead, where it would hold registers
  const int p = lane & 31, h = lane >> 5;
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const int c = 32 * b + 2 * r;  // and 4 h
      const f32x4 v = {acc[b][r] * factor, acc[b][r + 1] * factor, acc[b][r + 2] * factor, acc[b][r + 3] * factor};
      const uint32_t row = lds + p * Rows::kRowBytes;
      if constexpr (sizeof(T) == 2)
        *reinterpret_cast<__attribute__((address_space(3))) u32x2 *>(row + ((c / kElems ^ Rows::spread(p)) << 4) + 8 * h) =
            u32x2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
      else
        *reinterpret_cast<__attribute__((address_space(3))) f32x4 *>(row + (((c / kElems + h) ^ Rows::spread(p)) << 4)) = v;
    }
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int it = 0; it < Rows::kLoads; ++it) {
    const int row = it * Rows::kRowsApart + lane / Rows::kPieces, piece = lane % Rows::kPieces;
    const u32x4 v = *reinterpret_cast<__attribute__((address_space(3))) u32x4 *>(lds + row * Rows::kRowBytes + ((piece ^ Rows::spread(row)) << 4));
    if (row < rows && piece * kElems < width) *reinterpret_cast<u32x4_any *>(first + row * pitch + piece * kElems) = v;
  }
}

// Which key head a block works on, and which of its `each` pieces of work.  Workgroups go to the eight XCDs in turn, each with an L2 of its
// own: those that read the same keys and values (the runs and query heads of a key head) share as few XCDs as divide the key heads
// evenly, and where several XCDs share a key head they take its pieces in turn.  A grid of (8 turns, rounds) blocks, or a part of it: f(kv head,
// piece) for each.
constexpr int kXcds = 8;
struct WorkGrid {
  uint32_t turns, rounds, apart, each;
};
inline WorkGrid work_grid(int kv_heads, int64_t each) {
  const int apart = kv_heads % 8 == 0 ? 8 : kv_heads % 4 == 0 ? 4 : kv_heads % 2 == 0 ? 2 : 1;
  return {uint32_t(ceil_div_i64(each, kXcds / apart)), uint32_t(kv_heads / apart), uint32_t(apart), uint32_t(each)};
}
inline dim3 work_blocks(const WorkGrid &g) {
  return dim3(kXcds * (g.turns < 1u << 17 ? g.turns : 1u << 17), g.rounds < 4096 ? g.rounds : 4096);
}
template <class F>
__device__ __forceinline__ void for_work(const WorkGrid &g, F &&f) {
  for (uint32_t y = blockIdx.y; y < g.rounds; y += gridDim.y)
    for (uint32_t x = blockIdx.x; x < kXcds * g.turns; x += gridDim.x) {
      const uint32_t xcd = x % kXcds, piece = x / kXcds * (kXcds / g.apart) + xcd / g.apart;
      if (piece < g.each) f(int(y * g.apart + xcd % g.apart), piece);
    }
}

// Run number `turn` (of `turns`, some of which are none) of `high` rows.  Of up to 64 sequences those of more than twice the mean
// length come first, then those of more than it, so that no long walk starts when the others are done.  Backward: of a sequence its last run
// first, which sees the most keys in a causal call.
__device__ __forceinline__ Run run_in_turn(const AttentionArgs &a, int high, int turn, int turns, bool backward) {
  if (a.parts > 64) return run_of(a.offsets, a.parts, a.rows, high, backward ? turns - 1 - turn : turn);
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = -1;
  if (lane < a.parts) lo = within(a.offsets[lane], a.rows), hi = within(a.offsets[lane + 1], a.rows);
  const int length = hi - lo, runs = length > 0 ? (length - 1) / high + 1 : 0;
  const int mean = a.rows / a.parts, kind = length / 2 >= mean ? 0 : length > mean ? 1 : 2;
  int start = 0, before = 0;  // runs of the sequences that come before
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const int upto = wave_scan(kind == k ? runs : 0);
    if (kind == k) start = before + upto - runs;
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  const unsigned long long holds = __ballot(turn >= start && turn < start + runs);
  if (!holds) return {-1, 0, 0, 0};
  const int at = __builtin_amdgcn_readfirstlane(__ffsll(holds)) - 1;
  const int nth = turn - __builtin_amdgcn_readlane(start, at);
  Run r;
  r.lo = __builtin_amdgcn_readlane(lo, at), r.hi = __builtin_amdgcn_readlane(hi, at);
  r.part = at, r.first = r.lo + (backward ? __builtin_amdgcn_readlane(runs, at) - 1 - nth : nth) * high;
  return r;
}

// Whether a block's wavefronts share the keys of 32 queries instead of having 32 queries each: where blocks of 128 queries would be few, the
// longest walk over the keys is what takes the time.  Causal, microseconds (shared, not), forward and gradient.  bf16, 8 heads of 128: one sequence of
// 512 rows 11, 16 and 31, 41; of 2048 36, 48 and 86, 116; of 4096 114, 91 and 227, 237; 16 of 256 28, 13 and 66, 46.  fp32, 8 heads of 64: one of
// 2048 59, 162 and 259, 390; four of 1024 69, 86 and 257, 274; 16 heads of 128, 8 key heads, eight of 512 157, 167 and 586, 577.
inline bool attention_splits(const AttentionArgs &a, bool bf16) {
  return (int64_t(a.rows / 128) + a.parts / 2 + 1) * a.heads <= (bf16 ? 256 : 512);
}

// Whether panels go straight from memory to LDS: whole pieces in rows that start on whole dwords, and offsets that a buffer counts.
inline bool panels_direct(const void *p, int64_t pitch, int width, size_t elem) {
  return reinterpret_cast<uintptr_t>(p) % 4 == 0 && pitch * int64_t(elem) % 4 == 0 && width * int(elem) % 16 == 0 && 256 * pitch * int64_t(elem) < kBufferMax;
}

}  // namespace detag

// What the kernels of a layer's products share (k_linear.hip, k_linear_few.hip).
#pragma once

#include "dev_common.hpp"

namespace detag {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// pieces at any address their elements may have
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

struct LinearArgs {
  const void *w;       // n x ld weights, already at the layer's first column
  const void *rows_a;  // A, or dY for the input gradient
  const void *rows_b;  // weight gradient: A (rows_a is dY); input gradient: H or null
  void *c;             // Y, dA or G at the layer's first column
  const int32_t *offsets;
  int64_t ld, lda, ldb, ldc;  // pitches in elements: of w (and G), rows_a, rows_b, c
  int n, rows, in, out;
  int flag;  // forward: relu; weight gradient: accumulate; with an epilogue: what it reads may come through a buffer
  // calls with an epilogue (linear_epilogue.hpp)
  const void *bias = nullptr, *residual = nullptr;  // bias: at its first column of the n x ld matrix
  void *pre = nullptr;                              // what the activation is taken of; the input gradient's is rows_b
  int64_t ldr = 0, ldz = 0;
  int act = 0;
};

// A worker's rows, kept inside the row matrices whatever the offsets say.
__device__ __forceinline__ void worker_rows(const LinearArgs &a, int i, int &lo, int &hi) {
  lo = a.offsets[i], hi = a.offsets[i + 1];
  lo = lo < 0 ? 0 : lo > a.rows ? a.rows : lo;
  hi = hi < lo ? lo : hi > a.rows ? a.rows : hi;
}

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
      *reinterpret_cast<u32x2_any *>(p) = u32x2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
    } else {
      *reinterpret_cast<f32x4_any *>(p) = v;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < inside) p[e] = from_f32<T>(v[e]);
  }
}

constexpr int kStepBytes = 128;  // of the contraction, per LDS step: a cache line
constexpr int kPieces = kStepBytes / 16;
constexpr int kParts = 2;       // of a step: one MFMA of bf16, four of fp32 each
constexpr int64_t kBufferMax = (int64_t(1) << 31) - 8;  // bytes a buffer resource is made for at most

enum Layout : int { kAlong, kAcross };

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
  static constexpr bool kOneOffset = kRowsApart % (L == kAlong ? (Mixed ? 32 : 8) : sizeof(T) == 2 ? 4 : 16) == 0;
  uint32_t off[Direct ? (kOneOffset ? 1 : kLoads) : 1];
  uint32_t now;  // the step's
  int left;      // bytes of the buffer that the step's loads use
  int64_t away[Direct ? 1 : kLoads];  // through registers: a thread's pieces from `base` on
  u32x4 held[Direct ? 1 : kLoads];

  // Which position of an LDS row a piece is kept at: bits that are xor-ed to the piece's number.
  __device__ static __forceinline__ int spread(int row) {
    if constexpr (L == kAlong) return Mixed ? (row & 3) | ((row >> 3) & 1) << 2 : row & 7;
    else if constexpr (sizeof(T) == 2) return (row & 3) << 1;
    else return (((row >> 2) & 3) << 2) & (kRowPieces - 1);
  }

  // THREADS move a step's pieces: the block, or (64) every wavefront for itself.
  __device__ static __forceinline__ int thread() { return THREADS == 64 ? int(threadIdx.x & 63) : int(threadIdx.x); }

  __device__ __forceinline__ void place(int it, int &row, int &piece) const {
    const int id = it * THREADS + thread();
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
    } else {
#pragma unroll
      for (int it = 0; it < kLoads; ++it) {
        int row, piece;
        place(it, row, piece);
        away[it] = (L == kAlong && row >= valid ? valid - 1 : row) * pitch + 16 * piece;
      }
    }
    aim();
  }

  // A step is requested piece by piece (directly into LDS, or into registers), then advance() goes on to the next.  What lies past
  // the end of the contraction arrives as zeros.
  __device__ __forceinline__ void request(int it, uint32_t lds) {
    if constexpr (Direct) {
      const int wave = __builtin_amdgcn_readfirstlane(thread() >> 6);
      const int on = kOneOffset ? it * kRowsApart * int(pitch) : 0;
      const uint64_t from = reinterpret_cast<uint64_t>(base) + uint32_t(on);
      const u32x4 r = {uint32_t(from), uint32_t(from >> 32), uint32_t(left > on ? (left - on + 3) & ~3 : 0), 0x00020000u};  // whole dwords
      load_to_lds(r, kOneOffset ? now : off[it], lds + (it * THREADS + wave * 64) * 16);
    } else {
      // pieces that are not whole are put together by deliver(): a second way to fill `held` would let every load be waited for here
      u32x4 v;
      if (whole(contracted, bytes) || away[it] + 16 <= bytes) v = *reinterpret_cast<const u32x4_any *>(base + away[it]);
      held[it] = v;
    }
  }
  // Whether no piece of a step needs a look at the ends, with `contracted` elements and `bytes` from it on.  kAlong: rows past the last
  // one are the last one again, and are not stored.  kAcross: nor are columns past the last one, which may hold anything that can be
  // read: the next row's elements.
  __device__ __forceinline__ bool whole(int contracted, int64_t bytes) const {
    return contracted >= kSteps && (L == kAlong || bytes >= (kSteps - 1) * pitch + kRowBytes);
  }
  // Elements of a piece that belong to the contraction and, at the operand's end, to memory that may be read; the others are to be zero.
  __device__ __forceinline__ int inside(int it, int contracted, int64_t bytes) const {
    int row, piece;
    place(it, row, piece);
    if constexpr (L == kAlong) return contracted - piece * kElems;
    else return row >= contracted ? 0 : away[it] + 16 <= bytes ? kElems : valid - piece * kElems;
  }
  __device__ __forceinline__ void advance(int steps = 1) {
    const int64_t skip = steps * (L == kAlong ? int64_t(kStepBytes) : kSteps * pitch);
    base += skip, bytes -= skip, contracted -= steps * kSteps;
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

  // Zeroes what a step that came directly holds past the end of the contraction inside its last piece (the row's neighbours in
  // memory): `rest` elements of the step are contracted.  Call between the step's arrival and its first use.
  __device__ __forceinline__ void trim(uint32_t lds, int rest) const {
    if constexpr (Direct && L == kAlong) {
      using Bits = std::conditional_t<sizeof(T) == 2, uint16_t, uint32_t>;
      int id = thread();
      asm volatile("" : "+v"(id));  // what follows is not to be worked out ahead of the loop, where it would hold registers
      if ((id % kRowPieces ^ spread(id / kRowPieces)) != rest / kElems) return;
      for (int at = id * 16 + rest % kElems * int(sizeof(T)); at & 15; at += sizeof(T))
#pragma unroll
        for (int it = 0; it < kLoads; ++it) *reinterpret_cast<__attribute__((address_space(3))) Bits *>(lds + it * THREADS * 16 + at) = 0;
    }
  }

  // Writes what request() left in registers, `steps` before the one that is next now.
  __device__ __forceinline__ void deliver(uint32_t lds, int steps = 1) const {
    if constexpr (!Direct) {
      const int then = contracted + steps * kSteps;
      const int64_t back = steps * (L == kAlong ? int64_t(kStepBytes) : kSteps * pitch);
      const char *const from = base - back;
      const bool all = whole(then, bytes + back);
#pragma unroll
      for (int it = 0; it < kLoads; ++it) {
        u32x4 v = held[it];
        if (!all) {
          const int in = inside(it, then, bytes + back);
          if (in < kElems) {
            union {
              u32x4 v;
              T e[kElems];
            } u;
            u.v = u32x4{0, 0, 0, 0};
            if (away[it] + 16 <= bytes + back) {
#pragma unroll
              for (int w = 0; w < 4; ++w) {  // whole words, and half of one
                const int rest = in - w * int(4 / sizeof(T));
                u.v[w] = rest >= int(4 / sizeof(T)) ? v[w] : rest > 0 ? v[w] & 0xffffu : 0u;
              }
            } else {
#pragma unroll
              for (int e = 0; e < kElems; ++e)
                if (e < in) u.e[e] = reinterpret_cast<const T *>(from + away[it])[e];
            }
            v = u.v;
          }
        }
        *reinterpret_cast<__attribute__((address_space(3))) u32x4 *>(lds + (it * THREADS + thread()) * 16) = v;
      }
    }
  }

  // The group of 16 that fragment f of a wavefront is.
  __device__ static constexpr int group(int f, int wave) { return f * WAVES + wave; }

  // Where a lane reads: fragment f, part s of a step is at one of its bases plus constants.  kAcross with bf16: a group is 32 bytes of an
  // LDS row, four of which share 128 bytes and are xor-ed among each other.
  static constexpr int kFour = 4 / WAVES;  // fragments of a wavefront in four groups
  static_assert(WAVES == 1 || WAVES == 2 || WAVES == 4, "fragments repeat after four groups");
  static constexpr int kBases = L == kAlong ? kParts : sizeof(T) == 2 ? kFour : 4;
  struct Bases {
    uint32_t at[kBases];
  };
  template <int GROUPS>
  __device__ static __forceinline__ Bases bases(int wave) {
    const int lane = threadIdx.x & 63, p = lane & 15, q = lane >> 4;
    Bases b;
    if constexpr (L == kAlong) {
      const int row = Mixed ? 16 * GROUPS * wave + 8 * (p >> 2) + (p & 3) : 16 * group(0, wave) + p;
#pragma unroll
      for (int s = 0; s < kParts; ++s) b.at[s] = row * kRowBytes + (((4 * s + q) ^ spread(row)) << 4);
    } else if constexpr (sizeof(T) == 2) {
      const int k = 8 * q + (p >> 2);
#pragma unroll
      for (int v = 0; v < kBases; ++v) {
        const int piece = 2 * group(v, wave) + ((p >> 1) & 1);  // lane's 8 bytes: columns 4 * (p % 4) of the fragment
        b.at[v] = k * kRowBytes + ((piece ^ spread(k)) << 4) + (p & 1) * 8;
      }
    } else {
      const int col = 16 * group(0, wave) + p;
#pragma unroll
      for (int t = 0; t < 4; ++t) b.at[t] = (4 * q + t) * kRowBytes + (((col >> 2) ^ spread(4 * q + t)) << 4) + (col & 3) * 4;
    }
    return b;
  }

  // Lane's 16 bytes of fragment f.  Mixed: index p of fragment f stands for 32*(f/2) + 8*(p/4) + 4*(f%2) + p%4, so that two fragments
  // give a lane eight neighbours, and four lanes 32.
  __device__ __forceinline__ static u32x4 fragment(const Bases &b, uint32_t lds, int f, int s) {
    if constexpr (L == kAlong) {
      const int row = Mixed ? f / 2 * 32 + f % 2 * 4 : 16 * group(f, 0);
      return read_lds<u32x4>(b.at[s] + lds + row * kRowBytes);
    } else if constexpr (sizeof(T) == 2) {
      const uint32_t at = b.at[f % kBases] + lds + (group(f, 0) - group(f % kBases, 0)) * 32 + 32 * s * kRowBytes;
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
        const uint32_t at = (b.at[t] ^ (group(f, 0) % 4 << 6)) + group(f, 0) / 4 * 256;
        v[t] = read_lds<uint32_t>(at + lds + 16 * s * kRowBytes);
      }
      return v;
    }
  }
};

template <int N>
__device__ __forceinline__ void wait_loads() {  // all but the N newest loads have arrived
  __builtin_amdgcn_s_waitcnt((N & 15) | 7 << 4 | 15 << 8 | (N >> 4) << 14);
}
__device__ __forceinline__ void wait_lds() {  // LDS accesses are done
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(15 | 7 << 4 | 3 << 14);
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void wait_all() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(7 << 4);
}

// Eight neighbouring results as bf16.
__device__ __forceinline__ void store8(bf16_t *p, f32x4 a, f32x4 b) {
  *reinterpret_cast<u32x4_any *>(p) = u32x4{bf16_pair(a[0], a[1]), bf16_pair(a[2], a[3]), bf16_pair(b[0], b[1]), bf16_pair(b[2], b[3])};
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

// Where calls have few tiles and workers few rows (k_linear_few.hip).
template <bool Forward, class T, class TC, bool Epilogue = false>
int launch_linear_few(const LinearArgs &a, bool direct, bool small, void *stream);
template <class T>
int launch_linear_weight_split(const LinearArgs &a, void *stream);

}  // namespace detag

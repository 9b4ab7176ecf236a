// Dropout: every entry is kept with probability 1 - T / 65536 and then scaled by 65536 / (65536 - T), or set to zero; [+ residual].
//
// What is kept follows from a counter, so that no mask is stored and the gradient's pass draws the same one: the eight columns 8k .. 8k+7 of
// a worker's row take the eight halves of the four words of Philox-4x32-10 (noise_dev.hpp) with key seed and counter
// (k, 2^31 + row within the worker, worker, step): an even column the lower half of its word, the odd one after it the upper; kept where
// the half is at least T.  2^31 apart from the counters of the gradients' noise, whose second word counts blocks of columns.
//
// What bounds it is memory; a generator's block is 20 products of 32 bits for eight entries.  16384 rows of 4096 bf16 with a residual: 75 us
// (403 MB, 5.4 TB/s).  A wavefront has a row, so that the row's worker is found once and a lane's eight columns take one block of the generator.
#include "dev_common.hpp"
#include "detag_internal.h"
#include "noise_dev.hpp"
#include "rows_common.hpp"

namespace detag {
namespace {

struct DropoutArgs {
  const void *x, *residual;
  void *y;
  const int32_t *offsets;
  int64_t ldx, ldr, ldy;
  int n, rows, columns;
  uint32_t border, step, seed_lo, seed_hi;
  float scale;
};

constexpr int kThreads = 256, kEight = 8;

// A wavefront per row, eight columns a lane.
template <class T>
__global__ __launch_bounds__(kThreads) void dropout_kernel(DropoutArgs a) {
  constexpr int kElems = 16 / sizeof(T), kPieces = kEight / kElems;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  for (int64_t r = int64_t(blockIdx.x) * (kThreads / 64) + wave; r < a.rows; r += int64_t(gridDim.x) * (kThreads / 64)) {
    const Run own = run_of(a.offsets, a.n, a.rows, 0, int(r));
    if (own.part < 0) continue;
    const T *x = static_cast<const T *>(a.x) + r * a.ldx, *res = static_cast<const T *>(a.residual) + r * a.ldr;
    T *y = static_cast<T *>(a.y) + r * a.ldy;
    for (int64_t c = lane * kEight; c < a.columns; c += 64 * kEight) {
      const int inside = a.columns - int(c);
      u32x4 v[kPieces], add[kPieces];
#pragma unroll
      for (int k = 0; k < kPieces; ++k) v[k] = load_piece(x + c + k * kElems, inside - k * kElems);
#pragma unroll
      for (int k = 0; k < kPieces; ++k) add[k] = a.residual ? load_piece(res + c + k * kElems, inside - k * kElems) : u32x4{0, 0, 0, 0};
      uint32_t word[4];
      philox4x32_10(uint32_t(c / kEight), 0x80000000u + uint32_t(r - own.lo), uint32_t(own.part), a.step, a.seed_lo, a.seed_hi, word);
#pragma unroll
      for (int k = 0; k < kPieces; ++k) {
        float out[kElems];
#pragma unroll
        for (int e = 0; e < kElems; ++e) {
          const int at = k * kElems + e;
          const uint32_t half = at % 2 ? word[at / 2] >> 16 : word[at / 2] & 0xffffu;
          out[e] = (half >= a.border ? element<T>(v[k], e) * a.scale : 0.f) + element<T>(add[k], e);
        }
        store_piece(y + c + k * kElems, out, inside - k * kElems);
      }
    }
  }
}

}  // namespace

int launch_dropout(const Shape &s, const void *X, int64_t ldx, bool bf16, const int32_t *rows, int M, int columns, uint32_t border, uint64_t seed,
                   uint32_t step, const void *R, int64_t ldr, void *Y, int64_t ldy, void *stream) {
  const DropoutArgs a{X, R, Y, rows, ldx, ldr, ldy, s.n, M, columns, border, step, uint32_t(seed), uint32_t(seed >> 32),
                      float(65536.0 / (65536.0 - double(border)))};
  int64_t blocks = ceil_div_i64(M, kThreads / 64);
  if (blocks > 1 << 20) blocks = 1 << 20;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (bf16) dropout_kernel<bf16_t><<<dim3(uint32_t(blocks)), kThreads, 0, st>>>(a);
  else dropout_kernel<float><<<dim3(uint32_t(blocks)), kThreads, 0, st>>>(a);
  return hip_rc(hipGetLastError());
}

}  // namespace detag

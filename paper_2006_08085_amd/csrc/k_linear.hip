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
#include "linear_tiles.hpp"

namespace detag {

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

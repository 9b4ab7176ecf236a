// Products of a layer with their epilogue (k_linear.hip has the products):
//
//   forward       Z[r,:] = A[r,:] W_i^T + b_i,  Y[r,:] = R[r,:] + act(Z[r,:])
//   grad input    dA[r,:] = (dY[r,:] W_i) * act'(Z[r,:]),  Z what the layer's input came out of the activation of
//
// Bias, activation, residual and slope are taken of the fp32 sums in registers, where a pass of their own over the result would cost a
// read and a write of it; Z is stored beside Y for the way back.  Y and Z are rounded once each, from the same sums: Y is not computed from
// the rounded Z.
//
// What bounds the large ones is the product's own rounds of tiles, then the stores.  bf16, 8192 rows of 16 uneven workers, 1024 -> 4096 with gelu and
// Z 132 us (the product alone 97); its way back through gelu 135 (130 with relu's mask).  Eight rows, 1024 -> 1024 with bias and residual 6.4 (5.7).
// The 256 x 256 kernels hold 21 to 31 registers in scratch memory for their epilogue (0 to 2 without one).  Smaller tiles, whose epilogues
// cover each other's products, were slower: 128 x 128 forward 159 for 140 at the time, gradient 178 for 163.
#include "linear_tiles.hpp"

namespace detag {

int launch_linear_act(const Shape &s, const void *W, int64_t offset, int64_t bias, bool bf16, const void *A, int64_t lda, const int32_t *rows,
                      int M, int in, int out, int act, void *Z, int64_t ldz, const void *R, int64_t ldr, void *Y, int64_t ldy, bool y_bf16,
                      void *stream) {
  const size_t e = bf16 ? 2 : 4;
  const char *w = static_cast<const char *>(W);
  LinearArgs a{w + offset * e, A, nullptr, Y, rows, s.ld, lda, 0, ldy, s.n, M, in, out, 0};
  a.bias = bias < 0 ? nullptr : w + bias * e, a.residual = R, a.pre = Z, a.ldr = ldr, a.ldz = ldz, a.act = act;
  const bool direct = on_dwords(a.w, in, e) && s.ld * e % 4 == 0 && on_dwords(A, lda, e);
  if (!bf16) return launch_product<kForward, float, float, true>(a, direct, stream);
  return y_bf16 ? launch_product<kForward, bf16_t, bf16_t, true>(a, direct, stream) : launch_product<kForward, bf16_t, float, true>(a, direct, stream);
}

int launch_linear_grad_input_act(const Shape &s, const void *W, int64_t offset, bool bf16, const void *dY, int64_t ldy, const int32_t *rows, int M,
                                 int in, int out, int act, const void *Z, int64_t ldz, void *dA, int64_t lda, void *stream) {
  const size_t e = bf16 ? 2 : 4;
  LinearArgs a{static_cast<const char *>(W) + offset * e, dY, Z, dA, rows, s.ld, ldy, ldz, lda, s.n, M, in, out, 0};
  a.act = act, a.flag = Z && reads_by_buffer(Z, ldz, e);
  const bool direct = on_dwords(a.w, in, e) && s.ld * e % 4 == 0 && on_dwords(dY, ldy, e);
  return bf16 ? launch_product<kGradInput, bf16_t, bf16_t, true>(a, direct, stream) : launch_product<kGradInput, float, float, true>(a, direct, stream);
}

}  // namespace detag

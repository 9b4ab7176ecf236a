"""Operators of residual blocks at sizes that reach the kernels which the cases of their own tests do not: every tile of a product with an
epilogue in both directions, its slopes read through a buffer and not, and attention's blocks of 128 queries with more sequences than a
wavefront has lanes, heads of odd widths, and one key head for all.  References and bounds are those of test_gpu_linear_act and
test_gpu_attention."""
import pytest
import torch

from tests import test_gpu_attention as attention
from tests.block_util import (ACTS, BF16, DEV, F32, U, _built, act64, act_error, assert_within, context, half_step, matrix, offsets,  # noqa: F401
                              parameters, slope64, slope_error, spans)

pytestmark = pytest.mark.gpu

MANY, FEW = [100, 0, 150, 90, 110, 130, 120, 100], [50, 0, 75, 45, 55, 65, 60, 50]
# kernel | worker's rows | columns of the result | contracted | type
TILES = [
    ("256 x 256", [700, 900], 4804, 200, BF16), ("256 x 256", [257, 1300, 43], 4866, 72, BF16), ("128 x 128", MANY, 3300, 200, BF16),
    ("128 x 128", MANY, 3330, 74, BF16), ("64 x 128", FEW, 3300, 200, BF16), ("64 x 128", FEW, 3398, 66, BF16),
    ("64 x 64", [257, 3, 0, 300], 700, 72, BF16), ("64 x 64 through registers", [257, 3, 0, 300], 701, 75, BF16),
    ("64 x 128 through registers", FEW, 3301, 75, BF16), ("64 x 64", [257, 3, 0, 300], 700, 72, F32), ("64 x 64", [257, 3, 0, 300], 1031, 130, F32),
    ("64 rows of few tiles", [257, 3, 0, 300], 700, 600, BF16), ("64 rows of few tiles", [257, 3, 0, 300], 700, 302, F32),
]


def _layer(counts, inn, out, dtype):
    n, weights = len(counts), inn * out
    bias = weights + weights % 2
    ctx = context(n, bias + out)
    return ctx, bias, parameters(n, ctx.ld, dtype, [(0, weights, 0.0, inn ** -0.5), (bias, out, 0.0, 0.5)], 1)


def _ids(c):
    return f"{c[0]}-{c[2]}-{c[3]}-{'bf16' if c[4] is BF16 else 'f32'}"


@pytest.mark.parametrize("case", TILES, ids=_ids)
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("spare", [0, 2, 1])               # elements a row of Z: with one its rows start on half dwords
def test_every_kernel_of_an_input_gradient_with_slope(case, act, spare):
    _, counts, inn, out, dtype = case
    M = sum(counts)
    ctx, _, W = _layer(counts, inn, out, dtype)
    dY, _ = matrix(M + 2, out, dtype, 2, out % 2)
    dY[M:] = float("nan")
    Z, _ = matrix(M + 2, inn, dtype, 3, spare, scale=2.0)
    Z[:, 0] = 0.0
    dA, buf = matrix(M + 2, inn, dtype, None, spare, around=7.0)
    before = buf.clone()
    ctx.linear_grad_input_act(W, 0, dY, offsets(counts), dA, act=ACTS[act], pre=Z if act != "none" else None)
    torch.cuda.synchronize()
    for i, lo, hi in spans(counts):
        Wi, y, z = W[i, :inn * out].double().view(out, inn), dY[lo:hi].double(), Z[lo:hi].double()
        ref, size, slope = y @ Wi, y.abs() @ Wi.abs(), slope64(z, act)
        off = 2 * (out + 8) * U * size * slope.abs() + 2 * slope_error(z, act, dtype) * ref.abs() + 2 * U * (ref * slope).abs()
        assert_within(dA[lo:hi], ref * slope, off + half_step(dtype) * (ref * slope).abs())
    dA[:M] = 7.0
    assert torch.equal(buf, before)


@pytest.mark.parametrize("case", TILES, ids=_ids)
@pytest.mark.parametrize("act, pre, residual, wide", [("gelu", True, False, False), ("silu", True, True, True), ("relu", False, True, False),
                                                      ("none", False, True, True)])
def test_every_kernel_of_a_product_with_epilogue(case, act, pre, residual, wide):
    _, counts, out, inn, dtype = case
    M, y_type = sum(counts), F32 if wide else dtype
    ctx, bias, W = _layer(counts, inn, out, dtype)
    A, _ = matrix(M + 2, inn, dtype, 2, inn % 2)
    A[M:] = float("nan")
    R, _ = matrix(M + 2, out, y_type, 3, 3)
    Y, Ybuf = matrix(M + 2, out, y_type, None, around=7.0)
    Z, Zbuf = matrix(M + 2, out, dtype, None, 1, around=5.0)
    before = Ybuf.clone(), Zbuf.clone()
    ctx.linear_act(W, 0, A, offsets(counts), Y, bias=bias, act=ACTS[act], pre=Z if pre else None, residual=R if residual else None)
    torch.cuda.synchronize()
    for i, lo, hi in spans(counts):
        Wi, a, b = W[i, :inn * out].double().view(out, inn), A[lo:hi].double(), W[i, bias:bias + out].double()
        z, off = a @ Wi.t() + b, 2 * (inn + 9) * U * (a.abs() @ Wi.abs().t() + b.abs())
        if pre:
            assert_within(Z[lo:hi], z, off + half_step(dtype) * z.abs())
        y, r = act64(z, act), R[lo:hi].double() if residual else torch.zeros_like(z)
        slope = 1.0 if act in ("none", "relu") else 1.13
        assert_within(Y[lo:hi], y + r, slope * off + 2 * act_error(z, act, y_type) + 2 * U * (y.abs() + r.abs()) + half_step(y_type) * (y + r).abs())
    Y[:M], Z[:M] = 7.0, 5.0
    assert torch.equal(Ybuf, before[0]) and torch.equal(Zbuf, before[1])


@pytest.mark.parametrize("contracted", [40, 300])          # tiles; the kernels of few rows
def test_fp32_rows_too_far_apart_for_a_buffer(contracted):
    """256 rows of 2^21 and more floats do not fit a buffer's 2^31 bytes: operands pass registers, and the same values come out."""
    counts, inn, far = [12, 0, 8], 90, (1 << 21) + 4
    M, rows = sum(counts), offsets(counts)
    buf = torch.zeros(M * far, device=DEV).view(M, far)

    def apart(t):
        buf[:, :t.shape[1]] = t
        return buf[:, :t.shape[1]]
    ctx, bias, W = _layer(counts, contracted, inn, F32)
    A, Z, Y = matrix(M, contracted, F32, 2)[0], torch.zeros(M, inn, device=DEV), torch.zeros(M, inn, device=DEV)
    near = torch.zeros_like(Y), torch.zeros_like(Z)
    ctx.linear_act(W, 0, apart(A), rows, Y, bias=bias, act=ACTS["gelu"], pre=Z, residual=A[:, :1].expand(M, inn).contiguous())
    ctx.linear_act(W, 0, A, rows, near[0], bias=bias, act=ACTS["gelu"], pre=near[1], residual=A[:, :1].expand(M, inn).contiguous())
    # two orders of a sum of K terms of about K^-1/2: each is off by at most (K + 9) u of the magnitudes, which are below 6 K^1/2
    most = 2 * (contracted + 9) * U * 6 * contracted ** 0.5
    assert (Z - near[1]).abs().max() <= most and (Y - near[0]).abs().max() <= 1.13 * most + 64 * U * Z.abs().max()
    ctx, _, W = _layer(counts, inn, contracted, F32)
    dA, near = torch.zeros(M, inn, device=DEV), torch.zeros(M, inn, device=DEV)
    ctx.linear_grad_input_act(W, 0, apart(A), rows, dA, act=ACTS["silu"], pre=Z)
    ctx.linear_grad_input_act(W, 0, A, rows, near, act=ACTS["silu"], pre=Z)
    assert dA.any() and (dA - near).abs().max() <= 1.1 * most * (contracted / inn) ** 0.5 + 1e-6


# as test_gpu_attention's: sequences' rows | heads | key heads | width | spare elements a row | elements before the first | type
SEQUENCES = [0, 1, 130, 2, 33, 128, 5] * 10 + [0, 300]     # 72 of them: their runs are found in two rounds
HEADS = [(SEQUENCES, 32, 8, 128, 0, 0, BF16), (SEQUENCES, 32, 8, 64, 8, 0, BF16), (SEQUENCES, 32, 16, 20, 3, 1, BF16), (SEQUENCES, 32, 8, 128, 0, 0, F32),
         (SEQUENCES, 32, 32, 33, 1, 0, F32), ([300, 130, 128, 129], 96, 8, 99, 3, 1, F32), ([300, 130, 128, 129], 96, 4, 100, 0, 0, BF16),
         ([300, 130, 128, 129], 96, 96, 101, 1, 1, BF16), ([2900], 16, 1, 64, 0, 0, BF16), ([2900], 32, 1, 24, 0, 0, F32),
         ([300, 5, 0, 77], 2, 1, 99, 0, 0, F32)]           # and few heads: a block's wavefronts share keys that pass registers


@pytest.mark.parametrize("case", HEADS, ids=attention._ids)
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
def test_every_kernel_of_attention(case, causal):
    attention.test_attention(case, causal)
    attention.test_attention_grad(case, causal)

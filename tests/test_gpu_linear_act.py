"""Products of a layer with bias, activation and residual, and the gradient of that epilogue, against plain implementations in 64 bits
(bounds: block_util.py; a product's sum of K terms is off by at most (K + 8) u of their magnitudes)."""
import pytest
import torch

from tests.block_util import (ACTS, BF16, DEV, F32, U, _built, act64, act_error, assert_within, context, half_step, matrix, offsets,  # noqa: F401
                              parameters, slope64, slope_error, spans)

pytestmark = pytest.mark.gpu

# worker's rows | in | out | first column | spare elements a row | elements before the first | type: every kernel of the products
LAYERS = [
    ([1, 1, 1], 64, 64, 0, 0, 0, BF16), ([1], 1, 1, 0, 0, 0, F32), ([3, 0, 2], 1, 5, 3, 0, 0, BF16), ([2, 1], 7, 1, 1, 1, 1, F32),
    ([0, 0, 0], 40, 24, 0, 0, 0, BF16), ([1] * 8, 1024, 1024, 0, 0, 0, BF16), ([1, 3], 600, 90, 0, 0, 0, F32),
    ([5, 0, 130, 0, 1, 127], 128, 96, 8, 0, 0, BF16), ([5, 0, 130, 0, 1, 127], 100, 136, 4, 0, 0, F32),
    ([257, 3, 0, 300], 264, 520, 16, 8, 8, BF16), ([257, 3, 0, 300], 132, 260, 4, 4, 4, F32), ([33, 64, 65], 77, 131, 5, 3, 1, BF16),
    ([33, 64, 65], 77, 131, 5, 3, 1, F32), ([17, 1, 15], 1032, 200, 0, 0, 0, BF16), ([2, 9, 1, 4], 333, 515, 7, 5, 3, BF16),
    ([70, 60], 1024, 1000, 0, 0, 0, BF16), ([700, 900], 384, 640, 0, 0, 0, BF16), ([1100, 500], 520, 1288, 0, 0, 0, BF16),
    ([2000, 900, 1500, 3], 192, 2056, 0, 0, 0, BF16),
]


def _ids(c):
    return f"{len(c[0])}x{sum(c[0])}-{c[1]}-{c[2]}-{c[3]}-{c[4]}-{'bf16' if c[6] is BF16 else 'f32'}"


def _layer(case):
    counts, inn, out, offset, extra, shift, dtype = case
    n, M = len(counts), sum(counts)
    bias = offset + inn * out + 1
    d = bias + out
    ctx = context(n, d, d + 5 if extra else None)
    W = parameters(n, ctx.ld, dtype, [(offset, inn * out, 0.0, inn ** -0.5), (bias, out, 0.0, 0.5)], 1)
    return ctx, n, M, bias, W


@pytest.mark.parametrize("case", LAYERS, ids=_ids)
@pytest.mark.parametrize("act,with_bias,pre,residual,wide", [("gelu", True, True, False, False), ("relu", True, False, True, True),
                                                             ("silu", False, True, True, False), ("none", True, False, True, False),
                                                             ("gelu", True, True, True, True), ("none", False, False, False, False)])
def test_linear_act(case, act, with_bias, pre, residual, wide):
    counts, inn, out, offset, extra, shift, dtype = case
    ctx, n, M, bias, W = _layer(case)
    y_type = F32 if wide else dtype
    A, _ = matrix(M + 2, inn, dtype, 2, extra, shift)
    A[M:] = float("nan")
    R, _ = matrix(M + 2, out, y_type, 3, extra, 0)
    Y, Ybuf = matrix(M + 2, out, y_type, None, extra, shift, around=7.0)
    Z, Zbuf = matrix(M + 2, out, dtype, None, extra, shift, around=5.0)
    before = Ybuf.clone(), Zbuf.clone()
    rows = offsets(counts)
    more = dict(bias=bias if with_bias else None, act=ACTS[act], pre=Z if pre else None)
    ctx.linear_act(W, offset, A, rows, Y, residual=R if residual else None, **more)
    torch.cuda.synchronize()
    first = Y.clone()
    for i, lo, hi in spans(counts):
        Wi, a = W[i, offset:offset + inn * out].double().view(out, inn), A[lo:hi].double()
        b = W[i, bias:bias + out].double() if with_bias else torch.zeros(out, dtype=torch.float64, device=DEV)
        z = a @ Wi.t() + b
        off = 2 * (inn + 9) * U * (a.abs() @ Wi.abs().t() + b.abs())
        if pre:
            assert_within(Z[lo:hi], z, off + half_step(dtype) * z.abs())
        y, r = act64(z, act), R[lo:hi].double() if residual else torch.zeros_like(z)
        slope = 1.0 if act in ("none", "relu") else 1.13
        assert_within(Y[lo:hi], y + r, slope * off + 2 * act_error(z, act, y_type) + 2 * U * (y.abs() + r.abs()) + half_step(y_type) * (y + r).abs())
    if residual:                                          # over the residual: the same bits
        ctx.linear_act(W, offset, A, rows, R, residual=R, **more)
        assert torch.equal(R[:M], first[:M])
    if act in ("none", "relu") and not with_bias and not residual:
        ctx.linear(W, offset, A, rows, R, relu=act == "relu")
        assert torch.equal(R[:M], first[:M])
    Y[:M], Z[:M] = 7.0, 5.0
    assert torch.equal(Ybuf, before[0]) and torch.equal(Zbuf, before[1])


@pytest.mark.parametrize("case", LAYERS, ids=_ids)
@pytest.mark.parametrize("act", list(ACTS))
def test_linear_grad_input_act(case, act):
    counts, inn, out, offset, extra, shift, dtype = case
    ctx, n, M, bias, W = _layer(case)
    dY, _ = matrix(M + 2, out, dtype, 2, extra, shift)
    dY[M:] = float("nan")
    Z, _ = matrix(M + 2, inn, dtype, 3, extra, 0, scale=2.0)
    Z[:, 0] = 0.0
    dA, buf = matrix(M + 2, inn, dtype, None, extra, shift, around=7.0)
    before = buf.clone()
    ctx.linear_grad_input_act(W, offset, dY, offsets(counts), dA, act=ACTS[act], pre=Z if act != "none" else None)
    torch.cuda.synchronize()
    for i, lo, hi in spans(counts):
        Wi, y, z = W[i, offset:offset + inn * out].double().view(out, inn), dY[lo:hi].double(), Z[lo:hi].double()
        ref, size, slope = y @ Wi, y.abs() @ Wi.abs(), slope64(z, act)
        off = 2 * (out + 8) * U * size * slope.abs() + 2 * slope_error(z, act, dtype) * ref.abs() + 2 * U * (ref * slope).abs()
        assert_within(dA[lo:hi], ref * slope, off + half_step(dtype) * (ref * slope).abs())
    dA[:M] = 7.0
    assert torch.equal(buf, before)


# worker's rows | outputs | first column | spare elements a row | elements before the first | type
BIASES = [([1], 1, 0, 0, 0, F32), ([1, 0, 1], 5, 3, 0, 1, BF16), ([0, 0], 40, 0, 0, 0, BF16), ([5, 0, 17, 8, 9], 264, 8, 8, 0, BF16),
          ([33, 7], 1001, 1, 3, 1, BF16), ([33, 7], 1001, 1, 3, 1, F32), ([100, 3], 4099, 0, 0, 0, BF16), ([40] * 70, 24, 0, 0, 0, F32),
          ([9000, 0, 1, 700], 72, 4, 0, 0, BF16), ([1], 2000, 0, 0, 0, F32)]


@pytest.mark.parametrize("case", BIASES, ids=lambda c: f"{len(c[0])}x{sum(c[0])}-{c[1]}-{c[3]}-{'bf16' if c[5] is BF16 else 'f32'}")
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("accumulate", [False, True])
def test_linear_grad_bias(case, act, accumulate):
    counts, out, offset, extra, shift, dtype = case
    n, M = len(counts), sum(counts)
    ctx = context(n, offset + out + 2)
    dY, _ = matrix(M + 2, out, dtype, 2, extra, shift)
    dY[M:] = float("inf")
    Z, _ = matrix(M + 2, out, dtype, 3, extra, 0, scale=2.0)
    dZ, buf = matrix(M + 2, out, dtype, None, extra, shift, around=7.0)
    before = buf.clone()
    G = torch.randn(n, ctx.ld, generator=torch.Generator().manual_seed(3)).to(DEV)
    G0, rows = G.clone(), offsets(counts)
    ctx.linear_grad_bias(dY, rows, G, offset, act=ACTS[act], pre=None if act == "none" else Z, dZ=None if act == "none" else dZ, accumulate=accumulate)
    torch.cuda.synchronize()
    kept = G.clone()
    here = slice(offset, offset + out)
    for i, lo, hi in spans(counts):
        y, z = dY[lo:hi].double(), Z[lo:hi].double()
        ref = y * slope64(z, act)
        off = 2 * slope_error(z, act, dtype) * y.abs() + 2 * U * ref.abs()
        if act != "none":
            assert_within(dZ[lo:hi], ref, off + half_step(dtype) * ref.abs())
        start = G0[i, here].double() * accumulate
        assert_within(G[i, here], ref.sum(0) + start, off.sum(0) + 2 * (hi - lo + 8) * U * (ref.abs().sum(0) + start.abs()))
    if act != "none" and not accumulate:                  # over dY and over Z: the same bits
        for over_z in (False, True):
            y, z = dY.clone(), Z.clone()
            ctx.linear_grad_bias(y, rows, G, offset, act=ACTS[act], pre=z, dZ=z if over_z else y)
            assert torch.equal((z if over_z else y)[:M], dZ[:M]) and torch.equal(G, kept)
    G[:, here] = G0[:, here]
    dZ[:M] = 7.0
    assert torch.equal(G, G0) and torch.equal(buf, before)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_ends_of_the_line(act, dtype):
    """Sums that are infinite, huge or not a number: the limits of the activation and of its slope."""
    inf, nan = float("inf"), float("nan")
    z = torch.tensor([[inf, -inf, nan, 0.0, 1e30, -1e30, 300.0, -300.0]], device=DEV, dtype=dtype)
    ctx = context(1, 72)
    eye = torch.zeros(1, ctx.ld, dtype=dtype, device=DEV)
    eye[0, :64] = torch.eye(8, dtype=dtype, device=DEV).view(-1)
    rows, G = offsets([1]), torch.zeros(1, ctx.ld, device=DEV)
    eye[0, 64:72] = z[0]
    Y, dZ = torch.zeros_like(z), torch.zeros_like(z)
    ctx.linear_act(eye, 0, torch.zeros_like(z), rows, Y, bias=64, act=ACTS[act])
    ctx.linear_grad_bias(torch.ones_like(z), rows, G, 0, act=ACTS[act], pre=z, dZ=dZ)
    top = torch.tensor(1e30).to(dtype).item()
    assert Y[0, :2].tolist() == [inf, 0.0] and Y[0, 2].isnan() and Y[0, 3:].tolist() == [0.0, top, 0.0, 300.0, 0.0]
    assert dZ[0, :2].tolist() == [1.0, 0.0] and dZ[0, 3:].tolist() == [0.0 if act == "relu" else 0.5, 1.0, 0.0, 1.0, 0.0]
    assert dZ[0, 2].item() == 0.0 if act == "relu" else dZ[0, 2].isnan()


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_gradient_against_differences(act):
    """The loss sum(dY * act(A W^T + b)) in 64 bits, along a direction of the layer's input's own sums and of the bias."""
    n, inn, out, counts = 2, 40, 24, [3, 5]
    case = (counts, inn, out, 0, 0, 0, F32)
    ctx, n, M, bias, W = _layer(case)
    below, _ = matrix(M, inn, F32, 4)
    A, Z, Y = torch.zeros(M, inn, device=DEV), torch.zeros(M, out, device=DEV), torch.zeros(M, out, device=DEV)
    A.copy_(act64(below.double(), act))
    rows, G = offsets(counts), torch.zeros(n, ctx.ld, device=DEV)
    ctx.linear_act(W, 0, A, rows, Y, bias=bias, act=ACTS[act], pre=Z)
    dY, _ = matrix(M, out, F32, 5)
    dZ, dbelow = torch.zeros_like(dY), torch.zeros_like(A)
    ctx.linear_grad_bias(dY, rows, G, bias, act=ACTS[act], pre=Z, dZ=dZ)
    ctx.linear_grad_input_act(W, 0, dZ, rows, dbelow, act=ACTS[act], pre=below)
    g = torch.Generator(device=DEV).manual_seed(9)
    v, vb = (torch.randn(*s, generator=g, device=DEV, dtype=torch.float64) for s in ((M, inn), (n, out)))

    def loss(t):
        total = 0
        for i, lo, hi in spans(counts):
            a = act64(below[lo:hi].double() + t * v[lo:hi], act)
            z = a @ W[i, :inn * out].double().view(out, inn).t() + W[i, bias:bias + out].double() + t * vb[i]
            total = total + (act64(z, act) * dY[lo:hi].double()).sum()
        return total.item()
    h = 1e-4
    by_difference = (loss(h) - loss(-h)) / (2 * h)
    terms = torch.cat([(dbelow.double() * v).view(-1), (G[:, bias:bias + out].double() * vb).view(-1)])
    # 1e-5: sums of 40 and 24 terms and their slopes, each within 50 u of its magnitudes; h^2 = 1e-8
    assert abs(by_difference - terms.sum().item()) <= 1e-5 * terms.abs().sum().item()

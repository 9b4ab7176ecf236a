"""Layer norm of every worker's rows and its gradient, against plain implementations in 64 bits (bounds: block_util.py)."""
import pytest
import torch

import paper_2006_08085_amd as D
from tests.block_util import BF16, DEV, F32, U, _built, assert_within, context, half_step, matrix, offsets, parameters, spans  # noqa: F401

pytestmark = pytest.mark.gpu
EPS = 1e-5

# worker's rows | columns | first column of the gain | spare elements a row | elements before the first | type
CASES = [
    ([1], 1, 0, 0, 0, F32), ([1], 1, 0, 0, 0, BF16), ([3, 0, 2], 7, 3, 0, 1, BF16), ([0, 0, 0], 40, 0, 0, 0, BF16),
    ([1, 1, 1, 1], 1024, 0, 0, 0, BF16), ([5, 0, 17, 1], 512, 8, 8, 0, BF16), ([5, 0, 17, 1], 513, 5, 3, 1, BF16), ([9, 30], 256, 4, 4, 0, F32),
    ([9, 30], 259, 1, 2, 3, F32), ([33, 8, 7], 1100, 0, 0, 0, BF16), ([2, 0, 11], 777, 5, 0, 0, F32), ([2, 9], 2048, 0, 0, 0, BF16),
    ([2, 9], 2049, 0, 1, 0, BF16), ([12], 4096, 16, 0, 0, BF16), ([3, 10], 4097, 0, 0, 1, BF16), ([3, 10], 8192, 0, 0, 0, BF16),
    ([1, 9], 16384, 0, 0, 0, BF16), ([4, 5], 16383, 1, 0, 0, BF16), ([3, 8], 2048, 0, 0, 0, F32), ([3, 8], 4095, 0, 0, 0, F32),
    ([3, 8], 8190, 2, 2, 2, F32), ([2, 3], 16384, 0, 0, 0, F32), ([1] * 70 + [3, 0, 5], 24, 0, 0, 0, F32), ([40, 0, 1] * 25, 64, 0, 0, 0, BF16),
]


def _ids(c):
    return f"{len(c[0])}x{sum(c[0])}-{c[1]}-{c[2]}-{c[3]}-{c[4]}-{'bf16' if c[5] is BF16 else 'f32'}"


def _setup(case, seed=1, bias=True):
    counts, C, gain, extra, shift, dtype = case
    n, M = len(counts), sum(counts)
    d = gain + 2 * C + 3
    ctx = context(n, d, d + (1 if extra else 0))
    at = gain + C + 3
    P = parameters(n, ctx.ld, dtype, [(gain, C, 1.0, 0.2)] + ([(at, C, 0.0, 0.3)] if bias else []), seed)
    level = 3 * torch.randn(M + 2, 1, generator=torch.Generator().manual_seed(seed + 5))
    x = level + torch.randn(M + 2, C, generator=torch.Generator().manual_seed(seed + 6))
    X, _ = matrix(M + 2, C, dtype, None, extra, shift, values=x)
    X[M:] = float("nan")                                  # rows that nobody owns
    return ctx, counts, n, M, C, gain, at if bias else None, P, X


def _statistics(x, C):
    """xhat, s, and what xhat may be off by."""
    mean = x.mean(1, keepdim=True)
    s = 1 / torch.sqrt((x - mean).pow(2).mean(1, keepdim=True) + EPS)
    xhat = (x - mean) * s
    size = x.abs().mean(1, keepdim=True) * s
    off = min(C, 80) * U * (size + xhat.abs() * (1 + 2 * size * size * 80 * U)) + 12 * U * xhat.abs() + 2 * U * size
    return xhat, s, off


@pytest.mark.parametrize("case", CASES, ids=_ids)
@pytest.mark.parametrize("bias", [True, False])
def test_layer_norm(case, bias):
    ctx, counts, n, M, C, gain, at, P, X = _setup(case, bias=bias)
    dtype, extra, shift = case[5], case[3], case[4]
    Y, Ybuf = matrix(M + 2, C, dtype, None, extra, shift, around=7.0)
    before = Ybuf.clone()
    ctx.layer_norm(P, gain, at, X, offsets(counts), Y, eps=EPS)
    torch.cuda.synchronize()
    for i, lo, hi in spans(counts):
        xhat, s, off = _statistics(X[lo:hi].double(), C)
        g, b = P[i, gain:gain + C].double(), P[i, at:at + C].double() if bias else torch.zeros(C, dtype=torch.float64, device=DEV)
        ref = xhat * g + b
        assert_within(Y[lo:hi], ref, 2 * (off * g.abs() + 3 * U * (xhat * g).abs() + U * b.abs()) + half_step(dtype) * ref.abs())
    Y[:M] = 7.0
    assert torch.equal(Ybuf, before)                      # nothing else was written


def _reference(x, dy, g, C):
    """dX (without add), the terms of dg, and their bounds."""
    xhat, s, off = _statistics(x, C)
    h = dy * g
    K = min(C, 80) * U
    hx = (h * xhat).mean(1, keepdim=True)
    dx = s * (h - h.mean(1, keepdim=True) - xhat * hx)
    size = (h * xhat).abs().mean(1, keepdim=True)
    hx_off = K * size + (h.abs() * off).mean(1, keepdim=True) + 4 * U * size
    bound = s * ((K + 16 * U) * (h.abs() + h.abs().mean(1, keepdim=True)) + off * size + xhat.abs() * (hx_off + K * size + 8 * U * size))
    return dx, 2 * bound, dy * xhat, (dy * xhat).abs() * 2 * U + dy.abs() * off


@pytest.mark.parametrize("case", CASES, ids=_ids)
@pytest.mark.parametrize("bias,add,accumulate", [(True, True, False), (True, False, True), (False, True, True), (False, False, False)])
def test_layer_norm_grad(case, bias, add, accumulate):
    ctx, counts, n, M, C, gain, at, P, X = _setup(case, bias=bias)
    dtype, extra, shift = case[5], case[3], case[4]
    dY, _ = matrix(M + 2, C, dtype, 11, extra, shift, scale=0.1)
    dY[M:] = float("inf")
    past, _ = matrix(M + 2, C, dtype, 12, extra, 0, scale=0.1)
    dX, dXbuf = matrix(M + 2, C, dtype, None, extra, shift, around=7.0)
    G = torch.randn(n, ctx.ld, generator=torch.Generator().manual_seed(3)).to(DEV)
    before, G0 = dXbuf.clone(), G.clone()
    rows = offsets(counts)
    ctx.layer_norm_grad(P, gain, at, X, dY, rows, dX, G, eps=EPS, add=past if add else None, accumulate=accumulate)
    torch.cuda.synchronize()
    kept = (dX.clone(), G.clone())
    for i, lo, hi in spans(counts):
        dy, c = dY[lo:hi].double(), hi - lo
        dx, off, terms, terms_off = _reference(X[lo:hi].double(), dy, P[i, gain:gain + C].double(), C)
        more = past[lo:hi].double() if add else torch.zeros_like(dx)
        assert_within(dX[lo:hi], dx + more, off + 4 * U * (dx.abs() + more.abs()) + half_step(dtype) * (dx + more).abs())
        start = G0[i].double() * accumulate
        for first, t, t_off in [(gain, terms, terms_off)] + ([(at, dy, 0 * dy)] if bias else []):
            here = slice(first, first + C)
            size = t.abs().sum(0) + start[here].abs()
            assert_within(G[i, here], t.sum(0) + start[here], 2 * (t_off.sum(0) + (c + 8) * U * size))
    dX[:M] = 7.0
    G[:, gain:gain + C] = G0[:, gain:gain + C]
    if bias:
        G[:, at:at + C] = G0[:, at:at + C]
    assert torch.equal(dXbuf, before) and torch.equal(G, G0)
    if not accumulate:                                    # and the same bits again, in place too
        for target in ("fresh", "dY", "X") + (("add",) if add else ()):
            x, dy, p = X.clone(), dY.clone(), past.clone()
            out = {"fresh": torch.zeros_like(x), "dY": dy, "X": x, "add": p}[target]
            ctx.layer_norm_grad(P, gain, at, x, dy, rows, out, G, eps=EPS, add=p if add else None)
            assert torch.equal(out[:M], kept[0][:M]) and torch.equal(G, kept[1])


def test_in_place_and_rows_apart():
    """Y over X; rows that begin and end inside the matrix; a worker's rows far from its neighbour's first."""
    n, C, M = 3, 640, 50
    ctx = context(n, 2 * C)
    P = parameters(n, ctx.ld, F32, [(0, C, 1.0, 0.1), (C, C, 0.0, 0.1)], 1)
    X, _ = matrix(M, C, F32, 2)
    rows = torch.tensor([7, 9, 9, 43], dtype=torch.int32, device=DEV)
    Y = torch.zeros_like(X)
    ctx.layer_norm(P, 0, C, X, rows, Y)
    start = X.clone()
    ctx.layer_norm(P, 0, C, X, rows, X)
    assert torch.equal(X[7:43], Y[7:43]) and torch.equal(X[:7], start[:7]) and torch.equal(X[43:], start[43:])
    assert not Y[:7].any() and not Y[43:].any()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_constant_rows_and_rows_that_are_not_finite(dtype):
    """A constant row has nothing but its bias; what is not finite stays in its row, and reaches the sums of its worker only."""
    n, C, M = 2, 300, 6
    ctx = context(n, 2 * C)
    P = parameters(n, ctx.ld, dtype, [(0, C, 1.0, 0.1), (C, C, 0.0, 0.1)], 1)
    X, _ = matrix(M, C, dtype, 2)
    X[0], X[1, 7], X[2, 9] = 2.5, float("nan"), float("inf")
    rows = offsets([3, 3])
    Y, dX, G = torch.zeros_like(X), torch.zeros_like(X), torch.zeros(n, ctx.ld, device=DEV)
    ctx.layer_norm(P, 0, C, X, rows, Y)
    assert torch.equal(Y[0], P[0, C:2 * C]) and Y[1].isnan().all() and Y[2].isnan().all() and Y[3:].isfinite().all()
    dY, _ = matrix(M, C, dtype, 3)
    ctx.layer_norm_grad(P, 0, C, X, dY, rows, dX, G)
    assert dX[0].isfinite().all() and dX[1:3].isnan().all() and dX[3:].isfinite().all()
    assert G[0, :C].isnan().all() and G[0, C:].isfinite().all() and G[1].isfinite().all()


def test_gradient_against_differences():
    """Along a direction of all inputs at once, with the loss sum(dY * y) in 64 bits; the step's error is h^2 of the third derivative."""
    n, C, counts = 2, 130, [3, 4]
    case = (counts, C, 0, 0, 0, F32)
    ctx, counts, n, M, C, gain, at, P, X = _setup(case)
    dY, _ = matrix(M + 2, C, F32, 11)
    dX, G = torch.zeros_like(X), torch.zeros(n, ctx.ld, device=DEV)
    ctx.layer_norm_grad(P, gain, at, X, dY, offsets(counts), dX, G)
    g = torch.Generator(device=DEV).manual_seed(9)
    vx = torch.randn(M, C, generator=g, device=DEV, dtype=torch.float64)
    vp = torch.randn(n, ctx.ld, generator=g, device=DEV, dtype=torch.float64)

    def loss(t):
        total = 0
        for i, lo, hi in spans(counts):
            x, p = X[lo:hi].double() + t * vx[lo:hi], P[i].double() + t * vp[i]
            y = torch.nn.functional.layer_norm(x, (C,), p[gain:gain + C], p[at:at + C], eps=1e-5)
            total = total + (y * dY[lo:hi].double()).sum()
        return total.item()
    h = 1e-4
    by_difference = (loss(h) - loss(-h)) / (2 * h)
    parts = [(dX[:M].double() * vx).sum(), (G[:, gain:gain + C].double() * vp[:, gain:gain + C]).sum(), (G[:, at:at + C].double() * vp[:, at:at + C]).sum()]
    size = (dX[:M].double() * vx).abs().sum() + (G.double()[:, gain:at + C] * vp[:, gain:at + C]).nan_to_num().abs().sum()
    # 1e-6: entries are off by less than 80 u of terms a few times their size; h^2 = 1e-8 of derivatives of order one
    assert abs(by_difference - sum(p.item() for p in parts)) <= 1e-6 * size.item() + 1e-6 * abs(by_difference)

"""Per-worker products, cross-entropy and AdamW against plain implementations in 64 bits.

Tolerances.  A sum of K fp32 products of given operands, in any order, is off by at most (K + 8) 2^-24 times the sum of the
products' magnitudes (one rounding per addition; the matrix cores add a few terms at a time); a bf16 result adds half a spacing, at most
2^-8 of itself.  exp and log of the hardware are within 2^-22 of their argument's scale: relative 2^-20 for a softmax of logits below 64 in
magnitude, plus the sum's roundings.  The fp32 bounds are doubled."""
import numpy as np
import pytest
import torch

import paper_2006_08085_amd as D

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2006_08085_amd.build import ensure_built
    ensure_built()
    assert torch.cuda.is_available(), "these tests need the GPU"


def _context(n, d, ld=None, dtype=D.DETAG_F32):
    return D.detag_create(D.Topology.ring(), n, d, D.padded_ld(d) if ld is None else ld, dtype)


def _offsets(counts, first=0):
    return torch.tensor(np.concatenate([[first], first + np.cumsum(counts)]), dtype=torch.int32, device=DEV)


def _rows_matrix(M, cols, dtype, seed, pitch=None, shift=0, scale=1.0, fill=float("nan")):
    """An M x cols view with the given pitch, its first element `shift` elements into the allocation; all around is `fill`."""
    pitch = cols if pitch is None else pitch
    g = torch.Generator().manual_seed(seed)
    buf = torch.full((shift + M * pitch + 64,), fill, dtype=dtype)
    view = buf[shift:shift + M * pitch].view(M, pitch)
    view[:, :cols] = (scale * torch.randn(M, cols, generator=g)).to(dtype)
    buf = buf.to(DEV)
    return buf[shift:shift + M * pitch].view(M, pitch)[:, :cols] if M else torch.empty(0, cols, dtype=dtype, device=DEV), buf


def _weights(n, ld, offset, out, inn, dtype, seed):
    """n x ld with the layer's weights from `offset` on and NaN elsewhere."""
    g = torch.Generator().manual_seed(seed)
    W = torch.full((n, ld), float("nan"), dtype=dtype)
    W[:, offset:offset + out * inn] = (inn ** -0.5 * torch.randn(n, out * inn, generator=g)).to(dtype)
    return W.to(DEV)


def _close(got, ref, magnitude, K, what):
    """Entry by entry: roundings of the sum, and of the result's type."""
    got, ref = got.double(), ref.double()
    bound = 2 * (K + 8) * 2.0 ** -24 * magnitude + (2.0 ** -8 * ref.abs() if what is BF16 else 2 * 2.0 ** -24 * ref.abs()) + 1e-37
    off = (got - ref).abs()
    assert torch.isfinite(got).all()
    assert (off <= bound).all(), f"worst {float((off / bound).max()):.3g} of the bound"


# worker's rows | in | out | first column | pitches beyond the rows | elements before the first | operands
LAYERS = [
    ([1, 1, 1], 64, 64, 0, 0, 0, BF16),                       # one sample each, whole pieces
    ([1], 1, 1, 0, 0, 0, F32), ([3, 0, 2], 1, 5, 3, 0, 0, BF16), ([2, 1], 7, 1, 1, 1, 1, F32),
    ([0, 0, 0], 40, 24, 0, 0, 0, BF16),                       # nobody has any
    ([5, 0, 130, 0, 1, 127, 128, 129], 128, 96, 8, 0, 0, BF16),
    ([5, 0, 130, 0, 1, 127, 128, 129], 100, 136, 4, 0, 0, F32),
    ([257, 3, 0, 300], 264, 520, 16, 8, 8, BF16),             # more than one tile each way, pitches of whole pieces
    ([257, 3, 0, 300], 132, 260, 4, 4, 4, F32),
    ([33, 64, 65], 77, 131, 5, 3, 1, BF16),                   # nothing on a piece
    ([33, 64, 65], 77, 131, 5, 3, 1, F32),
    ([200, 100], 8, 8, 0, 0, 0, BF16), ([200, 100], 520, 8, 0, 0, 0, BF16), ([16] * 70, 72, 40, 0, 0, 0, BF16),
    ([17, 1, 15, 16, 30], 1032, 200, 0, 0, 0, BF16), ([2, 9, 1, 4], 333, 515, 7, 5, 3, BF16), ([2, 9, 1, 4], 512, 384, 0, 0, 0, F32),
    ([700, 900], 384, 640, 0, 0, 0, BF16),
]


def _ids(c):
    return f"{len(c[0])}x{sum(c[0])}-{c[1]}-{c[2]}-{c[3]}-{c[4]}-{c[5]}-{'bf16' if c[6] is BF16 else 'f32'}"


def _spans(counts):
    at = 0
    for i, c in enumerate(counts):
        yield i, at, at + c
        at += c


@pytest.mark.parametrize("case", LAYERS, ids=_ids)
@pytest.mark.parametrize("relu,wide", [(False, False), (True, True)])
def test_linear(case, relu, wide):
    counts, inn, out, offset, extra, shift, dtype = case
    n, M = len(counts), sum(counts)
    spare = 2  # rows that nobody owns, at the end
    ld = offset + inn * out + 5 if extra else D.padded_ld(offset + inn * out)
    ctx = _context(n, offset + inn * out, ld)
    W = _weights(n, ld, offset, out, inn, dtype, 1)
    A, _ = _rows_matrix(M + spare, inn, dtype, 2, inn + extra, shift)
    A[M:] = float("nan")
    y_type = F32 if wide else dtype
    Y, Ybuf = _rows_matrix(M + spare, out, y_type, 3, out + extra, shift, fill=7.0)
    before = Ybuf.clone()
    ctx.linear(W, offset, A, _offsets(counts), Y, relu=relu)
    torch.cuda.synchronize()
    for i, lo, hi in _spans(counts):
        Wi, a = W[i, offset:offset + inn * out].double().view(out, inn), A[lo:hi].double()
        ref = a @ Wi.t()
        _close(Y[lo:hi], ref.clamp(min=0) if relu else ref, a.abs() @ Wi.abs().t(), inn, y_type)
    Y[:M] = before[shift:shift + (M + spare) * (out + extra)].view(M + spare, out + extra)[:M, :out]  # nothing else was written
    assert torch.equal(Ybuf, before)


@pytest.mark.parametrize("case", LAYERS, ids=_ids)
@pytest.mark.parametrize("masked", [False, True])
def test_linear_grad_input(case, masked):
    counts, inn, out, offset, extra, shift, dtype = case
    n, M = len(counts), sum(counts)
    ld = offset + inn * out + 5 if extra else D.padded_ld(offset + inn * out)
    ctx = _context(n, offset + inn * out, ld)
    W = _weights(n, ld, offset, out, inn, dtype, 1)
    dY, _ = _rows_matrix(M + 2, out, dtype, 2, out + extra, shift)
    dY[M:] = float("nan")
    H, _ = _rows_matrix(M + 2, inn, dtype, 4, inn + extra, shift)
    H.clamp_(min=0)
    dA, buf = _rows_matrix(M + 2, inn, dtype, 3, inn + extra, shift, fill=7.0)
    before = buf.clone()
    ctx.linear_grad_input(W, offset, dY, _offsets(counts), dA, relu_of=H if masked else None)
    torch.cuda.synchronize()
    for i, lo, hi in _spans(counts):
        Wi, dy = W[i, offset:offset + inn * out].double().view(out, inn), dY[lo:hi].double()
        keep = (H[lo:hi] > 0).double() if masked else 1.0
        _close(dA[lo:hi], (dy @ Wi) * keep, (dy.abs() @ Wi.abs()) * keep, out, dtype)
    dA[:M] = before[shift:shift + (M + 2) * (inn + extra)].view(M + 2, inn + extra)[:M, :inn]
    assert torch.equal(buf, before)


@pytest.mark.parametrize("case", LAYERS, ids=_ids)
@pytest.mark.parametrize("accumulate", [False, True])
def test_linear_grad_weight(case, accumulate):
    counts, inn, out, offset, extra, shift, dtype = case
    n, M = len(counts), sum(counts)
    ld = offset + inn * out + 5 if extra else D.padded_ld(offset + inn * out)
    ctx = _context(n, offset + inn * out, ld)
    dY, _ = _rows_matrix(M + 2, out, dtype, 2, out + extra, shift)
    A, _ = _rows_matrix(M + 2, inn, dtype, 3, inn + extra, shift)
    dY[M:], A[M:] = float("nan"), float("nan")
    G = torch.randn(n, ld, generator=torch.Generator().manual_seed(5)).to(DEV)
    before = G.clone()
    ctx.linear_grad_weight(dY, A, _offsets(counts), G, offset, accumulate=accumulate)
    torch.cuda.synchronize()
    here = slice(offset, offset + inn * out)
    for i, lo, hi in _spans(counts):
        dy, a = dY[lo:hi].double(), A[lo:hi].double()
        start = before[i, here].double().view(out, inn) if accumulate else torch.zeros(out, inn, dtype=torch.float64, device=DEV)
        _close(G[i, here].view(out, inn), start + dy.t() @ a, start.abs() + dy.abs().t() @ a.abs(), hi - lo, F32)
    G[:, here] = before[:, here]
    assert torch.equal(G, before)


@pytest.mark.parametrize("n,M,inn,out", [(8, 3600, 1544, 2056), (3, 9000, 1000, 2056), (64, 7000, 200, 520), (9, 1200, 1544, 1288), (70, 9000, 72, 264)],
                         ids=["256-many", "256-few", "128-many", "128-few", "70-workers"])
def test_products_of_every_tile(n, M, inn, out):
    """Calls with enough tiles for the larger ones (bf16, rows of whole pieces): uneven workers, tiles that few rows fill, contractions
    that end inside a step."""
    rng = np.random.default_rng(n)
    share = rng.dirichlet(np.full(n, 0.5))
    counts = np.floor(share * M).astype(int)
    counts[-1] += M - counts.sum()
    counts = counts.tolist()
    d = inn * out
    ctx, rows = _context(n, d), _offsets(counts)
    W = _weights(n, D.padded_ld(d), 0, out, inn, BF16, 1)
    A, _ = _rows_matrix(M, inn, BF16, 2)
    A.clamp_(min=0)
    dY, _ = _rows_matrix(M, out, BF16, 3)
    Y, dA = torch.zeros(M, out, dtype=BF16, device=DEV), torch.zeros(M, inn, dtype=BF16, device=DEV)
    G = torch.zeros(n, D.padded_ld(d), device=DEV)
    ctx.linear(W, 0, A, rows, Y, relu=True)
    ctx.linear_grad_input(W, 0, dY, rows, dA, relu_of=A)
    ctx.linear_grad_weight(dY, A, rows, G, 0)
    torch.cuda.synchronize()
    for i, lo, hi in _spans(counts):
        w, a, dy = W[i, :d].double().view(out, inn), A[lo:hi].double(), dY[lo:hi].double()
        _close(Y[lo:hi], (a @ w.t()).clamp(min=0), a @ w.abs().t(), inn, BF16)
        _close(dA[lo:hi], (dy @ w) * (a > 0), (dy.abs() @ w.abs()) * (a > 0), out, BF16)
        _close(G[i, :d].view(out, inn), dy.t() @ a, dy.abs().t() @ a, hi - lo, F32)


def test_a_worker_sees_nothing_of_the_others():
    """Infinities and NaN in one worker's rows and weights stay with that worker, and max(0, NaN) is NaN."""
    counts, inn, out = [40, 33, 7, 64], 72, 200
    ctx, rows = _context(4, inn * out), _offsets([40, 33, 7, 64])
    for dtype in (BF16, F32):
        W = _weights(4, D.padded_ld(inn * out), 0, out, inn, dtype, 1)
        A, _ = _rows_matrix(sum(counts), inn, dtype, 2)
        dY, _ = _rows_matrix(sum(counts), out, dtype, 3)
        A[40:73], dY[40:73], W[1] = float("nan"), float("inf"), float("nan")
        Y, dA = torch.zeros(sum(counts), out, dtype=dtype, device=DEV), torch.zeros(sum(counts), inn, dtype=dtype, device=DEV)
        G = torch.zeros(4, D.padded_ld(inn * out), device=DEV)
        ctx.linear(W, 0, A, rows, Y, relu=True)
        ctx.linear_grad_input(W, 0, dY, rows, dA)
        ctx.linear_grad_weight(dY, A, rows, G, 0)
        torch.cuda.synchronize()
        other = torch.ones(sum(counts), dtype=torch.bool, device=DEV)
        other[40:73] = False
        assert torch.isfinite(Y[other]).all() and torch.isnan(Y[~other]).all()
        assert torch.isfinite(dA[other]).all() and torch.isnan(dA[~other]).all()
        assert torch.isfinite(G[[0, 2, 3]]).all() and torch.isnan(G[1, :inn * out]).all()


def test_the_same_bits_again_and_on_another_stream():
    counts, inn, out = [300, 0, 45, 260], 520, 264
    ctx, rows = _context(4, inn * out), _offsets(counts)
    W = _weights(4, D.padded_ld(inn * out), 0, out, inn, BF16, 1)
    A, _ = _rows_matrix(sum(counts), inn, BF16, 2)
    dY, _ = _rows_matrix(sum(counts), out, BF16, 3)
    labels = torch.randint(out, (sum(counts),), dtype=torch.int32, device=DEV)

    def once():
        Y, dA = torch.empty(sum(counts), out, device=DEV), torch.empty(sum(counts), inn, dtype=BF16, device=DEV)
        G, loss = torch.zeros(4, D.padded_ld(inn * out), device=DEV), torch.empty(4, device=DEV)
        ctx.linear(W, 0, A, rows, Y)
        ctx.linear_grad_input(W, 0, dY, rows, dA)
        ctx.linear_grad_weight(dY, A, rows, G, 0)
        ctx.cross_entropy(Y, labels, rows, Y, loss)
        return Y, dA, G, loss
    first = once()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = once()
    side.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(first, second))


def test_recorded_into_a_graph():
    """A forward and backward pass and a step, replayed several times with other work between, against the same done eagerly."""
    counts, inn, out = [30, 12], 64, 40
    d = inn * out
    ctx, rows = _context(2, d), _offsets(counts)
    ctx.reserve_cross_entropy(sum(counts))
    opt = D.AdamW(ctx, [(0, d)], bits=8)
    A, _ = _rows_matrix(sum(counts), inn, BF16, 2)
    labels = torch.randint(out, (sum(counts),), dtype=torch.int32, device=DEV)

    def state():
        X = _weights(2, D.padded_ld(d), 0, out, inn, F32, 1).nan_to_num(0.0)
        return dict(X=X, X16=X.to(BF16), G=torch.zeros_like(X), Y=torch.zeros(sum(counts), out, device=DEV), m=opt.new_moments(),
                    dY=torch.zeros(sum(counts), out, dtype=BF16, device=DEV), loss=torch.zeros(2, device=DEV))

    def step(s):
        ctx.linear(s["X16"], 0, A, rows, s["dY"])
        ctx.cross_entropy(s["dY"], labels, rows, s["dY"], s["loss"])
        ctx.linear_grad_weight(s["dY"], A, rows, s["G"], 0)
        opt.step(s["X"], s["G"], *s["m"], lr=0.01, t=3, limit=4.0, X16=s["X16"])
    eager, recorded = state(), state()
    step(state())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(recorded)
    for _ in range(4):
        step(eager)
        graph.replay()
        torch.randn(1000, device=DEV).sum().item()
        assert torch.equal(eager["X"], recorded["X"]) and torch.equal(eager["loss"], recorded["loss"])
        assert all(torch.equal(x, y) for x, y in zip(eager["m"], recorded["m"]))


# ---------------------------------------------------------------- cross-entropy

def _xent_reference(z, labels, counts, C):
    z = z.double()
    loss, grad = torch.zeros(len(counts), dtype=torch.float64), torch.zeros_like(z)
    for i, lo, hi in _spans(counts):
        ok = [r for r in range(lo, hi) if 0 <= int(labels[r]) < C]
        for r in ok:
            p = torch.softmax(z[r], 0)
            loss[i] += (torch.logsumexp(z[r], 0) - z[r, int(labels[r])]) / len(ok)
            p[int(labels[r])] -= 1
            grad[r] = p / len(ok)
    return loss, grad


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("counts,C,extra,shift", [
    ([4], 1, 0, 0), ([3, 0, 5], 2, 0, 0), ([1, 1, 1], 10, 0, 0), ([64, 128, 1], 10, 6, 0), ([5, 4], 15, 1, 1), ([5, 4], 16, 0, 0), ([5, 4], 17, 2, 3),
    ([9, 2], 63, 0, 0), ([9, 2], 64, 0, 8), ([9, 300], 65, 0, 0), ([7, 1], 257, 0, 1), ([3, 2], 1000, 8, 0), ([2, 3], 2049, 0, 0), ([2, 1], 4099, 5, 2),
    ([1, 2], 8192, 0, 0), ([1, 2], 16385, 0, 0), ([2, 1], 32000, 0, 0), ([1, 1], 40001, 0, 1), ([1, 1], 65537, 0, 0), ([1, 1], 131073, 0, 0), ([1], 300007, 0, 0)])
def test_cross_entropy(counts, C, extra, shift, dtype):
    n, M = len(counts), sum(counts)
    ctx = _context(n, 4)
    z, _ = _rows_matrix(M + 1, C, dtype, C, C + extra, shift, scale=3.0)
    g, buf = _rows_matrix(M + 1, C, dtype, 9, C + extra, shift, fill=7.0)
    before = buf.clone()
    labels = torch.randint(C, (M + 1,), generator=torch.Generator().manual_seed(C), dtype=torch.int32)
    if M > 3:
        labels[1], labels[M - 1] = -100, C
    loss = torch.full((n,), 5.0, device=DEV)
    ctx.cross_entropy(z, labels.to(DEV), _offsets(counts), g, loss)
    torch.cuda.synchronize()
    ref_loss, ref = _xent_reference(z[:M].cpu(), labels, counts, C)
    got = g[:M].cpu().double()
    most = max([c for c in counts if c], default=1)
    tol = 2 * (2.0 ** -20 + C / 64 * 2.0 ** -24)     # relative, of p; p - 1 cancels near p = 1: absolute there
    bound = tol * ref.abs().clamp(min=0) + tol / 1.0 * (ref < 0) + (2.0 ** -8 * ref.abs() if dtype is BF16 else 0) + 1e-37
    assert ((got - ref).abs() <= bound).all()
    assert torch.allclose(loss.cpu().double(), ref_loss, rtol=2e-6, atol=2e-5 * min(1, most))
    g[:M] = before[shift:shift + (M + 1) * (C + extra)].view(M + 1, C + extra)[:M, :C]
    assert torch.equal(buf, before)                  # rows without an owner, and what lies between rows
    copy = z[:M].clone()
    ctx.cross_entropy(copy, labels[:M].to(DEV), _offsets(counts), copy)
    torch.cuda.synchronize()
    assert torch.equal(copy.cpu().double(), got)     # in place, without the loss


@pytest.mark.parametrize("counts,C,dtype", [([700, 0, 500], 30001, F32), ([1000, 600], 50000, BF16), ([3000], 12, F32), ([6000, 1, 12000], 90, BF16)],
                         ids=["stream-f32", "stream-bf16", "one-worker", "many-rows"])
def test_cross_entropy_of_many_rows(counts, C, dtype):
    n, M = len(counts), sum(counts)
    ctx, rows = _context(n, 4), _offsets(counts)
    g = torch.Generator(device=DEV).manual_seed(1)
    z = torch.randn(M, C, generator=g, device=DEV).to(dtype)
    labels = torch.randint(-1, C, (M,), generator=g, device=DEV, dtype=torch.int32)
    grad, loss = torch.empty_like(z), torch.empty(n, device=DEV)
    ctx.cross_entropy(z, labels, rows, grad, loss)
    tol = 2 * (2.0 ** -20 + C / 64 * 2.0 ** -24)
    for i, lo, hi in _spans(counts):
        if hi == lo:
            assert float(loss[i]) == 0.0
            continue
        ok = labels[lo:hi] >= 0
        total = torch.zeros((), dtype=torch.float64, device=DEV)
        for a in range(lo, hi, 500):  # a few rows at a time: 64 bits
            b = min(a + 500, hi)
            logp = torch.log_softmax(z[a:b].double(), 1)
            at = labels[a:b].clamp(min=0).long()[:, None]
            total -= (logp.gather(1, at)[:, 0] * (labels[a:b] >= 0)).sum()
            ref = logp.exp_()
            ref.scatter_add_(1, at, torch.full_like(at, -1, dtype=torch.float64))
            ref *= ((labels[a:b] >= 0).double() / ok.sum())[:, None]
            off = (grad[a:b].double() - ref).abs()
            assert (off <= tol * ref.abs() + tol * (ref < 0) / float(ok.sum()) + (2.0 ** -8 * ref.abs() if dtype is BF16 else 0) + 1e-37).all()
        assert abs(float(loss[i]) - float(total / ok.sum())) < 2e-6 * max(1.0, float(loss[i]))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("C", [10, 100, 3000, 70001])
def test_cross_entropy_of_masked_and_broken_logits(C, dtype):
    inf, nan = float("inf"), float("nan")
    ctx = _context(3, 4)
    z = torch.randn(7, C, generator=torch.Generator().manual_seed(1)).to(dtype)
    low = torch.finfo(dtype).min
    z[0, 1:] = -inf                 # one class left, the label's
    z[1, ::2] = -inf                # half the classes masked
    z[2] = low                      # masks of the type's lowest value everywhere: uniform
    z[3, 4], z[4, 3], z[5] = nan, inf, -inf
    labels = torch.tensor([0, 1, 2, 3, 0, 0, -1], dtype=torch.int32)
    g, loss = torch.zeros(7, C, dtype=dtype, device=DEV), torch.zeros(3, device=DEV)
    ctx.cross_entropy(z.to(DEV), labels.to(DEV), _offsets([3, 3, 1]), g, loss)
    torch.cuda.synchronize()
    g, loss = g.cpu().double(), loss.cpu().double()
    p0, p1 = torch.zeros(C).double(), torch.softmax(z[1].double(), 0)
    p1[1] -= 1
    assert torch.equal(g[0], p0)
    tol = 2.0 ** -8 if dtype is BF16 else 1e-5
    assert torch.allclose(g[1], p1 / 3, rtol=tol, atol=1e-7) and (g[1][::2] == 0).all()
    u = torch.full((C,), 1.0 / C).double()
    u[2] -= 1
    assert torch.allclose(g[2], u / 3, rtol=tol, atol=1e-7)
    assert torch.isnan(g[3:6]).all() and (g[6] == 0).all()
    ref = (torch.logsumexp(z[1].double(), 0) - z[1, 1].double() + np.log(C)) / 3
    assert abs(float(loss[0] - ref)) < 1e-4 * max(1.0, float(ref))
    assert torch.isnan(loss[1]) and float(loss[2]) == 0.0


def test_the_gradient_of_a_network_is_that_of_its_loss():
    """Two layers, relu and cross-entropy in fp32 against central differences of the loss along random directions."""
    counts, sizes = [20, 7, 0, 33], (24, 40, 11)
    n, M = len(counts), sum(counts)
    d1, d = sizes[0] * sizes[1], sizes[0] * sizes[1] + sizes[1] * sizes[2]
    ctx, rows = _context(n, d, d), _offsets(counts)
    g = torch.Generator().manual_seed(3)
    X = (0.3 * torch.randn(n, d, generator=g)).to(DEV)
    A = torch.randn(M, sizes[0], generator=g).to(DEV)
    labels = torch.randint(sizes[2], (M,), generator=g, dtype=torch.int32).to(DEV)
    H, Z = torch.empty(M, sizes[1], device=DEV), torch.empty(M, sizes[2], device=DEV)
    dZ, dH, G, loss = torch.empty_like(Z), torch.empty_like(H), torch.zeros(n, d, device=DEV), torch.zeros(n, device=DEV)

    def forward(P):
        ctx.linear(P, 0, A, rows, H, relu=True)
        ctx.linear(P, d1, H, rows, Z)
    forward(X)
    ctx.cross_entropy(Z, labels, rows, dZ, loss)
    ctx.linear_grad_weight(dZ, H, rows, G, d1)
    ctx.linear_grad_input(X, d1, dZ, rows, dH, relu_of=H)
    ctx.linear_grad_weight(dH, A, rows, G, 0)

    def losses(P):  # in 64 bits
        out = []
        for i, lo, hi in _spans(counts):
            h = (A[lo:hi].double() @ P[i, :d1].view(sizes[1], sizes[0]).t()).clamp(min=0)
            z = h @ P[i, d1:].view(sizes[2], sizes[1]).t()
            out.append(-torch.log_softmax(z, 1)[torch.arange(hi - lo), labels[lo:hi].long()].mean() if hi > lo else z.new_zeros(()))
        return torch.stack(out)
    assert torch.allclose(loss.double(), losses(X.double()), rtol=1e-5, atol=1e-6)
    for seed in range(4):
        v = torch.randn(n, d, generator=torch.Generator().manual_seed(seed), dtype=torch.float64).to(DEV)
        h = 1e-6  # second-order error h^2, roundings of 64 bits 1e-16 / h; kinks of relu are crossed with probability about 1e-4
        slope = (losses(X.double() + h * v) - losses(X.double() - h * v)) / (2 * h)
        along = (G.double() * v).sum(1)
        assert torch.allclose(along, slope, rtol=1e-4, atol=1e-4)


# ---------------------------------------------------------------- AdamW

def _tensors(d, cuts):
    at = [0, *cuts, d]
    return [(a, b - a) for a, b in zip(at, at[1:])]


@pytest.mark.parametrize("state", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,d,cuts,ld", [(1, 1, [], 1), (3, 700, [256, 300, 301], 704), (2, 1031, [3, 7, 500], 1031), (5, 5000, [4096], 5056),
                                         (300, 40, [17], 64)])
def test_adamw_in_32_bits(n, d, cuts, ld, state):
    ctx = _context(n, d, ld, D.DETAG_BF16 if state is BF16 else D.DETAG_F32)
    spans = _tensors(d, cuts)
    if len(spans) > 2:
        del spans[1]                                  # columns of no tensor
    decay, factor = [0.1 * k for k in range(len(spans))], [1.0 / (k + 1) for k in range(len(spans))]
    opt = D.AdamW(ctx, spans, decay, factor)
    g = torch.Generator().manual_seed(d)
    X = torch.randn(n, ld, generator=g).to(state).to(DEV)
    M, V, S = opt.new_moments(DEV)
    assert S is None
    copy = torch.full((n, ld), 3.0, dtype=BF16, device=DEV)
    inside = torch.zeros(ld, dtype=torch.bool)
    w, s = torch.zeros(ld, dtype=torch.float64), torch.zeros(ld, dtype=torch.float64)
    for k, (a, length) in enumerate(spans):
        inside[a:a + length], w[a:a + length], s[a:a + length] = True, decay[k], factor[k]
    m, v = torch.zeros(n, ld).double(), torch.zeros(n, ld).double()
    start = X.clone()
    lr, b1, b2, eps = 0.02, 0.8, 0.99, 1e-6
    for t in range(1, 4):
        G = torch.randn(n, ld, generator=g)
        G[:, ::5] = 0.0
        x = X.cpu().double()                          # from the stored model: a step rounds it once, by half a spacing (2^-8 in bf16)
        opt.step(X, G.to(DEV), M, V, lr=lr, t=t, beta1=b1, beta2=b2, eps=eps, X16=copy)
        m, v = b1 * m + (1 - b1) * G.double(), b2 * v + (1 - b2) * G.double() ** 2
        x = x * (1 - lr * s * w) - lr * s * (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + eps)
        assert torch.allclose(X.cpu().double()[:, inside], x[:, inside], rtol=2e-6 + (2.0 ** -8 if state is BF16 else 0.0), atol=2e-7)
    assert torch.allclose(M.cpu().double()[:, inside], m[:, inside], rtol=1e-6, atol=1e-7)
    assert torch.allclose(V.cpu().double()[:, inside], v[:, inside], rtol=1e-6, atol=1e-12)
    assert torch.equal(X[:, ~inside.to(DEV)], start[:, ~inside.to(DEV)]) and (M.cpu()[:, ~inside] == 0).all()
    assert torch.equal(copy[:, inside.to(DEV)], X[:, inside.to(DEV)].to(BF16)) and (copy.cpu()[:, ~inside] == 3).all()


def test_adamw_of_models_that_stream():
    """Moments beyond the memory-side cache, odd tensors."""
    n, d = 3, 4_000_003
    ctx = _context(n, d)
    opt = D.AdamW(ctx, _tensors(d, [1001, 2_500_000, 2_500_001]), [0.1] * 4)
    g = torch.Generator(device=DEV).manual_seed(1)
    X, G, M = (torch.randn(n, ctx.ld, generator=g, device=DEV) for _ in range(3))
    V = torch.rand(n, ctx.ld, generator=g, device=DEV)
    x, m, v = X.double(), 0.9 * M.double() + 0.1 * G.double(), 0.999 * V.double() + 0.001 * G.double() ** 2
    opt.step(X, G, M, V, lr=0.01, t=7)
    x = x * (1 - 0.01 * 0.1) - 0.01 * (m / (1 - 0.9 ** 7)) / ((v / (1 - 0.999 ** 7)).sqrt() + 1e-8)
    for got, ref in ((X, x), (M, m), (V, v)):
        assert torch.allclose(got[:, :d].double(), ref[:, :d], rtol=2e-6, atol=2e-7)


def _philox(blocks, worker, t, seed):
    """The words of a worker's columns, (blocks, 256), from the generator's definition."""
    mask, out = np.uint64(0xFFFFFFFF), []
    c = [np.arange(blocks * 64, dtype=np.uint64), np.full(blocks * 64, 0x41646157, np.uint64), np.full(blocks * 64, worker, np.uint64),
         np.full(blocks * 64, t, np.uint64)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), p1 & mask, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), p0 & mask]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(c, 1).reshape(blocks, 256)


def _codes(x, r, bias):
    """Codes and exponent of a block (fp32 values, 16-bit random numbers) from the description in the header."""
    mag = np.abs(x.astype(np.float64))
    ok = np.isfinite(x)
    E = max(16, (np.max(np.where(ok, mag, 0)).astype(np.float32).view(np.int32) >> 23).item())
    y = np.where(ok, mag, 0) * 2.0 ** ((134 if bias == 7 else 142) - E)
    e = np.maximum(np.floor(np.log2(np.maximum(y, 1e-300))), 1 - bias)
    steps = np.floor(y / 2.0 ** (e - 3) + r / 65536.0)            # in units of the spacing at y
    code = np.where(y < 2.0 ** (1 - bias), steps, steps - 8 + 8 * (e + bias))
    code = np.where(ok, code, 127 if bias == 7 else 255).astype(np.int64)
    return code + (128 * np.signbit(x) if bias == 7 else 0), E


def _value(code, E, bias):
    mag = code % 128 if bias == 7 else code
    y = np.where(mag < 8, mag * 2.0 ** (-bias - 2), (1 + (mag % 8) / 8) * 2.0 ** (mag // 8 - bias)) * 2.0 ** (E - (134 if bias == 7 else 142))
    y = np.where(mag == (127 if bias == 7 else 255), np.nan, y)
    return np.where(code >= 128, -y, y) if bias == 7 else y


@pytest.mark.parametrize("state", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,d,cuts,ld", [(1, 1, [], 1), (3, 700, [256, 300, 301], 704), (2, 1031, [3, 7, 500], 1031), (4, 5000, [4096], 5056)])
def test_adamw_in_8_bits(n, d, cuts, ld, state):
    """Codes and scales bit by bit, with a moment arithmetic that is rounded operation by operation in fp32; the models to fp32's roundings."""
    ctx = _context(n, d, ld, D.DETAG_BF16 if state is BF16 else D.DETAG_F32)
    spans = _tensors(d, cuts)
    if len(spans) > 2:
        del spans[1]
    opt = D.AdamW(ctx, spans, [0.1] * len(spans), bits=8)
    assert opt.blocks == sum(-(-length // 256) for _, length in spans)
    rng = np.random.default_rng(d)
    X = torch.tensor(rng.standard_normal((n, ld)), dtype=state).to(DEV)
    M, V, S = opt.new_moments(DEV)
    seed, lr, b1, b2, eps, f = (1 << 40) + 77, 0.02, 0.9, 0.999, 1e-6, np.float32
    for t in range(1, 4):
        G = (rng.standard_normal((n, ld)) * np.exp(3 * rng.standard_normal((1, ld)))).astype(f)
        G[:, ::7] = 0
        before, was = (M.cpu().numpy(), V.cpu().numpy(), S.cpu().numpy()), X.cpu().double().numpy()
        opt.step(X, torch.tensor(G).to(DEV), M, V, S, lr=lr, t=t, beta1=b1, beta2=b2, eps=eps, seed=seed)
        torch.cuda.synchronize()
        now, x = (M.cpu().numpy(), V.cpu().numpy(), S.cpu().numpy()), X.cpu().double().numpy()
        for i in range(n):
            words, b = _philox(opt.blocks, i, t, seed), 0
            for a, length in spans:
                for c in range(a, a + length, 256):
                    k = slice(c, min(c + 256, a + length))
                    count = k.stop - k.start
                    m, v = (_value(before[j][i, k].astype(np.int64), int(before[2][i, 2 * b + j]) or 16, bias).astype(f) for j, bias in ((0, 7), (1, 15)))
                    m = m * f(b1) + G[i, k] * f(1 - b1)
                    v = v * f(b2) + G[i, k] * G[i, k] * f(1 - b2)
                    for j, (val, bias, r) in enumerate(((m, 7, words[b, :count] & np.uint64(0xFFFF)), (v, 15, words[b, :count] >> np.uint64(16)))):
                        code, E = _codes(val, r.astype(np.float64), bias)
                        assert int(now[2][i, 2 * b + j]) == E
                        # fp32 holds 2^9 y + 2^-16 r exactly up to 24 bits: a denormal code may differ where that is a near tie
                        off = now[j][i, k].astype(np.int64) - code
                        assert (off == 0).mean() > 0.99 and np.abs(off).max() <= 1 if count > 64 else np.abs(off).max() <= 1
                    want = was[i, k] * (1 - lr * 0.1) - lr * (m.astype(np.float64) / (1 - b1 ** t)) / (np.sqrt(v.astype(np.float64) / (1 - b2 ** t)) + eps)
                    assert np.allclose(x[i, k], want, rtol=2.0 ** -8 if state is BF16 else 2e-6, atol=2e-6)
                    b += 1
    values = [torch.full((n, ld), 3.0, dtype=dt, device=DEV) for dt in (F32, F32, BF16, BF16)]
    opt.values(M, V, S, *values[:2])
    opt.values(M, V, S, *values[2:])
    torch.cuda.synchronize()
    assert torch.equal(values[0], values[2].float()) and torch.equal(values[1], values[3].float())
    b = 0
    for a, length in spans:
        for c in range(a, a + length, 256):
            k = slice(c, min(c + 256, a + length))
            for j, bias in ((0, 7), (1, 15)):
                got, code, E = values[j].cpu().double().numpy()[0, k], (M, V)[j].cpu().numpy()[0, k].astype(np.int64), int(S[0, 2 * b + j])
                assert np.array_equal(got, _value(code, E, bias))
            b += 1
    if len(spans) > 2:
        hole = slice(spans[0][0] + spans[0][1], spans[1][0])
        assert (M[:, hole] == 0).all() and (values[0][:, hole] == 3).all()


def test_rounding_to_8_bits_is_right_on_average():
    """A v that moves by a thousandth a step, far below the spacing of its codes, follows the exact one on average."""
    n, d, T = 8, 4096, 400
    ctx = _context(n, d)
    opt = D.AdamW(ctx, [(0, d)], bits=8)
    M, V, S = opt.new_moments(DEV)
    X = D.new_matrix(n, d, device=DEV)
    G = torch.rand(n, d, generator=torch.Generator().manual_seed(1)).to(DEV) + 0.5
    for t in range(1, T + 1):
        opt.step(X, G, M, V, S, lr=1e-3, t=t, seed=5)
    m, v = torch.empty(n, d, device=DEV), torch.empty(n, d, device=DEV)
    opt.values(M, V, S, m, v)
    ratio = (v / (G * G * (1 - 0.999 ** T))).double()
    # a code's spacing is at most 1/8 of it, so a step's variance at most 1/8 * 1/1000 * v^2 and the sum's a third of v^2 here: the
    # mean over 32,768 columns is within 5 * 0.6 / 181 of one
    assert abs(float(ratio.mean()) - 1) < 0.02
    assert abs(float((m / (G * (1 - 0.9 ** T))).double().mean()) - 1) < 0.02


def test_what_is_not_finite_stays_where_it_is():
    n, d = 2, 600
    ctx = _context(n, d)
    for bits in (8, 32):
        opt = D.AdamW(ctx, [(0, d)], bits=bits)
        moments = opt.new_moments(DEV)
        X, clean = D.new_matrix(n, d, device=DEV), D.new_matrix(n, d, device=DEV)
        G = torch.randn(n, D.padded_ld(d), generator=torch.Generator().manual_seed(1)).to(DEV)
        opt.step(clean, G, *opt.new_moments(DEV), lr=0.1, t=1, seed=3)
        G[0, 5], G[1, 300], G[1, 599] = float("nan"), float("inf"), -float("inf")
        opt.step(X, G, *moments, lr=0.1, t=1, seed=3)
        torch.cuda.synchronize()
        broken = torch.zeros(n, d, dtype=torch.bool, device=DEV)
        broken[0, 5] = broken[1, 300] = broken[1, 599] = True
        assert torch.isnan(X[:, :d][broken]).all() and torch.equal(X[:, :d][~broken], clean[:, :d][~broken])
        if bits == 8:
            values = [D.new_matrix(n, d, device=DEV) for _ in range(2)]
            opt.values(*moments, *values)
            assert all(torch.isnan(v[:, :d][broken]).all() and torch.isfinite(v[:, :d][~broken]).all() for v in values)


def test_the_limit_holds_a_step_whose_second_moment_was_lost():
    n, d = 1, 256
    ctx = _context(n, d)
    opt = D.AdamW(ctx, [(0, d)], bits=8)
    M, V, S = opt.new_moments(DEV)
    M[0, :2], S[0, 0] = 120, 127          # m of order one over a v of zero
    X, G = D.new_matrix(n, d, device=DEV), D.new_matrix(n, d, device=DEV)
    other = [t.clone() for t in (X, M, V, S)]
    opt.step(other[0], G, *other[1:], lr=0.5, t=1000)
    opt.step(X, G, M, V, S, lr=0.5, t=1000, limit=4.0)
    torch.cuda.synchronize()
    assert float(other[0][0, 0]) < -1e6 and float(X[0, 0]) == -2.0 and float(X[0, 2]) == 0.0


# ---------------------------------------------------------------- refusals

def test_refusals():
    n, inn, out, M = 3, 16, 8, 12
    d = inn * out
    ctx, rows = _context(n, d), _offsets([4, 4, 4])
    W, G = D.new_matrix(n, d, device=DEV), D.new_matrix(n, d, device=DEV)
    A, Y = torch.zeros(M, inn, device=DEV), torch.zeros(M, out, device=DEV)
    labels, loss = torch.zeros(M, dtype=torch.int32, device=DEV), torch.zeros(n, device=DEV)

    def refused(status, call, *a, **k):
        with pytest.raises(D.DetagError) as e:
            call(*a, **k)
        assert e.value.status == status and e.value.message
    refused(D.DETAG_EINVAL, ctx.linear, W, 1, A, rows, Y)                    # past the end of the row
    refused(D.DETAG_EINVAL, ctx.linear, W, -1, A, rows, Y)
    refused(D.DETAG_EINVAL, ctx.linear, W, 1 << 62, A, rows, Y)
    refused(D.DETAG_EINVAL, ctx.linear, W, 0, A, rows, A)                    # in place
    refused(D.DETAG_EINVAL, ctx.linear_grad_input, W, 0, Y, rows, A, relu_of=A)
    refused(D.DETAG_EINVAL, ctx.linear_grad_weight, Y, A, rows, G, 1)
    with pytest.raises(ValueError, match="bfloat16"):
        ctx.linear(W.to(BF16), 0, A, rows, Y)                                # types that do not go together
    with pytest.raises(ValueError, match="12 rows"):
        ctx.linear(W, 0, A, rows, Y[:5])
    with pytest.raises(ValueError, match="rows must be"):
        ctx.linear(W, 0, A, rows[:3], Y)
    with pytest.raises(ValueError, match="rows must be"):
        ctx.linear(W, 0, A, rows.long(), Y)
    with pytest.raises(ValueError, match="contiguous rows"):
        ctx.linear(W, 0, torch.zeros(inn, M, device=DEV).t(), rows, Y)
    with pytest.raises(ValueError, match="pitch"):
        ctx.linear(W[:, :64], 0, A, rows, Y)
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        ctx.linear(W.half(), 0, A, rows, Y)
    with pytest.raises(ValueError, match="GPU"):
        ctx.linear(W, 0, A.cpu(), rows, Y)
    with pytest.raises(ValueError, match="relu_of"):
        ctx.linear_grad_input(W, 0, Y, rows, A, relu_of=torch.zeros(M, inn - 1, device=DEV))
    Yb = torch.zeros(M, out, dtype=BF16, device=DEV)
    refused(D.DETAG_EINVAL, ctx.linear, W, 0, A, rows, Yb)                   # fp32 operands, bf16 result
    with pytest.raises(ValueError, match="labels"):
        ctx.cross_entropy(Y, labels.long(), rows, Y)
    with pytest.raises(ValueError, match="loss"):
        ctx.cross_entropy(Y, labels, rows, Y, loss[:2])
    wide = torch.zeros(M, 2 * out, device=DEV)
    refused(D.DETAG_EINVAL, ctx.cross_entropy, wide[:, :out], labels, rows, wide.view(2 * M, out)[:M])
    refused(D.DETAG_EINVAL, ctx.reserve_cross_entropy, -1)

    for spans in ([(0, d + 1)], [(-1, 4)], [(0, 8), (7, 8)], [(4, -1)], [(1 << 62, 1 << 62)]):
        refused(D.DETAG_EINVAL, D.AdamW, ctx, spans)
    refused(D.DETAG_EINVAL, D.AdamW, ctx, [(0, d)], bits=16)
    refused(D.DETAG_EINVAL, D.AdamW, ctx, [(0, d)], [float("nan")])
    with pytest.raises(ValueError, match="one number per tensor"):
        D.AdamW(ctx, [(0, d)], [0.1, 0.2])
    opt, opt8 = D.AdamW(ctx, [(0, d)]), D.AdamW(ctx, [(0, d)], bits=8)
    X = D.new_matrix(n, d, device=DEV)
    M32, V32, _ = opt.new_moments(DEV)
    M8, V8, S8 = opt8.new_moments(DEV)
    refused(D.DETAG_EINVAL, opt.step, X, G, M32, V32, S8, lr=0.1, t=1) if S8.shape == (n, 2 * opt.blocks) else None
    refused(D.DETAG_EINVAL, opt8.step, X, G, M8, V8, lr=0.1, t=1)            # without scales
    refused(D.DETAG_EINVAL, opt.step, X, X, M32, V32, lr=0.1, t=1)
    for bad in (dict(t=0), dict(lr=float("inf")), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0), dict(limit=-1.0), dict(limit=float("nan"))):
        refused(D.DETAG_EINVAL, opt.step, X, G, M32, V32, **{**dict(lr=0.1, t=1), **bad})
    refused(D.DETAG_EINVAL, opt.values, M8, V8, S8, X, G)
    with pytest.raises(ValueError, match="M must be"):
        opt.step(X, G, M8, V8, lr=0.1, t=1)
    other = _context(n, d)
    opt.ctx = other
    refused(D.DETAG_EINVAL, opt.step, X, G, M32, V32, lr=0.1, t=1)           # another context's
    opt.ctx = ctx


def test_capture_refuses_to_allocate_for_the_loss():
    ctx = _context(2, 4)
    z, rows = torch.zeros(4, 3, device=DEV), _offsets([2, 2])
    labels, graph = torch.zeros(4, dtype=torch.int32, device=DEV), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        with pytest.raises(D.DetagError, match="reserve"):
            ctx.cross_entropy(z, labels, rows, z)
        z.add_(0)
    ctx.reserve_cross_entropy(4)
    ctx.cross_entropy(z, labels, rows, z)
    torch.cuda.synchronize()


def test_offsets_that_make_no_sense_stay_within_the_matrices():
    """Descending or outside: no result is promised, but nothing is written outside the rows and the layer's columns."""
    n, inn, out, M = 4, 40, 24, 50
    ctx = _context(n, inn * out)
    W, G = _weights(n, D.padded_ld(inn * out), 0, out, inn, F32, 1), D.new_matrix(n, inn * out, device=DEV)
    buf = torch.full((3 * M, 40), 7.0, device=DEV)
    A, Y = torch.zeros(M, inn, device=DEV), buf[M:2 * M, :out]
    labels = torch.zeros(M, dtype=torch.int32, device=DEV)
    for offs in ([-5, 10, 20, 30, 99], [0, 40, 10, 45, 50], [60, 70, 80, 90, 100], [50, 40, 30, 20, 10]):
        rows = torch.tensor(offs, dtype=torch.int32, device=DEV)
        ctx.linear(W, 0, A, rows, Y)
        ctx.linear_grad_input(W, 0, torch.zeros(M, out, device=DEV), rows, buf[M:2 * M])
        ctx.linear_grad_weight(torch.zeros(M, out, device=DEV), A, rows, G, 0)
        ctx.cross_entropy(Y, labels, rows, Y)
        torch.cuda.synchronize()
        assert (buf[:M] == 7).all() and (buf[2 * M:] == 7).all() and (G == 0).all()

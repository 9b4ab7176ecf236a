"""Products whose tiles' height is chosen on the GPU from the workers' rows, against the same in 64 bits.

Tolerance: a sum of K fp32 products in any order is off by at most (K + 8) 2^-24 times the sum of magnitudes, doubled; a bf16 result adds
half a spacing, at most 2^-8 of itself."""
import numpy as np
import pytest
import torch

import paper_2006_08085_amd as D

pytestmark = pytest.mark.gpu
DEV, BF16 = "cuda:0", torch.bfloat16

CASES = {
    "half": ([256] * 8, 72, 2824),                  # 96 tiles of 256 rows or 192 of 128, one for each compute unit
    "three-quarters": ([384] * 16, 88, 1544),       # 224 tiles of 256 or of 192, but 336 of 128
    "whole": ([512] * 8, 64, 4096),                 # 256 tiles
    "two-rounds": ([800, 0, 900, 700, 130, 400, 1, 333], 136, 6664),
    "70-workers": ([int(c) for c in np.random.default_rng(3).integers(0, 410, 70)], 104, 776),
    "130-workers": ([200 + 3 * (i % 7) for i in range(130)], 40, 264),
}


@pytest.mark.parametrize("name", CASES)
def test_products_with_chosen_heights(name):
    counts, inn, out = CASES[name]
    n, M = len(counts), sum(counts)
    g = torch.Generator().manual_seed(M)
    rows = torch.tensor([0, *np.cumsum(counts)], dtype=torch.int32, device=DEV)
    for forward in (True, False):                   # the input gradient has the many columns then
        a, b = (inn, out) if forward else (out, inn)
        d = inn * out
        ctx = D.detag_create(D.Topology.ring(), n, d, D.padded_ld(d))
        W = torch.full((n, ctx.ld), float("nan"), dtype=BF16)
        W[:, :d] = (inn ** -0.5 * torch.randn(n, d, generator=g)).to(BF16)
        W, x = W.to(DEV), torch.randn(M + 1, inn, generator=g).to(BF16).to(DEV)
        x[M:] = float("nan")
        y = torch.full((M + 1, out), 7.0, dtype=BF16, device=DEV)
        if forward:
            ctx.linear(W, 0, x, rows, y)
        else:
            ctx.linear_grad_input(W, 0, x, rows, y)
        assert (y[M:] == 7).all()
        for i in range(n):
            w, r = W[i, :d].double().view(b, a), x[rows[i]:rows[i + 1]].double()
            w = w.t() if forward else w
            ref, size = r @ w, r.abs() @ w.abs()
            off = (y[rows[i]:rows[i + 1]].double() - ref).abs()
            assert (off <= 2 * (inn + 8) * 2.0 ** -24 * size + 2.0 ** -8 * ref.abs() + 1e-37).all(), (name, forward, i)


@pytest.mark.parametrize("offset", [0, 3])
def test_fp32_weight_gradients_of_many_tiles(offset):
    counts = [(7 * i) % 70 if i % 5 else 0 for i in range(64)]
    inn, out, n, M = 517, 261, len(counts), sum(counts)
    g = torch.Generator().manual_seed(5)
    ctx = D.detag_create(D.Topology.ring(), n, offset + inn * out, offset + inn * out)
    rows = torch.tensor([0, *np.cumsum(counts)], dtype=torch.int32, device=DEV)
    dY, A = (torch.randn(M, c, generator=g).to(DEV) for c in (out, inn))
    G = torch.full((n, ctx.ld), 7.0, device=DEV)
    for accumulate in (False, True):
        ctx.linear_grad_weight(dY, A, rows, G, offset, accumulate=accumulate)
        for i in range(n):
            y, a = dY[rows[i]:rows[i + 1]].double(), A[rows[i]:rows[i + 1]].double()
            ref, size, got = y.t() @ a, y.abs().t() @ a.abs(), G[i, offset:].double().view(out, inn)
            if accumulate:
                ref, size = 2 * ref, 2 * size
            assert ((got - ref).abs() <= 2 * (counts[i] + 8) * 2.0 ** -24 * size + 2 * 2.0 ** -24 * ref.abs() + 1e-37).all()
    assert (G[:, :offset] == 7).all()


@pytest.mark.parametrize("inn,out", [(71, 199), (641, 77), (333, 1025)])
@pytest.mark.parametrize("dtype", [BF16, torch.float32], ids=["bf16", "f32"])
def test_odd_rows_see_nothing_of_their_neighbours(inn, out, dtype):
    """Rows that end inside a piece, whose neighbours in memory are NaN: between rows, of other workers, behind the last."""
    counts = [40, 33, 7, 0, 64]
    n, M, d = len(counts), sum(counts), inn * out
    g = torch.Generator().manual_seed(inn)
    ctx = D.detag_create(D.Topology.ring(), n, 1 + d, 1 + d)
    rows = torch.tensor([0, *np.cumsum(counts)], dtype=torch.int32, device=DEV)

    def matrix(cols):                               # NaN after every row and after the last
        buf = torch.full((M * (cols + 2) + 1,), float("nan"), dtype=dtype)
        view = buf[1:].view(M, cols + 2)[:, :cols]
        view.copy_(torch.randn(M, cols, generator=g))
        return buf.to(DEV)[1:].view(M, cols + 2)[:, :cols]
    A, dY = matrix(inn), matrix(out)
    W = torch.full((n, ctx.ld), float("nan"), dtype=dtype)
    W[:, 1:] = torch.randn(n, d, generator=g).to(dtype)
    W = W.to(DEV)
    A[40:73], dY[40:73], W[1] = float("nan"), float("inf"), float("nan")
    Y, dA, G = torch.zeros(M, out, dtype=dtype, device=DEV), torch.zeros(M, inn, dtype=dtype, device=DEV), torch.zeros(n, ctx.ld, device=DEV)
    ctx.linear(W, 1, A, rows, Y)
    ctx.linear_grad_input(W, 1, dY, rows, dA)
    ctx.linear_grad_weight(dY, A, rows, G, 1)
    own = torch.zeros(M, dtype=torch.bool, device=DEV)
    own[40:73] = True
    assert torch.isfinite(Y[~own]).all() and torch.isnan(Y[own]).all()
    assert torch.isfinite(dA[~own]).all() and torch.isnan(dA[own]).all()
    assert torch.isfinite(G[[0, 2, 3, 4]]).all() and torch.isnan(G[1, 1:]).all()

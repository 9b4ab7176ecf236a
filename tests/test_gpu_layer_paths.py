"""Products whose sizes reach each kernel and tile that the launch rules choose, against the same in 64 bits.

Which one a call takes follows from its sizes and alignment (the comments beside the rules in k_linear.hip); the cases are made from those
bounds and run in all three directions.  Results are NaN beforehand, so that a tile that nobody computes shows.

Tolerance: a sum of K fp32 products in any order is off by at most (K + 8) 2^-24 times the sum of magnitudes, doubled; a bf16 result adds
half a spacing, at most 2^-8 of itself."""
import numpy as np
import pytest
import torch

import paper_2006_08085_amd as D

pytestmark = pytest.mark.gpu
DEV, BF16, F32 = "cuda:0", torch.bfloat16, torch.float32


def _uneven(n, M, seed, empty=0):
    """n numbers of rows, M in all, some of them zero."""
    rng = np.random.default_rng(seed)
    share = rng.dirichlet(np.full(n, 0.7))
    share[rng.permutation(n)[:empty]] = 0
    counts = np.floor(share / share.sum() * M).astype(int)
    counts[int(np.argmax(counts))] += M - counts.sum()
    return counts.tolist()


# workers' rows, inputs, outputs, operands, first column, elements between rows
CASES = {
    # fp32 tiles: more than one deal of 64 to the XCDs, the last of them ragged, empty workers, odd widths
    "f32-tiles": (_uneven(24, 1500, 1, empty=5), 300, 771, F32, 0, 0),
    "f32-tiles-shallow": (_uneven(70, 3001, 2, empty=20), 77, 333, F32, 5, 3),
    "f32-tiles-wide": (_uneven(5, 2111, 3, empty=1), 1003, 517, F32, 1, 0),
    # calls of few tiles in blocks of 64 rows, fp32 and bf16, contractions that end inside a piece
    "f32-64-rows": ([200, 0, 137, 263], 522, 645, F32, 3, 0),
    "bf16-64-rows": ([200, 0, 137, 263], 522, 646, BF16, 0, 0),
    "bf16-64-rows-even": ([64, 64], 1032, 1048, BF16, 8, 8),
    # ... of 16 rows, rows on dwords and not
    "f32-16-rows": ([2, 9, 0, 4], 1031, 515, F32, 0, 0),
    "bf16-16-rows": ([2, 9, 0, 4], 1032, 518, BF16, 0, 0),
    "bf16-16-rows-odd": ([2, 9, 0, 4], 1031, 515, BF16, 7, 1),
    # fp32 weight gradients: 64 x 64 with many rows, 128 x 128 with few, rows shared out in a block
    "f32-weights-many-rows": ([400, 1, 300, 199], 1000, 1003, F32, 0, 0),
    "f32-weights-few-rows": (_uneven(9, 900, 4), 1000, 1003, F32, 2, 0),
    "f32-weights-shared": ([900, 77], 261, 130, F32, 0, 0),
    # bf16 with rows on dwords: 64 x 64, 64 x 128 (few rows a worker), 128 x 128 and 256 x 256, the many columns on either side
    "bf16-64x64": (_uneven(40, 2000, 9, empty=8), 200, 256, BF16, 0, 0),
    "bf16-64x128": (_uneven(40, 2000, 5, empty=8), 256, 1024, BF16, 0, 0),
    "bf16-64x128-inputs": (_uneven(40, 2000, 6, empty=8), 1034, 522, BF16, 0, 2),
    "bf16-128x128": (_uneven(20, 2500, 7, empty=2), 266, 2054, BF16, 4, 0),
    "bf16-256x256": (_uneven(9, 3333, 8, empty=1), 1290, 2314, BF16, 0, 0),
    "bf16-256x256-inputs": (_uneven(9, 3333, 12, empty=1), 2314, 1290, BF16, 2, 0),
    # ... through registers
    "bf16-odd-64x64": (_uneven(6, 300, 11, empty=1), 131, 701, BF16, 0, 0),
    "bf16-odd-64x128": (_uneven(20, 2500, 10, empty=2), 267, 2055, BF16, 1, 0),
    "bf16-odd-64x128-inputs": (_uneven(20, 2500, 13, empty=2), 2055, 267, BF16, 1, 0),
    "bf16-odd-widths-on-dwords": (_uneven(20, 2500, 14, empty=2), 267, 2055, BF16, 0, 1),
}


def _matrix(M, cols, dtype, seed, gap):
    """M x cols of a matrix whose rows lie `gap` elements apart, with NaN in between and behind."""
    buf = torch.full((M + 1, cols + gap), float("nan"), dtype=dtype)
    buf[:M, :cols] = torch.randn(M, cols, generator=torch.Generator().manual_seed(seed)).to(dtype)
    return buf.to(DEV)[:M, :cols]


def _check(got, ref, size, K, dtype, what):
    bound = 2 * (K + 8) * 2.0 ** -24 * size + (2.0 ** -8 if dtype is BF16 else 2.0 ** -23) * ref.abs() + 1e-37
    off = (got.double() - ref).abs()
    assert (off <= bound).all(), (what, int((~(off <= bound)).sum()))


@pytest.mark.parametrize("name", CASES)
def test_every_direction(name):
    counts, inn, out, dtype, offset, gap = CASES[name]
    n, M, d = len(counts), sum(counts), inn * out
    ends = np.cumsum(counts)
    spans = [(i, int(e - c), int(e)) for i, (c, e) in enumerate(zip(counts, ends)) if c]
    ld = offset + d + (d + offset) % 2                # whole dwords from worker to worker where the rest is
    ctx = D.detag_create(D.Topology.ring(), n, offset + d, ld)
    rows = torch.tensor([0, *ends], dtype=torch.int32, device=DEV)
    W = torch.full((n, ld), float("nan"), dtype=dtype)
    W[:, offset:offset + d] = (inn ** -0.5 * torch.randn(n, d, generator=torch.Generator().manual_seed(1))).to(dtype)
    W = W.to(DEV)
    A, dY = _matrix(M, inn, dtype, 2, gap), _matrix(M, out, dtype, 3, gap)
    weights = {i: W[i, offset:offset + d].double().view(out, inn) for i, _, _ in spans}

    for relu, y_type in ((False, dtype), (True, F32)):
        Y = torch.full((M, out), float("nan"), dtype=y_type, device=DEV)
        ctx.linear(W, offset, A, rows, Y, relu=relu)
        for i, lo, hi in spans:
            a, w = A[lo:hi].double(), weights[i]
            ref = a @ w.t()
            _check(Y[lo:hi], ref.clamp(min=0) if relu else ref, a.abs() @ w.abs().t(), inn, y_type, ("forward", relu, i))
    for H in (None, A):
        dA = torch.full((M, inn), float("nan"), dtype=dtype, device=DEV)
        ctx.linear_grad_input(W, offset, dY, rows, dA, relu_of=H)
        for i, lo, hi in spans:
            y, w = dY[lo:hi].double(), weights[i]
            keep = 1.0 if H is None else (H[lo:hi] > 0).double()
            _check(dA[lo:hi], (y @ w) * keep, (y.abs() @ w.abs()) * keep, out, dtype, ("input gradient", H is not None, i))
    G = torch.full((n, ld), float("nan"), device=DEV)
    ctx.linear_grad_weight(dY, A, rows, G, offset)
    once = G.clone()
    ctx.linear_grad_weight(dY, A, rows, G, offset, accumulate=True)
    assert torch.isnan(G[:, :offset]).all() and torch.isnan(G[:, offset + d:]).all()
    for i, count in enumerate(counts):
        if not count:
            assert (G[i, offset:offset + d] == 0).all() and (once[i, offset:offset + d] == 0).all()
    for i, lo, hi in spans:
        y, a = dY[lo:hi].double(), A[lo:hi].double()
        ref, size = y.t() @ a, y.abs().t() @ a.abs()
        _check(once[i, offset:offset + d].view(out, inn), ref, size, hi - lo, F32, ("weight gradient", i))
        _check(G[i, offset:offset + d].view(out, inn), 2 * ref, 2 * size, hi - lo, F32, ("added", i))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("inn,out", [(137, 65), (140, 600)])
def test_rows_too_far_apart_for_a_buffer(inn, out, dtype):
    """A pitch with which 256 rows pass 2^31 bytes: nothing goes straight to LDS, fp32 neither."""
    counts, pitch = [3, 0, 70], 1 << 22
    n, M, d = len(counts), sum(counts), inn * out
    ctx = D.detag_create(D.Topology.ring(), n, d, d + d % 2)
    rows = torch.tensor([0, *np.cumsum(counts)], dtype=torch.int32, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    buf = torch.full((M, pitch), float("nan"), dtype=dtype, device=DEV)
    A, dY, Y, dA = buf[:, 10:10 + inn], buf[:, 1000:1000 + out], buf[:, 2000:2000 + out], buf[:, 3000:3000 + inn]
    A.copy_(torch.randn(M, inn, generator=g, device=DEV)), dY.copy_(torch.randn(M, out, generator=g, device=DEV))
    W, G = torch.randn(n, ctx.ld, generator=g, device=DEV).to(dtype), torch.full((n, ctx.ld), float("nan"), device=DEV)
    ctx.linear(W, 0, A, rows, Y)
    ctx.linear_grad_input(W, 0, dY, rows, dA)
    ctx.linear_grad_weight(dY, A, rows, G, 0)
    for i, lo, hi in ((0, 0, 3), (2, 3, 73)):
        w, a, y = W[i, :d].double().view(out, inn), A[lo:hi].double(), dY[lo:hi].double()
        _check(Y[lo:hi], a @ w.t(), a.abs() @ w.abs().t(), inn, dtype, "forward")
        _check(dA[lo:hi], y @ w, y.abs() @ w.abs(), out, dtype, "input gradient")
        _check(G[i, :d].view(out, inn), y.t() @ a, y.abs().t() @ a.abs(), hi - lo, F32, "weight gradient")
    assert (G[1, :d] == 0).all()
    del buf, A, dY, Y, dA
    torch.cuda.empty_cache()

"""Dropout against its definition (Philox-4x32-10 of oracle/noise.py, which is pinned to the authors' vectors), kept entry by kept entry."""
import math

import numpy as np
import pytest
import torch

from oracle.noise import philox4x32_10
from tests.block_util import BF16, DEV, F32, U, _built, assert_within, context, half_step, matrix, offsets, spans  # noqa: F401

pytestmark = pytest.mark.gpu


def kept(rows, columns, worker, p, seed, step):
    """Which entries of a worker's rows stay, from the definition."""
    k = np.arange(-(-columns // 8))[None, :]
    j = np.arange(rows)[:, None]
    words = philox4x32_10((k + 0 * j, 2 ** 31 + j + 0 * k, worker, step), (seed & 0xFFFFFFFF, seed >> 32))
    words = np.stack([np.broadcast_to(w, (rows, k.shape[1])) for w in words], axis=2)
    halves = np.stack([words & 0xFFFF, words >> 16], axis=3).reshape(rows, 8 * k.shape[1])[:, :columns]
    return torch.from_numpy(halves.astype(np.int64) >= math.floor(65536 * p + 0.5))


CASES = [([1], 1, 0, 0, F32), ([1], 1, 0, 0, BF16), ([3, 0, 2], 7, 0, 1, BF16), ([0, 0], 16, 0, 0, F32), ([5, 0, 17, 1], 512, 8, 0, BF16),
         ([5, 0, 17, 1], 777, 3, 1, F32), ([5, 0, 17, 1], 777, 3, 1, BF16), ([1, 2], 4099, 0, 0, BF16), ([2, 0, 1] * 40, 24, 0, 0, F32),
         ([1] * 8, 1024, 0, 0, BF16), ([300, 20], 96, 0, 0, BF16)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{len(c[0])}x{sum(c[0])}-{c[1]}-{c[2]}-{'bf16' if c[4] is BF16 else 'f32'}")
@pytest.mark.parametrize("p,residual", [(0.1, True), (0.5, False), (0.0, True), (0.9999, False)])
def test_dropout(case, p, residual):
    counts, C, extra, shift, dtype = case
    n, M = len(counts), sum(counts)
    ctx = context(n, 8)
    X, _ = matrix(M + 2, C, dtype, 1, extra, shift)
    R, _ = matrix(M + 2, C, dtype, 2, extra, 0)
    Y, buf = matrix(M + 2, C, dtype, None, extra, shift, around=7.0)
    before, rows, seed, step = buf.clone(), offsets(counts), (3 << 40) + 12345, 9
    ctx.dropout(X, rows, Y, p=p, seed=seed, step=step, residual=R if residual else None)
    torch.cuda.synchronize()
    factor = 65536 / (65536 - math.floor(65536 * p + 0.5))
    for i, lo, hi in spans(counts):
        mask = kept(hi - lo, C, i, p, seed, step).to(DEV)
        x, r = X[lo:hi].double(), R[lo:hi].double() if residual else torch.zeros(hi - lo, C, dtype=torch.float64, device=DEV)
        assert torch.equal(Y[lo:hi].double()[~mask], r[~mask])
        ref = (x * factor + r)[mask]
        assert_within(Y[lo:hi][mask], ref, 3 * U * ((x * factor).abs() + r.abs())[mask] + half_step(dtype) * ref.abs())
    first = Y[:M].clone()
    for target in ("X", "R")[:1 + residual]:              # in place
        x, res = X.clone(), R.clone()
        out = x if target == "X" else res
        ctx.dropout(x, rows, out, p=p, seed=seed, step=step, residual=res if residual else None)
        assert torch.equal(out[:M], first)
    Y[:M] = 7.0
    assert torch.equal(buf, before)


def test_shares_steps_and_the_way_back():
    """As many kept as p says, other ones with another step, seed or worker, the same ones for a gradient."""
    n, C, each, p = 2, 2048, 64, 0.25
    ctx = context(n, 8)
    X, rows = torch.ones(n * each, C, device=DEV), offsets([each] * n)

    def draw(x=X, **more):
        Y = torch.zeros_like(x)
        ctx.dropout(x, rows, Y, **dict(dict(p=p, seed=5, step=1), **more))
        return Y
    Y = draw()
    share = (Y != 0).double().mean().item()
    assert abs(share - 0.75) < 5 * math.sqrt(0.25 * 0.75 / Y.numel())
    assert torch.equal(draw(), Y) and torch.equal(draw(2 * X), 2 * Y)
    for other in (draw(step=2), draw(seed=6), draw(seed=5 + (1 << 32)), torch.roll(Y, each, 0)):
        agree = ((other != 0) == (Y != 0)).double().mean().item()   # independent: 0.75^2 + 0.25^2
        assert abs(agree - 0.625) < 5 * math.sqrt(0.625 * 0.375 / Y.numel())
    dropped = draw(torch.full_like(X, float("nan")))
    assert torch.equal(dropped.isnan(), Y != 0) and not dropped[Y == 0].any()

"""Operators of residual blocks whose workers' rows, or sequences, do not start at the first row and do not end at the last one: the same bits as
for the same rows elsewhere in the matrices, and all other rows stay as they were.  Offsets past the matrices end at their last row."""
import pytest
import torch

from tests.block_util import ACTS, BF16, DEV, F32, _built, context, offsets  # noqa: F401

pytestmark = pytest.mark.gpu

SPARE = 37
COUNTS = [[70, 0, 33, 130], [3, 0, 41] * 24]               # 72 of them: more than a wavefront has lanes


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("counts", COUNTS, ids=["4", "72"])
@pytest.mark.parametrize("heads", [4, 48])
def test_first_rows_of_nobody(counts, heads, dtype):
    n, inside, W, out = len(counts), sum(counts), 16, 72
    C, M = heads * W, inside + SPARE
    ctx = context(n, C * out + out + 2 * C)
    g = torch.Generator(device=DEV).manual_seed(3)
    P = torch.randn(n, ctx.ld, device=DEV, generator=g).to(dtype)
    given = [torch.randn(inside, c, device=DEV, generator=g).to(dtype) for c in (C, C, out, C, C // 2, C // 2)]

    def run(first, last=None):
        def place(t):
            whole = torch.full((M, t.shape[1]), float("nan"), dtype=t.dtype, device=DEV)
            whole[first:first + inside] = t
            return whole

        def new(cols, dtype=dtype):
            kept.append(torch.full((M, cols), 7.0, dtype=dtype, device=DEV))
            return kept[-1]
        kept, at = [], offsets(counts, first)
        if last is not None:
            at[-1] = last
        X, dX, dY, Q, K, V = map(place, given)
        G, lse = torch.zeros(n, ctx.ld, device=DEV), torch.full((heads, M), 7.0, device=DEV)
        b = C * out
        ctx.layer_norm(P, b + out, b + out + C, X, at, new(C))
        ctx.layer_norm_grad(P, b + out, b + out + C, X, dX, at, new(C), G, add=Q)
        ctx.linear_act(P, 0, X, at, new(out), bias=b, act=ACTS["gelu"], pre=new(out), residual=dY)
        ctx.linear_grad_bias(dY, at, G, b, act=ACTS["silu"], pre=dY, dZ=new(out))
        ctx.linear_grad_input_act(P, 0, dY, at, new(C), act=ACTS["gelu"], pre=X)
        ctx.dropout(X, at, new(C), p=0.3, seed=5, step=2, residual=dX)
        O = new(C)
        ctx.attention(Q, K, V, at, O, heads, heads // 2, lse=lse)
        ctx.attention_grad(Q, K, V, at, O, lse, dX, new(C), new(C // 2), new(C // 2), heads, heads // 2)
        kept.append(lse.t())
        torch.cuda.synchronize()
        for t in kept:
            assert (t[:first] == 7.0).all() and (t[first + inside:] == 7.0).all() and t[first:first + inside].isfinite().all()
        return [t[first:first + inside].clone() for t in kept] + [G]
    plain = run(0)
    assert all(a.any() for a in plain)
    for other in (run(SPARE), run(SPARE, last=M + 1000), run(SPARE - 5)):
        assert all(torch.equal(a, b) for a, b in zip(plain, other))

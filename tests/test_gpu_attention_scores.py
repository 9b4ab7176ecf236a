"""Attention and its gradient where the scores are far from zero: a softmax does not see a number that is added to all scores of a row,
so the checks and bounds are those of test_gpu_attention, on other inputs.  Every key of a sequence has a level; column 0 of every head
adds it to its scores, whose other columns are random as there.

One term is added to the bounds.  With levels that differ by 88 and more some probabilities are below 2^-126, the smallest normal number of
fp32, and the hardware's exp2 gives zero for them.  An entry of a result sums at most 300 rows times 4 query heads, 1200 < 2^11 terms.  What
such a probability is multiplied with is at most 2^13: dO and V are below 6; in dz = p (dP - delta) scale a product of 128 pairs of
normal numbers is below 6 sqrt(128) = 68 and so is delta, q is at most 8 and k at most 300 sqrt(128) / 8 = 425, scale is 128^-0.5 = 0.09 there:
2 * 68 * 425 * 0.09 = 5200 < 2^13, and less for smaller heads.  In all 2^-126 2^11 2^13 = 2^-102."""
import math

import pytest
import torch

from tests import test_gpu_attention as plain
from tests.block_util import BF16, DEV, F32, _built, assert_within, context, half_step, matrix, offsets, spans  # noqa: F401

pytestmark = pytest.mark.gpu

# level of key r of a sequence
LEVELS = {
    "150 and 300 in turn": lambda r: torch.where(r % 64 < 32, 150.0, 300.0),
    "all -200": lambda r: torch.full_like(r, -200.0),
    "rising from -300": lambda r: r - 300.0,                                      # causal: every row's own key is its largest
    "-300, then 0": lambda r: torch.where(r < 140, -300.0, 0.0),                  # more keys than a panel holds
    "0, then -300": lambda r: torch.where(r < 140, 0.0, -300.0),
    "-95 and -80 in turn": lambda r: torch.where(r % 64 < 32, -95.0, -80.0),      # wavefronts that share a panel have 32 keys each
}
COUNTS = [300, 1, 0, 40]
FLUSHED = 2.0 ** -102


def _inputs(level, case, seed=1):
    counts, H, KV, W, extra, shift, dtype = case
    M = sum(counts) + 2
    Q, K, V, dO = (matrix(M, h * W, dtype, seed + k, extra, shift)[0] for k, h in enumerate((H, KV, KV, H)))
    r = torch.zeros(M, device=DEV)
    for _, lo, hi in spans(counts):
        r[lo:hi] = torch.arange(hi - lo, device=DEV)
    Q[:, ::W] = 8.0
    K[:, ::W] = (level(r) * W ** 0.5 / 8.0).to(dtype)[:, None]
    for t in (Q, K, V, dO):
        t[M - 2:] = float("nan")
    return Q, K, V, dO, M


def _case(dtype, W, heads, odd):
    """heads few enough that a block's wavefronts share the keys of 32 queries, or enough for blocks of 128 queries."""
    H, KV = (4, 2) if heads == "few" else (160, 40)
    return COUNTS, H, KV, W, 3 * odd, odd, dtype


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("W, odd", [(64, 0), (17, 1), (128, 0)])
@pytest.mark.parametrize("heads", ["few", "many"])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
@pytest.mark.parametrize("level", LEVELS)
def test_low_scores(monkeypatch, level, causal, heads, W, odd, dtype):
    monkeypatch.setattr(plain, "_inputs", lambda case: _inputs(LEVELS[level], case))
    monkeypatch.setattr(plain, "assert_within", lambda got, ref, bound: assert_within(got, ref, bound + FLUSHED))
    case = _case(dtype, W, heads, odd)
    plain.test_attention(case, causal)
    plain.test_attention_grad(case, causal)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("W, odd", [(64, 0), (17, 1), (128, 0)])
@pytest.mark.parametrize("heads", ["few", "many"])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
def test_low_scores_after_keys_without_probability(causal, heads, W, odd, dtype):
    """Scores of -inf over more than a panel, then some of -150."""
    counts, H, KV, W, extra, shift, dtype = case = _case(dtype, W, heads, odd)
    Q, K, V, _, M = _inputs(lambda r: torch.where(r < 140, -math.inf, -150.0), case)
    ctx, seqs = context(1, 8), offsets(counts)
    O, lse = torch.zeros(M, H * W, dtype=dtype, device=DEV), torch.zeros(H, M, device=DEV)
    ctx.attention(Q, K, V, seqs, O, H, KV, causal=causal, lse=lse)
    # the first 140 rows of a causal call see no key with a finite score, nor does a sequence of no more keys
    for _, lo, hi in spans(counts):
        none = min(hi - lo, 140) if causal or hi - lo <= 140 else 0
        assert O[lo:lo + none].isnan().all() and (lse[:, lo:lo + none] == -math.inf).all()
        if none == hi - lo:
            continue
        for j in range(H):
            q, k, v = (plain._head(t, lo, hi, h, W)[140 * (t is not Q):] for t, h in ((Q, j), (K, j // (H // KV)), (V, j // (H // KV))))
            # the keys that count, and the rows that see one: those from 140 on see a triangle of them
            p, ref_lse, e, p_off = plain._softmax(q[none:], k, W ** -0.5, causal, dtype)
            ref, size = p @ v, p @ v.abs()
            rounded = half_step(dtype) if dtype is BF16 else 0.0
            assert_within(plain._head(O, lo + none, hi, j, W), ref, (p_off + rounded + (hi - lo + 8) * plain.U) * size + 2 * p_off * ref.abs()
                          + half_step(dtype) * ref.abs())
            assert_within(lse[j, lo + none:hi], ref_lse, e[:, 0] + p_off[:, 0] + 4 * plain.U * (1 + ref_lse.abs()))

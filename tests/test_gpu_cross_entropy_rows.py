"""Cross-entropy of more rows than one launch takes, and of as many rows or classes as an int32 counts.

Tolerances: exp of the hardware is within 2^-22 relative, so that a softmax of two or a few classes is within 2^-20, and a bf16 result
adds half a spacing, at most 2^-8 of itself.  A worker's loss is a sum of terms of one sign, whose 1024 threads each add a share of
the rows one after the other: the first test allows 2^-24 of it for every addition, the last one next to nothing."""
import pytest
import torch

import paper_2006_08085_amd as D

pytestmark = pytest.mark.gpu
DEV, BF16 = "cuda:0", torch.bfloat16


def _offsets(ends):
    return torch.tensor([0, *ends], dtype=torch.int32, device=DEV)


# rows, classes: 16 lanes a row (2^28 rows are 2^32 threads), 64 lanes a row (2^26 rows are)
@pytest.mark.parametrize("M,C", [((1 << 28) + 8, 2), ((1 << 26) + 5, 129)], ids=["16-lanes", "64-lanes"])
def test_rows_beyond_one_launch(M, C):
    torch.cuda.empty_cache()
    n, spare = 5, 3                                   # the last rows belong to nobody
    ends = [M // 3, M // 3, M // 2 + 1, M - spare - 2, M - spare]
    ctx, rows = D.detag_create(D.Topology.ring(), n, 4, 4), _offsets(ends)
    g = torch.Generator(device=DEV).manual_seed(1)
    z = torch.empty(M, C, dtype=BF16, device=DEV).normal_(generator=g)
    labels = torch.randint(-1, C, (M,), generator=g, device=DEV, dtype=torch.int32)
    labels[ends[3]:] = 1
    grad, loss = torch.full_like(z, float("nan")), torch.full((n,), -1.0, device=DEV)
    ctx.cross_entropy(z, labels, rows, grad, loss)
    assert torch.isnan(grad[M - spare:]).all() and not any(torch.isnan(part).any() for part in grad[:M - spare].split(1 << 24))
    at = [0, *ends]
    for i, (lo, hi) in enumerate(zip(at, at[1:])):
        if hi == lo:
            assert float(loss[i]) == 0.0
            continue
        count, total = int((labels[lo:hi] >= 0).sum()), torch.zeros((), dtype=torch.float64, device=DEV)
        step = 1 << 24 if C == 2 else 1 << 20
        # with many classes the loss from all rows, the gradient of every fourth stretch
        for k, a in enumerate(range(lo, hi, step)):
            b = min(a + step, hi)
            logp, own = torch.log_softmax(z[a:b].double(), 1), labels[a:b].clamp(min=0).long()[:, None]
            ok = (labels[a:b] >= 0).double()
            total -= (logp.gather(1, own)[:, 0] * ok).sum()
            if C > 2 and k % 4 and b < hi:
                continue
            ref = logp.exp_().scatter_add_(1, own, torch.full_like(own, -1, dtype=torch.float64)).mul_((ok / count)[:, None])
            off = (grad[a:b].double() - ref).abs_()
            assert (off <= 2.0 ** -8 * ref.abs() + 2.0 ** -19 / count).all(), (i, a)
            del logp, own, ref, off
        assert abs(float(loss[i]) * count / float(total) - 1) < (hi - lo) / 1024 * 2.0 ** -24 + 1e-5
    del z, grad, labels, ctx
    torch.cuda.empty_cache()


def test_as_many_rows_as_there_can_be():
    """One class: every row that counts has a gradient and a loss of zero, whatever its logit."""
    torch.cuda.empty_cache()
    n, M = 64, (1 << 31) - 1
    ctx = D.detag_create(D.Topology.ring(), n, 4, 4)
    rows = _offsets([(i + 1) * (M // n) for i in range(n - 1)] + [M])
    z, labels = torch.ones(M, 1, dtype=BF16, device=DEV), torch.zeros(M, dtype=torch.int32, device=DEV)
    labels[::1000] = -100
    grad, loss = torch.full((M, 1), float("nan"), dtype=BF16, device=DEV), torch.full((n,), -1.0, device=DEV)
    ctx.cross_entropy(z, labels, rows, grad, loss)
    assert (loss == 0).all() and all((part == 0).all() for part in grad.split(1 << 28))
    del z, grad, labels, ctx
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [BF16, torch.float32], ids=["bf16", "f32"])
def test_as_many_classes_as_there_can_be(dtype):
    """Equal logits but for the label's, which is the last: the others' sum is a whole number that fp32 holds lane by lane."""
    torch.cuda.empty_cache()
    C = (1 << 31) - 1
    ctx, rows = D.detag_create(D.Topology.ring(), 1, 4, 4), _offsets([1])
    z, labels = torch.zeros(1, C, dtype=dtype, device=DEV), torch.tensor([C - 1], dtype=torch.int32, device=DEV)
    z[0, C - 1] = 3.0
    grad, loss = torch.full_like(z, float("nan")), torch.zeros(1, device=DEV)
    ctx.cross_entropy(z, labels, rows, grad, loss)
    e = torch.tensor(3.0, dtype=torch.float64).exp()
    total = float(C - 1 + e)
    for part in grad[0, :C - 1].split(1 << 28):
        assert ((part.float() * total - 1).abs() <= (2.0 ** -8 if dtype is BF16 else 0) + 2.0 ** -19).all()
    assert abs(float(grad[0, C - 1]) - float(e / total - 1)) <= 2.0 ** -19
    assert abs(float(loss) - float(torch.tensor(total, dtype=torch.float64).log() - 3)) <= 2.0 ** -18
    del z, grad
    torch.cuda.empty_cache()


def test_the_loss_of_many_equal_rows():
    """A model that answers log C everywhere: log and the final product are within 2^-20 relative, whatever the number of rows."""
    n, M, C = 2, 3 << 23, 10
    ctx = D.detag_create(D.Topology.ring(), n, 4, 4)
    z, labels = torch.zeros(M, C, dtype=BF16, device=DEV), torch.zeros(M, dtype=torch.int32, device=DEV)
    loss = torch.zeros(n, device=DEV)
    ctx.cross_entropy(z, labels, _offsets([1 << 24, M]), z, loss)
    want = torch.tensor(float(C), dtype=torch.float64).log()
    assert ((loss.cpu().double() / want - 1).abs() < 2.0 ** -20).all()


# classes in pieces of 16 bytes: up to 16, 64, 128, 256, 512, 1024, 2048, 4096, 8192, 16384 of them, and more
@pytest.mark.parametrize("dtype", [BF16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("pieces", [15, 33, 128, 255, 300, 1024, 1025, 4000, 4097, 16383, 16385])
@pytest.mark.parametrize("streams", [False, True], ids=["stays", "streams"])
def test_every_width(pieces, streams, dtype):
    """More than 512 rows, and as many as make the call stream: the gradient of every row and the losses in 64 bits.

    exp is within 2^-22 relative, and a sum of C terms of one sign, taken by 16 to 1024 lanes, within C / 16 additions, 2^-24 each and in
    different directions: a tenth of that is allowed, and 2^-20 for the rest."""
    torch.cuda.empty_cache()
    elems = 8 if dtype is BF16 else 4
    C, n = pieces * elems - 3, 3
    M = 515 if not streams else max(515, -(-(1 << 28) // (2 * C * 16 // elems)) + 7)
    ends = [M // 5, M // 5, M - 1]                    # the last row is nobody's
    ctx, g = D.detag_create(D.Topology.ring(), n, 4, 4), torch.Generator(device=DEV).manual_seed(pieces)
    z = torch.empty(M, C, dtype=dtype, device=DEV).normal_(generator=g)
    labels = torch.randint(-1, C, (M,), generator=g, device=DEV, dtype=torch.int32)
    labels[0], labels[M - 2] = C - 1, 0
    grad, loss = torch.full_like(z, float("nan")), torch.full((n,), -1.0, device=DEV)
    ctx.cross_entropy(z, labels, _offsets(ends), grad, loss)
    assert torch.isnan(grad[M - 1]).all() and float(loss[1]) == 0.0
    rel = 2.0 ** -20 + C / 160 * 2.0 ** -24
    for i, (lo, hi) in ((0, (0, ends[0])), (2, (ends[1], ends[2]))):
        count, total = int((labels[lo:hi] >= 0).sum()), 0.0
        step = max(1, (1 << 25) // C)
        for a in range(lo, hi, step):
            b = min(a + step, hi)
            logp, own = torch.log_softmax(z[a:b].double(), 1), labels[a:b].clamp(min=0).long()[:, None]
            ok = (labels[a:b] >= 0).double()
            total -= float((logp.gather(1, own)[:, 0] * ok).sum())
            ref = logp.exp_().scatter_add_(1, own, torch.full_like(own, -1, dtype=torch.float64)).mul_((ok / count)[:, None])
            bound = (rel + (2.0 ** -8 if dtype is BF16 else 0.0)) * ref.abs() + rel / count * (ref < 0) + 1e-37
            assert ((grad[a:b].double() - ref).abs_() <= bound).all(), (i, a)
        assert abs(float(loss[i]) - total / count) < 2.0 ** -19 * (1 + total / count)
    del z, grad, logp, ref, bound
    torch.cuda.empty_cache()

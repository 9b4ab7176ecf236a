"""Products of as many rows, inputs or outputs as they take, and the refusal of more.  Operands are small whole numbers: sums are exact."""
import ctypes as C

import pytest
import torch

import paper_2006_08085_amd as D

pytestmark = pytest.mark.gpu
DEV, BF16, F32 = "cuda:0", torch.bfloat16, torch.float32
MOST = (1 << 31) - (1 << 16)


@pytest.fixture(autouse=True)
def _memory():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def test_more_is_refused():
    """Nothing of these sizes is there: the refusal comes before any launch."""
    ctx = D.detag_create(D.Topology.ring(), 1, 1 << 33, 1 << 33)
    some = torch.zeros(64, device=DEV)
    rows = torch.zeros(2, dtype=torch.int32, device=DEV)
    L, p, r, other = D.lib(), some.data_ptr(), rows.data_ptr(), some[32:].data_ptr()
    for M, inn, out in ((MOST + 1, 1, 1), ((1 << 31) - 1, 1, 1), (1, MOST + 1, 1), (1, (1 << 31) - 1, 2), (1, 1, MOST + 1), (1, 2, (1 << 31) - 1)):
        for st in (L.detag_linear(ctx._h, p, 0, D.DETAG_F32, p, inn, r, M, inn, out, 0, other, out, D.DETAG_F32, None),
                   L.detag_linear_grad_input(ctx._h, p, 0, D.DETAG_F32, p, out, r, M, inn, out, None, 0, other, inn, None),
                   L.detag_linear_grad_weight(ctx._h, D.DETAG_F32, p, out, p, inn, r, M, inn, out, other, 0, 0, None)):
            assert st == D.DETAG_EINVAL and b"2^31 - 2^16" in L.detag_last_error(ctx._h)


def _sparse(count, value, dtype):
    """Zeros but for `value` in eight places, the first and the last among them."""
    v, at = torch.zeros(count, dtype=dtype, device=DEV), [0, 1, 63, 70_000, 1 << 30, count - 65, count - 2, count - 1]
    v[at] = value
    return v, at


def test_as_many_rows_as_it_takes():
    n, each = 64, MOST // 64
    ctx = D.detag_create(D.Topology.ring(), n, 1, 1)
    rows = torch.tensor([i * each for i in range(n + 1)], dtype=torch.int32, device=DEV)
    W = (1 + torch.arange(n, device=DEV)).to(BF16).view(n, 1)
    a, at = _sparse(MOST, 3.0, BF16)
    A, Y = a.view(-1, 1), torch.full((MOST, 1), float("nan"), dtype=BF16, device=DEV)
    ctx.linear(W, 0, A, rows, Y)
    assert [float(Y[k]) for k in at] == [3.0 * (1 + k // each) for k in at]
    assert sum(int((part != 0).sum()) for part in Y.split(1 << 28)) == len(at)
    ctx.linear_grad_input(W, 0, A, rows, Y)
    assert [float(Y[k]) for k in at] == [3.0 * (1 + k // each) for k in at]
    assert sum(int((part != 0).sum()) for part in Y.split(1 << 28)) == len(at)
    G, want = torch.full((n, 1), 7.0, device=DEV), torch.zeros(n, 1)
    for k in at:
        want[k // each] += 6.0
    ctx.linear_grad_weight(A, Y.fill_(2.0), rows, G, 0)
    assert torch.equal(G.cpu(), want)


@pytest.mark.parametrize("wide_in", [True, False], ids=["inputs", "outputs"])
def test_as_many_columns_as_it_takes(wide_in):
    inn, out = (MOST, 1) if wide_in else (1, MOST)
    ctx = D.detag_create(D.Topology.ring(), 1, MOST, MOST)
    rows = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    one, (v, at) = torch.full((1, 1), 2.0, dtype=BF16, device=DEV), _sparse(MOST, 3.0, BF16)
    W, wide = v.view(1, MOST), torch.full((1, MOST), float("nan"), dtype=BF16, device=DEV)
    # spread over the many columns: each of them is a product of its own
    spread = (lambda: ctx.linear_grad_input(W, 0, one, rows, wide)) if wide_in else (lambda: ctx.linear(W, 0, one, rows, wide))
    spread()
    assert all(float(wide[0, k]) == 6.0 for k in at) and sum(int((part != 0).sum()) for part in wide[0].split(1 << 28)) == len(at)
    if wide_in:                                       # summed over them
        total = torch.zeros(1, 1, dtype=BF16, device=DEV)
        ctx.linear(W, 0, wide.fill_(1.0), rows, total)
        assert float(total) == 3.0 * len(at)
    G = torch.full((1, MOST), 7.0, device=DEV)
    if wide_in:
        ctx.linear_grad_weight(one, W, rows, G, 0)
    else:
        ctx.linear_grad_weight(W, one, rows, G, 0)
    assert all(float(G[0, k]) == 6.0 for k in at) and sum(int((part != 0).sum()) for part in G[0].split(1 << 28)) == len(at)

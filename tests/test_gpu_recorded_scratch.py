"""What a recorded call reads and writes of its context's memory outlives other calls on the same context."""
import pytest
import torch

import paper_2006_08085_amd as D

pytestmark = pytest.mark.gpu
DEV, F32 = "cuda:0", torch.float32


def _free():
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    return torch.cuda.mem_get_info()[0]


def _offsets(n, M):
    return torch.tensor([i * M // n for i in range(n + 1)], dtype=torch.int32, device=DEV)


def test_a_recorded_loss_after_a_larger_one():
    n, M, C, many = 2, 1300, 10, 1 << 26             # 2^26 rows are 512 MiB of scratch
    ctx = D.detag_create(D.Topology.ring(), n, 4, 4)
    g = torch.Generator(device=DEV).manual_seed(1)
    z = torch.randn(M, C, generator=g, device=DEV)
    labels = torch.randint(-1, C, (M,), generator=g, device=DEV, dtype=torch.int32)
    rows, grad, loss = _offsets(n, M), torch.zeros(M, C, device=DEV), torch.zeros(n, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(D.DetagError, match="detag_reserve_cross_entropy"):
            ctx.cross_entropy(z, labels, rows, grad, loss)
        loss.add_(0)                                  # so that the recording holds some node
    at_start = _free()
    ctx.reserve_cross_entropy(many)
    ctx.reserve_cross_entropy(2 * many)               # nobody has recorded the first: it is freed
    first = at_start - _free()
    assert 0.9 < first / (many * 16) < 1.1
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.cross_entropy(z, labels, rows, grad, loss)
    ctx.reserve_cross_entropy(3 * many)               # a recorded one stays
    assert 0.95 < (at_start - _free()) / (5 * many * 8) < 1.05
    want, want_loss = torch.empty_like(grad), torch.empty_like(loss)
    for k in range(4):
        z.copy_(torch.randn(M, C, generator=g, device=DEV))
        grad.fill_(7.0)
        graph.replay()
        ctx.cross_entropy(z, labels, rows, want, want_loss)
        assert torch.equal(grad, want) and torch.equal(loss, want_loss), k
    ctx.reserve_cross_entropy(3 * many)
    ctx.reserve_cross_entropy(4 * many)               # the eager calls recorded nothing
    assert 0.95 < (at_start - _free()) / (6 * many * 8) < 1.05
    del graph
    ctx.close()
    assert at_start - _free() < many


def test_a_recorded_gradient_after_a_larger_loss():
    n, d, m = 4, 700, 40
    ctx = D.detag_create(D.Topology.ring(), n, d, 704)
    g = torch.Generator(device=DEV).manual_seed(2)
    X, G, want = torch.randn(n, 704, generator=g, device=DEV), D.new_matrix(n, d, 704), D.new_matrix(n, d, 704)
    A, b = torch.randn(n, m, d, generator=g, device=DEV), torch.randn(n, m, generator=g, device=DEV)
    ctx.reserve_gradient(m=m)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.grad_lstsq(X, A, b, G)
    M = 1 << 20
    rows, labels, z = _offsets(n, M), torch.zeros(M, dtype=torch.int32, device=DEV), torch.zeros(M, 3, device=DEV)
    for k in range(4):
        ctx.cross_entropy(z, labels, rows, z)
        X.copy_(torch.randn(n, 704, generator=g, device=DEV))
        G.zero_()
        graph.replay()
        ctx.grad_lstsq(X, A, b, want)
        # the sums' order may differ between the recorded form and the eager one: 40 + 700 terms in fp32
        assert torch.allclose(G[:, :d], want[:, :d], rtol=1e-4, atol=1e-2), k
    del graph


def test_a_recorded_polynomial_after_others():
    """The context keeps four polynomials of the dense path; a fifth one takes the place of the oldest, but not under a recorded call."""
    n, d = 24, 1000
    ctx = D.detag_create(D.Topology.ring(), n, d, 1024)
    ctx.set_path(D.DETAG_PATH_DENSE)
    g = torch.Generator(device=DEV).manual_seed(3)
    Z = torch.randn(n, 1024, generator=g, device=DEV)
    want, start = Z.clone(), Z.clone()
    ctx.gossip_accel(want, 5)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.gossip_accel(Z, 5)
    for K in (1, 2, 3, 4, 6, 7, 8, 9, 5):
        other = start.clone()
        ctx.gossip_accel(other, K)
        assert torch.equal(other, want) == (K == 5)
        Z.copy_(start)
        graph.replay()
        assert torch.equal(Z, want), K
    del graph

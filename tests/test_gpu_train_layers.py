"""The products, the cross-entropy and AdamW together, as `train_layers` runs them, and the two ways to call them."""
import numpy as np
import pytest
import torch

import paper_2006_08085_amd as D
from paper_2006_08085_amd import train_layers

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("bits", [32, 8])
def test_workers_on_uneven_batches_learn(bits):
    """Ten classes: 2.3 nats and a tenth right before the first step.  The mean model has to know classes of which a worker saw few."""
    log = list(train_layers.train(workers=16, steps=150, bits=bits, records=3))
    assert [r["step"] for r in log] == [50, 100, 150]
    assert log[-1]["loss"] < 0.8 and log[-1]["accuracy_of_mean_model"] > 0.8
    assert np.isfinite(log[-1]["consensus_distance"])


def test_one_worker_and_one_step():
    log = list(train_layers.train(workers=1, steps=1))
    assert len(log) == 1 and log[0]["consensus_distance"] == 0.0


def test_both_ways_accept_the_same_and_give_the_same(monkeypatch):
    """The native form of the calls, and ctypes."""
    n, inn, out, M = 5, 72, 40, 90
    dev = "cuda"
    d = inn * out + 6
    ctx = D.detag_create(D.Topology.ring(), n, d, D.padded_ld(d))
    g = torch.Generator(device=dev).manual_seed(1)
    W = torch.randn(n, ctx.ld, device=dev, generator=g)
    A, dY = torch.randn(M, inn, device=dev, generator=g), torch.randn(M, out, device=dev, generator=g)
    labels = torch.randint(out, (M,), dtype=torch.int32, device=dev, generator=g)
    rows = torch.tensor([0, 10, 10, 33, 64, 88], dtype=torch.int32, device=dev)
    opts = {bits: D.AdamW(ctx, [(0, 100), (100, d - 100)], [0.1, 0.0], bits=bits) for bits in (32, 8)}

    def everything(f=float, i=int):
        kept = []
        for t in (torch.float32, BF16):
            w, a, y = W.to(t), A.to(t), dY.to(t, copy=True)  # y is overwritten below
            results = [torch.zeros(M, out, dtype=t, device=dev) for _ in range(3)] + [torch.zeros(M, out, device=dev)]
            grads, G, loss = [torch.zeros(M, inn, dtype=t, device=dev) for _ in range(2)], torch.zeros(n, ctx.ld, device=dev), torch.zeros(n, device=dev)
            ctx.linear(w, i(3), a, rows, results[0])
            ctx.linear(w, i(3), a, rows, results[1], relu=True)
            ctx.linear(w, i(3), a, rows, results[3], True)
            ctx.linear_grad_input(w, i(3), y, rows, grads[0])
            ctx.linear_grad_input(w, i(3), y, rows, grads[1], relu_of=a)
            ctx.linear_grad_weight(y, a, rows, G, i(3))
            ctx.linear_grad_weight(y, a, rows, G, i(3), accumulate=True)
            ctx.cross_entropy(y, labels, rows, results[2], loss)
            ctx.cross_entropy(y, labels, rows, y)
            kept += [*results, *grads, G, loss, y]
            for bits, opt in opts.items():
                X, (m, v, s), copy = W.clone(), opt.new_moments(dev), torch.zeros(n, ctx.ld, dtype=BF16, device=dev)
                opt.step(X, G, m, v, s, lr=f(0.5), t=i(1))
                opt.step(X, G, m, v, s, lr=f(0.01), t=i(2), beta1=f(0.8), beta2=f(0.9), eps=f(1e-6), limit=f(3), seed=i(7), X16=copy)
                kept += [X, m, v, copy]
                if bits == 8:
                    for o in (torch.float32, BF16):
                        m_out, v_out = (torch.zeros(n, ctx.ld, dtype=o, device=dev) for _ in range(2))
                        opt.values(m, v, s, m_out, v_out)
                        kept += [s, m_out, v_out]
        torch.cuda.synchronize()
        return kept

    native = everything()
    odd = everything(f=np.float64)
    Y, X, loss = torch.zeros(M, out, device=dev), W.clone(), torch.zeros(n, device=dev)
    m, v, s = opts[8].new_moments(dev)
    refusals = [(ValueError, lambda: ctx.linear(W, 0, A, rows, Y[:4])), (ValueError, lambda: ctx.linear(W.double(), 0, A, rows, Y)),
                (ValueError, lambda: ctx.linear(W, 0, A.t(), rows, Y)), (ValueError, lambda: ctx.linear(W, 0, A, rows[::2], Y)),
                (D.DetagError, lambda: ctx.linear(W, 7, A, rows, Y)), (ValueError, lambda: ctx.linear_grad_input(W, 0, dY, rows, A, relu_of=Y)),
                (ValueError, lambda: ctx.linear_grad_weight(dY, A[:-1], rows, X, 0)), (ValueError, lambda: ctx.cross_entropy(Y, rows, rows, Y)),
                (ValueError, lambda: ctx.cross_entropy(Y, labels, rows, Y, loss.double())), (ValueError, lambda: opts[32].step(X, W, m, v, lr=0.1, t=1)),
                (D.DetagError, lambda: opts[8].step(X, W, m, v, lr=0.1, t=1)), (D.DetagError, lambda: opts[8].step(X, W, m, v, s, lr=0.1, t=0)),
                (ValueError, lambda: opts[8].step(X, W, m, v, s[:, 1:], lr=0.1, t=1)), (ValueError, lambda: opts[8].values(m, v, s, X, X[:2])),
                (ValueError, lambda: opts[8].step(X, W, m, v, s, lr=0.1, t=1, X16=X))]

    def refused():
        words = []
        for kind, call in refusals:
            with pytest.raises(kind) as e:
                call()
            words.append(str(e.value))
        return words
    said = refused()

    class Nothing:
        def __getattr__(self, name):
            return lambda *a: None

    monkeypatch.setattr(ctx, "_fast", Nothing())
    by_ctypes = everything()
    assert refused() == said
    for one in (odd, by_ctypes):
        assert all(torch.equal(a, b) for a, b in zip(native, one))


@pytest.mark.parametrize("dtype,pitch", [(BF16, 0), (BF16, 6), (torch.float32, 0), (torch.float32, 3)])
@pytest.mark.parametrize("counts", [[1500], [0, 64, 63, 65, 1, 320, 700], [4097, 255]], ids=["one", "ragged", "two"])
def test_weight_gradients_of_small_layers_and_many_rows(counts, dtype, pitch):
    """Sums over many rows whose parts are added up at the end, to (K + 8) 2^-24 of the magnitudes, doubled."""
    inn, out, n, M, dev = 72, 134, len(counts), sum(counts), "cuda"
    ctx = D.detag_create(D.Topology.ring(), n, inn * out, inn * out)
    g = torch.Generator().manual_seed(M)
    dY, A = (torch.randn(M + 3, c + pitch, generator=g).to(dtype).to(dev)[:, :c] for c in (out, inn))
    dY[M:], A[M:] = float("nan"), float("inf")
    rows = torch.tensor([0, *np.cumsum(counts)], dtype=torch.int32, device=dev)
    G = torch.randn(n, inn * out, generator=g).to(dev)
    start = G.double().view(n, out, inn)
    for accumulate in (True, False):
        ctx.linear_grad_weight(dY, A, rows, G, 0, accumulate=accumulate)
        for i in range(n):
            y, a = dY[rows[i]:rows[i + 1]].double(), A[rows[i]:rows[i + 1]].double()
            ref, size = y.t() @ a, y.abs().t() @ a.abs()
            if accumulate:
                ref, size = ref + start[i], size + start[i].abs()
            off = (G[i].double().view(out, inn) - ref).abs()
            assert (off <= 2 * (counts[i] + 8) * 2.0 ** -24 * size + 2 * 2.0 ** -24 * ref.abs() + 1e-37).all()

"""The operators of a residual block together: a network's gradients, graphs, streams, refusals, and the two ways to call them."""
import math

import pytest
import torch

import paper_2006_08085_amd as D
from paper_2006_08085_amd import train_blocks
from tests.block_util import ACTS, BF16, DEV, F32, U, _built, context, matrix, normal, offsets, parameters, spans  # noqa: F401
from tests.test_gpu_dropout import kept

pytestmark = pytest.mark.gpu


def test_the_example_runs():
    log = list(train_blocks.train(workers=4, steps=6, records=3))
    assert [r["step"] for r in log] == [2, 4, 6] and all(math.isfinite(v) for r in log for v in r.values())
    assert len(list(train_blocks.train(workers=1, steps=1))) == 1


def _reference_loss(net, P, A, labels, counts, seq_counts, step, seed, p):
    """The network's mean loss of every worker, summed, in 64 bits, from its formulas; P requires gradients."""
    total, sequences = 0.0, list(spans(seq_counts))
    for i, lo, hi in spans(counts):
        if hi == lo:
            continue

        def layer(name, x):
            w, b = net.at[name]
            inn, out = net.shapes[name]
            return x @ P[i, w:b].view(out, inn).t() + P[i, b:b + out]

        def norm(name, x):
            w, b = net.at[name]
            x = x - x.mean(1, keepdim=True)
            return x / torch.sqrt(x.pow(2).mean(1, keepdim=True) + 1e-5) * P[i, w:b] + P[i, b:b + net.C]

        def drop(x, which):
            mask = kept(hi - lo, net.C, i, p, which + (seed << 8), step).to(DEV)
            return x * mask * (65536 / (65536 - math.floor(65536 * p + 0.5)))
        x = layer("in", A[lo:hi].double())
        for k in range(net.blocks):
            qkv = layer(f"qkv.{k}", norm(f"norm1.{k}", x))
            width, mixed = net.C // net.heads, []
            for _, s0, s1 in sequences:
                if lo <= s0 < s1 <= hi:
                    here = qkv[s0 - lo:s1 - lo]
                    seen, heads = torch.ones(s1 - s0, s1 - s0, device=DEV).tril().bool(), []
                    for j in range(net.heads):
                        m = net.heads + j // (net.heads // net.kv_heads)
                        q, key, v = (here[:, a * width:(a + 1) * width] for a in (j, m, m + net.kv_heads))
                        heads.append(torch.softmax((q @ key.t() / math.sqrt(width)).masked_fill(~seen, -math.inf), 1) @ v)
                    mixed.append(torch.cat(heads, 1))
            x = x + drop(layer(f"out.{k}", torch.cat(mixed)), 2 * k)
            h = layer(f"up.{k}", norm(f"norm2.{k}", x))
            x = x + drop(layer(f"down.{k}", h * normal(h)), 2 * k + 1)
        z = layer("classes", norm("norm", x))
        total = total + torch.nn.functional.cross_entropy(z, labels[lo:hi].long(), reduction="mean")
    return total


@pytest.mark.parametrize("dtype,p", [(F32, 0.25), (F32, 0.0), (BF16, 0.25)])
def test_a_networks_gradients(dtype, p):
    """Every parameter's gradient of two blocks, against automatic differentiation of the formulas in 64 bits.  Relative to the norm of a
    tensor's gradient: fp32 1e-4 (sums of up to 64 terms through some thirty operators, each within 100 u of its magnitudes: 2e-4 if all were in
    line); bf16 0.1 (some thirty roundings of 2^-8 in a row: 0.12 if all were in line)."""
    seq_counts, counts = [5, 1, 12, 7, 9, 3], [18, 0, 16, 3]          # sequences of worker 0, 2 and 3
    n, M = len(counts), sum(counts)
    net = train_blocks.Network(n, most=64, dtype=dtype, dropout=p)
    gen = torch.Generator(device=DEV).manual_seed(3)
    X = D.new_matrix(n, net.columns, device=DEV)
    net.start(X, gen)
    X += 0.05 * torch.randn(X.shape, device=DEV, generator=gen)
    P = X.to(dtype)
    A = torch.randn(64, train_blocks.INPUTS, device=DEV, generator=gen).to(dtype)
    labels = torch.randint(train_blocks.CLASSES, (64,), dtype=torch.int32, device=DEV, generator=gen)
    rows, seqs = offsets(counts), offsets(seq_counts)
    loss, dlogits, G = torch.zeros(n, device=DEV), torch.zeros_like(net.logits), torch.zeros(n, net.ctx.ld, device=DEV)
    logits = net.forward(P, A, rows, seqs, step=4)
    net.ctx.cross_entropy(logits, labels, rows, dlogits, loss)
    net.backward(P, A, rows, seqs, dlogits, G)
    P64 = P.double().requires_grad_(True)
    ref = _reference_loss(net, P64, A, labels, counts, seq_counts, 4, 1, p)
    ref.backward()
    most = 1e-4 if dtype is F32 else 0.1
    assert abs(loss.sum().item() - ref.item()) <= most * ref.item()
    for i in range(n):
        for first, length in net.spans:
            got, want = G[i, first:first + length].double(), P64.grad[i, first:first + length]
            # the keys' bias has no gradient: softmax does not see it; what is left there is rounding
            assert (got - want).norm() <= most * max(want.norm().item(), 0.05 * P64.grad[i].norm().item()), (i, first)
    assert not G[1, :net.columns].any()                                # a worker without rows


def test_a_captured_step_replays_like_the_eager_one():
    """Forward and backward as a graph, replayed on new inputs, with eager work of the same context between the replays."""
    counts, seq_counts = [20, 9, 30], [20, 4, 5, 30]
    nets = [train_blocks.Network(3, most=64) for _ in range(2)]
    gen = torch.Generator(device=DEV).manual_seed(3)
    X = D.new_matrix(3, nets[0].columns, device=DEV)
    nets[0].start(X, gen)
    P, rows, seqs = X.bfloat16(), offsets(counts), offsets(seq_counts)
    A = torch.zeros(64, train_blocks.INPUTS, dtype=BF16, device=DEV)
    labels, loss = torch.zeros(64, dtype=torch.int32, device=DEV), torch.zeros(3, device=DEV)

    def step(net, G, dlogits):
        logits = net.forward(P, A, rows, seqs, step=2)
        net.ctx.cross_entropy(logits, labels, rows, dlogits, loss)
        net.backward(P, A, rows, seqs, dlogits, G)
    G = [torch.zeros(3, nets[0].ctx.ld, device=DEV) for _ in range(2)]
    dlogits = [torch.zeros_like(nets[0].logits) for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(nets[0], G[0], dlogits[0])
    for k in range(4):
        A.copy_(torch.randn(A.shape, device=DEV, generator=gen))
        labels.random_(0, 10, generator=gen)
        G[0].zero_()
        graph.replay()
        step(nets[1], G[1], dlogits[1])
        torch.cuda.synchronize()
        assert torch.equal(G[0], G[1]) and torch.equal(dlogits[0], dlogits[1]) and G[0].abs().sum() > 0


def test_scratch_during_a_capture_and_after():
    """Without a reservation a call that is being captured is refused; a recorded one keeps its scratch when a larger call comes."""
    n, C, M = 2, 64, 40
    ctx = context(n, 2 * C)
    P = parameters(n, ctx.ld, F32, [(0, 2 * C, 0.5, 0.1)], 1)
    X, dY = matrix(M, C, F32, 2)[0], matrix(M, C, F32, 3)[0]
    rows, G, dX = offsets([30, 10]), torch.zeros(n, ctx.ld, device=DEV), torch.zeros_like(X)
    O, lse, dK, dV = torch.zeros_like(X), torch.zeros(4, M, device=DEV), torch.zeros_like(X), torch.zeros_like(X)
    torch.cuda.synchronize()
    calls = (lambda: ctx.layer_norm_grad(P, 0, C, X, dY, rows, dX, G), lambda: ctx.linear_grad_bias(dY, rows, G, 0),
             lambda: ctx.attention_grad(X, X, X, rows, O, lse, dY, dX, dK, dV, 4, 4))
    for call in calls:
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            with pytest.raises(D.DetagError, match="captured") as e:
                call()
            X.add_(0.0)                                                # a graph of nothing is warned about
        assert e.value.status == D.DETAG_EINVAL
    ctx.reserve_layer_gradient(M, C)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls[0]()
    ctx.reserve_attention(100000, 8)                                   # larger: another allocation
    X.mul_(2.0)
    for _ in range(3):
        graph.replay()
        got = dX.clone(), G.clone()
        calls[0]()
        torch.cuda.synchronize()
        assert torch.equal(got[0], dX) and torch.equal(got[1], G)


def test_calls_on_another_stream():
    """Each operator on a side stream, its inputs made there, gives what it gives on the default one."""
    counts, C = [30, 34], 64
    M, n = sum(counts), len(counts)
    ctx = context(n, C * C + 3 * C)
    rows, side = offsets(counts), torch.cuda.Stream()

    def run():
        g = torch.Generator(device=DEV).manual_seed(5)
        P = torch.randn(n, ctx.ld, device=DEV, generator=g)
        X, dY = torch.randn(M, C, device=DEV, generator=g), torch.randn(M, C, device=DEV, generator=g)
        out = [torch.zeros_like(X) for _ in range(9)]
        G, lse = torch.zeros(n, ctx.ld, device=DEV), torch.zeros(4, M, device=DEV)
        ctx.layer_norm(P, 0, C, X, rows, out[0])
        ctx.linear_act(P, 2 * C, out[0], rows, out[1], bias=C, act=ACTS["silu"], pre=out[2], residual=X)
        ctx.attention(out[1], out[1], out[1], rows, out[3], 4, 4, lse=lse)
        ctx.attention_grad(out[1], out[1], out[1], rows, out[3], lse, dY, out[4], out[5], out[6], 4, 4)
        ctx.linear_grad_bias(out[4], rows, G, C, act=ACTS["silu"], pre=out[2], dZ=out[7])
        ctx.layer_norm_grad(P, 0, 2 * C, X, out[7], rows, out[8], G, accumulate=True)
        ctx.dropout(out[8], rows, out[8], p=0.3, seed=1, step=1)
        return [*out, G, lse]
    here = run()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there = run()
    side.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(here, there))


def _arguments(dtype=F32):
    n, C, M, out = 3, 32, 20, 48
    ctx = context(n, C * out + out + 2 * C)
    g = torch.Generator(device=DEV).manual_seed(2)
    W = torch.randn(n, ctx.ld, device=DEV, generator=g).to(dtype)
    A, B, Y = (torch.randn(M, c, device=DEV, generator=g).to(dtype) for c in (C, C, out))
    return ctx, n, C, M, out, W, A, B, Y, offsets([8, 0, 12]), torch.zeros(n, ctx.ld, device=DEV)


class _Nothing:
    def __getattr__(self, name):
        return lambda *a: None


def test_both_ways_accept_the_same_and_give_the_same(monkeypatch):
    import numpy as np
    for dtype in (F32, BF16):
        ctx, n, C, M, out, W, A, B, Y, rows, G0 = _arguments(dtype)
        b = C * out

        def everything(f=float, i=int):
            G, lse, kept_ = G0.clone(), torch.zeros(4, M, device=DEV), []

            def new(t):
                kept_.append(torch.zeros_like(t))
                return kept_[-1]
            wide = torch.zeros(M, out, device=DEV)
            ctx.linear_act(W, i(0), A, rows, new(Y))
            z = new(Y)
            ctx.linear_act(W, i(0), A, rows, new(Y), bias=i(b), act=i(2), pre=z, residual=Y)
            ctx.linear_act(W, 0, A, rows, wide, b, 3, None, wide)
            ctx.linear_grad_bias(Y, rows, G, i(b))
            ctx.linear_grad_bias(Y, rows, G, b, act=2, pre=z, dZ=new(Y), accumulate=True)
            ctx.linear_grad_input_act(W, 0, Y, rows, new(A))
            ctx.linear_grad_input_act(W, 0, Y, rows, new(A), act=1, pre=A)
            ctx.layer_norm(W, b, None, A, rows, new(A))
            ctx.layer_norm(W, i(b), i(b + C), A, rows, new(A), eps=f(1e-3))
            ctx.layer_norm_grad(W, b, b + C, A, B, rows, new(A), G, add=B, accumulate=True)
            ctx.layer_norm_grad(W, b, None, A, B, rows, new(A), G, eps=f(0.5))
            ctx.dropout(A, rows, new(A), p=f(0.5), seed=i(7), step=i(1))
            ctx.dropout(A, rows, new(A), 0.25, 1 << 40, 2, B)
            o = new(A)
            ctx.attention(A, B, B, rows, o, 4, 4, lse=lse)
            ctx.attention(A, B[:, :16], B[:, 16:], rows, new(A), i(4), i(2), causal=False, scale=f(0.5))
            ctx.attention_grad(A, B, B, rows, o, lse, A, new(A), new(A), new(A), 4, 4)
            torch.cuda.synchronize()
            return [*kept_, G, lse, wide]
        native, odd = everything(), everything(f=np.float64)
        with monkeypatch.context() as m:
            m.setattr(ctx, "_fast", _Nothing())
            by_ctypes = everything()
        for one in (odd, by_ctypes):
            assert all(torch.equal(a, c) for a, c in zip(native, one))


def test_refusals(monkeypatch):
    """No launch follows: outputs stay as they are; both ways of calling word them alike."""
    ctx, n, C, M, out, W, A, B, Y, rows, G = _arguments()
    b, V, E = C * out, ValueError, D.DetagError
    o, o2, lse, y = torch.full_like(A, 9.0), torch.full_like(A, 9.0), torch.full((4, M), 9.0, device=DEV), torch.full_like(Y, 9.0)
    half = o.bfloat16()
    cases = [
        (V, lambda: ctx.linear_act(W, 0, A, rows, y, residual=A)), (V, lambda: ctx.linear_act(W, 0, A, rows, y, pre=half)),
        (V, lambda: ctx.linear_act(W, 0, A, rows, y, bias=-3)), (V, lambda: ctx.linear_act(W.double(), 0, A, rows, y)),
        (V, lambda: ctx.linear_act(W, 0, A, rows, y, residual=Y.bfloat16())), (V, lambda: ctx.linear_act(W, 0, A.t(), rows, y)),
        (E, lambda: ctx.linear_act(W, 0, A, rows, y, act=4)), (E, lambda: ctx.linear_act(W, 0, A, rows, y, act=-1)),
        (E, lambda: ctx.linear_act(W, 0, A, rows, y, bias=ctx.d - out + 1)), (E, lambda: ctx.linear_act(W, ctx.d, A, rows, y)),
        (E, lambda: ctx.linear_act(W, 0, A, rows, y, pre=y)), (E, lambda: ctx.linear_act(W, 0, o[:, :], rows, o)),
        (E, lambda: ctx.linear_grad_bias(Y, rows, G, b, act=1)), (E, lambda: ctx.linear_grad_bias(Y, rows, G, b, pre=Y)),
        (E, lambda: ctx.linear_grad_bias(Y, rows, G, b, dZ=y)), (E, lambda: ctx.linear_grad_bias(Y, rows, G, -1)),
        (E, lambda: ctx.linear_grad_bias(Y, rows, G, ctx.d - out + 1)), (V, lambda: ctx.linear_grad_bias(Y, rows, G.bfloat16(), b)),
        (V, lambda: ctx.linear_grad_bias(Y, rows[:-1], G, b)), (V, lambda: ctx.linear_grad_bias(Y, rows, G, b, act=2, pre=A, dZ=y)),
        (E, lambda: ctx.linear_grad_input_act(W, 0, Y, rows, o, act=2)), (E, lambda: ctx.linear_grad_input_act(W, 0, Y, rows, o, pre=A)),
        (E, lambda: ctx.linear_grad_input_act(W, 0, Y, rows, o, act=2, pre=o)), (V, lambda: ctx.linear_grad_input_act(W, 0, Y, rows, o, act=2, pre=Y)),
        (E, lambda: ctx.layer_norm(W, -1, None, A, rows, o)), (E, lambda: ctx.layer_norm(W, 0, ctx.d - C + 1, A, rows, o)),
        (E, lambda: ctx.layer_norm(W, 0, None, A, rows, o, eps=0.0)), (E, lambda: ctx.layer_norm(W, 0, None, A, rows, o, eps=float("nan"))),
        (E, lambda: ctx.layer_norm(W, 0, None, A, rows, o, eps=1e300)), (E, lambda: ctx.layer_norm(W, 0, None, A, rows, o, eps=1e-60)),
        (V, lambda: ctx.layer_norm(W, 0, None, A, rows, half)), (V, lambda: ctx.layer_norm(W, 0, -1, A, rows, o)),
        (V, lambda: ctx.layer_norm(W, 0, None, A, rows, o[:, 1:])), (V, lambda: ctx.layer_norm(W, 0, None, A, rows.long(), o)),
        (E, lambda: ctx.layer_norm_grad(W, 0, C - 1, A, B, rows, o, G)), (E, lambda: ctx.layer_norm_grad(W, 5, 5, A, B, rows, o, G)),
        (V, lambda: ctx.layer_norm_grad(W, 0, C, A, Y, rows, o, G)), (V, lambda: ctx.layer_norm_grad(W, 0, C, A, B, rows, o, G, add=Y)),
        (E, lambda: ctx.dropout(A, rows, o, p=1.0, seed=1, step=1)), (E, lambda: ctx.dropout(A, rows, o, p=-0.1, seed=1, step=1)),
        (E, lambda: ctx.dropout(A, rows, o, p=float("nan"), seed=1, step=1)), (E, lambda: ctx.dropout(A, rows, o, p=1 - 2.0 ** -18, seed=1, step=1)),
        (V, lambda: ctx.dropout(A, rows, y, p=0.1, seed=1, step=1)), (V, lambda: ctx.dropout(A, rows, o, p=0.1, seed=1, step=1, residual=half)),
        (V, lambda: ctx.attention(A, B, B, rows, o, 5, 5)), (V, lambda: ctx.attention(A, B, B, rows, o, 4, 2)),
        (V, lambda: ctx.attention(A, B, B, rows, y, 4, 4)), (V, lambda: ctx.attention(A, B, half, rows, o, 4, 4)),
        (V, lambda: ctx.attention(A, B[:-1], B, rows, o, 4, 4)), (V, lambda: ctx.attention(A, B, B, rows.long(), o, 4, 4)),
        (V, lambda: ctx.attention(A, B, B, rows[:0], o, 4, 4)), (V, lambda: ctx.attention(A, B, B, rows, o, 4, 4, lse=lse[:, 1:])),
        (V, lambda: ctx.attention(A, B, B, rows, o, 4, 4, lse=lse[:2])), (E, lambda: ctx.attention(A, B, B, rows, o, 4, 4, scale=0.0)),
        (E, lambda: ctx.attention(A, B[:, :24], B[:, :24], rows, o, 4, 3)), (E, lambda: ctx.attention(A, B, B, rows, o, 4, 4, scale=float("inf"))),
        (E, lambda: ctx.attention(o, B, B, rows, o, 4, 4)), (E, lambda: ctx.attention_grad(A, B, B, rows, o2, lse, A, o, o, o, 4, 4)),
        (E, lambda: ctx.attention_grad(A, B, B, rows, o2, lse, A, A, o, o, 4, 4)), (V, lambda: ctx.attention_grad(A, B, B, rows, o2, None or lse[:3], A, o, o, o, 4, 4)),
        (E, lambda: ctx.reserve_attention(-1, 2)), (E, lambda: ctx.reserve_attention(4, 0)), (E, lambda: ctx.reserve_layer_gradient(4, 0)),
        (E, lambda: ctx.reserve_layer_gradient(-1, 8)),
    ]

    def refused():
        words = []
        for k, (kind, call) in enumerate(cases):
            with pytest.raises(kind) as e:
                call()
                pytest.fail(f"case {k} was accepted")
            words.append(str(e.value))
        return words
    said = refused()
    with monkeypatch.context() as m:
        m.setattr(ctx, "_fast", _Nothing())
        assert refused() == said
    torch.cuda.synchronize()
    assert all((t == 9.0).all() for t in (o, o2, lse, y)) and not G.any()
    big = torch.zeros(1, 16385, device=DEV)
    far = context(1, 2 * 16385)
    P, r1 = torch.zeros(1, far.ld, device=DEV), offsets([1])
    wide = torch.zeros(1, 129, device=DEV)
    for call in (lambda: far.layer_norm(P, 0, None, big, r1, big), lambda: far.layer_norm_grad(P, 0, None, big, big.clone(), r1, big, P.clone()),
                 lambda: far.attention(wide, wide.clone(), wide.clone(), r1, wide.clone(), 1, 1)):
        with pytest.raises(D.DetagError) as e:
            call()
        assert e.value.status == D.DETAG_EUNSUPPORTED


def test_in_place_needs_one_pitch():
    ctx, n, C, M, out, W, A, B, Y, rows, G = _arguments()
    buf = torch.zeros(M * 64, device=DEV)
    one, other = buf.view(M, 64)[:, :C], buf[:M * 40].view(M, 40)[:, :C]
    for call in (lambda: ctx.layer_norm(W, 0, None, one, rows, other), lambda: ctx.dropout(one, rows, other, p=0.1, seed=1, step=1),
                 lambda: ctx.layer_norm_grad(W, 0, None, one, B, rows, other, G), lambda: ctx.layer_norm_grad(W, 0, None, A, B, rows, other, G, add=one),
                 lambda: ctx.linear_grad_bias(one, rows, G, 0, act=2, pre=B, dZ=other)):
        with pytest.raises(D.DetagError, match="pitches"):
            call()


def test_calls_of_no_rows():
    """Nothing to write but the sums, which are zero, or stay."""
    ctx, n, C, M, out, W, A, B, Y, rows, G = _arguments()
    none, zero = torch.zeros(0, C, device=DEV), torch.zeros(n + 1, dtype=torch.int32, device=DEV)
    ctx.layer_norm(W, 0, C, none, zero, none.clone())
    ctx.dropout(none, zero, none.clone(), p=0.1, seed=1, step=1)
    ctx.linear_act(W, 0, none, zero, torch.zeros(0, out, device=DEV), bias=5, act=2)
    ctx.attention(none, none.clone(), none.clone(), zero, none.clone(), 4, 4)
    ctx.attention(A, B, B, zero[:1], torch.zeros_like(A), 4, 4)         # no sequences
    G.fill_(3.0)
    ctx.linear_grad_bias(none, zero, G, 2, accumulate=True)
    ctx.layer_norm_grad(W, 0, C, none, none.clone(), zero, none.clone(), G, accumulate=True)
    assert (G == 3.0).all()
    ctx.linear_grad_bias(none, zero, G, 2 * C)
    ctx.layer_norm_grad(W, 0, C, none, none.clone(), zero, none.clone(), G)
    assert not G[:, :3 * C].any() and (G[:, 3 * C:] == 3.0).all()


@pytest.mark.parametrize("most", [1, 100, 257, 2047, 2048, 7680, 7681, 20000])
def test_a_reservation_serves_any_fewer_rows(most):
    """Captured calls of fewer rows than reserved are not refused for want of scratch."""
    n, C = 3, 40
    for rows in sorted({r for r in (1, 255, 256, 257, 2047, 2048, 5000, 7679, 7680, 7681, 9000, 20000, most) if r <= most}):
        ctx = context(n, 2 * C)
        ctx.reserve_layer_gradient(most, C)
        P, G = torch.ones(n, ctx.ld, device=DEV), torch.zeros(n, ctx.ld, device=DEV)
        X = torch.randn(rows, C, device=DEV)
        offs, dX, ones = offsets([rows // 3, 0, rows - rows // 3]), torch.zeros_like(X), torch.ones_like(X)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ctx.layer_norm_grad(P, 0, C, X, ones, offs, dX, G)
            ctx.linear_grad_bias(ones, offs, G, 0, accumulate=True)
        graph.replay()
        torch.cuda.synchronize()
        # ones, added up exactly; the rows' xhat have a mean of zero, so the gain's gradient adds little to the first of them
        assert G[0, C:2 * C].eq(rows // 3).all() and G[2, C:2 * C].eq(rows - rows // 3).all() and not G[1, :2 * C].any()


def test_numbers_that_a_launch_or_fp32_does_not_hold_are_refused():
    """A bias of more columns than a launch has threads for (2^32, at 16 a column), and scales whose exponent of two passes fp32."""
    d = 2 ** 28
    far = D.detag_create(D.Topology.ring(), 4, d, d)
    small, off = torch.full((64,), 9.0, device=DEV), offsets([1, 1, 1, 1])
    L, at, F = D.lib(), small.data_ptr(), D.DETAG_F32
    for rows in (0, 4):
        st = L.detag_linear_grad_bias(far._h, F, at, d, 0, None, 0, off.data_ptr(), rows, 2 ** 27 + 1, None, 0, at + 128, 0, 0, None)
        assert st == D.DETAG_EUNSUPPORTED and b"2^27" in L.detag_last_error(far._h)
    Q = small[:16].view(4, 4)
    for scale in (2.4e38, 3.4e38):  # the largest of fp32 is 3.4028e38; divided by log2(e) 2.3587e38
        with pytest.raises(D.DetagError, match="log2"):
            far.attention(Q, Q, Q, off, small[16:32].view(4, 4), 1, 1, scale=scale)
    torch.cuda.synchronize()
    assert (small == 9.0).all()
    zero = torch.zeros(4, 4, device=DEV)
    out = torch.empty_like(zero)
    far.attention(zero, zero, Q, off, out, 1, 1, scale=2.3e38)  # scores of zero
    assert (out == 9.0).all()

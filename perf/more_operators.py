"""The operators of a residual block of every worker's network, as measurable cases.

n simulated workers learn a network of residual blocks: every worker has its own parameters (slices of its row of the n x ld model
matrix) and its own rows, and attention works within the packed sequences that the rows are cut into.  The cases are passes of

  norm            layer norm of every row, with the gain and bias of the row's worker
  norm_grad       its gradient: of the rows, plus the gradient that comes past the block, and of every worker's gain and bias
  affine          a layer's product with its epilogue: Y = R + act(A W_i^T + b_i), with or without bias, activation, residual, and
                  the sums before the activation for the way back
  affine_grad     the gradient of the epilogue and of the activation below: dZ = dY act'(Z) and the bias's, dA = (dZ W_i) act'(Z_below)
  dropout         a share of the entries set to zero by a counter-based generator, the others scaled, added to the residual
  attention       softmax attention within packed sequences, causal or not, query heads sharing key heads
  attention_grad  its gradient

run() computes them in elementary torch operations where `own` is false, and through the library's entry points where it is true;
exact() restates them in 64 bits.
"""
import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5
STEP = 7


def _norm(name, n, M, C, dtype="bf16", kind="norm", offset=0, bias=True, add=False, accumulate=False, spread=0.5):
    """M rows of C entries in all; spread: how uneven the workers' numbers of rows are; add: a gradient comes past the block."""
    case = dict(name=name, kind=kind, n=n, M=M, C=C, dtype=dtype, offset=offset, bias=bias, spread=spread)
    return dict(case, add=add, accumulate=accumulate) if kind == "norm_grad" else case


def _affine(name, n, M, K, N, dtype="bf16", act="none", bias=True, pre=False, residual=False, wide=False, offset=0, spread=0.5):
    """K inputs and N outputs; wide: residual and result in fp32 from bf16 operands."""
    return dict(name=name, kind="affine", n=n, M=M, K=K, N=N, dtype=dtype, act=act, bias=bias, pre=pre, residual=residual, wide=wide,
                offset=offset, spread=spread)


def _affine_grad(name, n, M, K, N, dtype="bf16", act="none", below="gelu", accumulate=False, offset=0, spread=0.5):
    """act: of this layer; below: the one that its input came out of."""
    return dict(name=name, kind="affine_grad", n=n, M=M, K=K, N=N, dtype=dtype, act=act, below=below, accumulate=accumulate,
                offset=offset, spread=spread)


def _dropout(name, n, M, C, dtype="bf16", p=0.1, residual=True, spread=0.5):
    return dict(name=name, kind="dropout", n=n, M=M, C=C, dtype=dtype, p=p, residual=residual, spread=spread)


def _attention(name, sequences, M, heads, kv_heads, D, dtype="bf16", kind="attention", causal=True, spread=0.5):
    """M rows in all, in `sequences` sequences; kv_heads key and value heads of D entries, shared by the `heads` query heads."""
    return dict(name=name, kind=kind, sequences=sequences, M=M, heads=heads, kv_heads=kv_heads, D=D, dtype=dtype, causal=causal,
                spread=spread)


def listed():
    return [
        # every worker's model answers for one token: the smallest call, where latency counts
        _norm("norm_tokens", 8, 8, 1024, spread=0.0),
        # a batch of rows of the width of the largest listed layers
        _norm("norm_rows", 16, 16384, 4096),
        # the same on the way back, added to the gradient that comes past the block
        _norm("norm_grad_rows", 16, 16384, 4096, kind="norm_grad", add=True),
        # fp32 rows of a length that is no multiple of anything, few to a worker
        _norm("norm_grad_odd_f32", 32, 1999, 777, dtype="f32", kind="norm_grad", offset=5),
        # the narrowing layer for one token of every worker, into the residual
        _affine("affine_tokens", 8, 8, 1024, 1024, residual=True, spread=0.0),
        # the widening layer of a block in training: activation and what its gradient needs
        _affine("affine_mlp", 16, 8192, 1024, 4096, act="gelu", pre=True),
        # the way back through the narrowing layer: its bias, and its input through the activation
        _affine_grad("affine_grad_mlp", 16, 8192, 4096, 1024),
        # dropout of a branch of a block, added to the residual
        _dropout("dropout_residual", 16, 16384, 4096),
        # fp32, no residual, rows of odd length
        _dropout("dropout_odd_f32", 32, 1999, 777, dtype="f32", p=0.25, residual=False),
        # short fp32 sequences that see all of themselves, heads of no power of two
        _attention("attention_odd_f32", 9, 1500, 6, 2, 40, dtype="f32", causal=False),
        # the gradient of a batch of uneven packed sequences, four query heads to a key head
        _attention("attention_grad_packed", 24, 8192, 16, 4, 128, kind="attention_grad"),
        # two long prompts
        _attention("attention_long", 2, 16384, 32, 8, 128, spread=0.0),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(("norm", "norm_grad", "norm_grad", "affine", "affine", "affine_grad", "dropout", "attention", "attention",
                       "attention_grad", "attention_grad"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    spread = rng.choice((0.0, 0.5, 1.0))
    offset = rng.choice((0, 0, 8 * rng.randrange(1, 100), rng.randrange(1, 100)))
    if kind in ("norm", "norm_grad", "dropout"):
        while True:
            n, C, M = _log(rng, 1, 64), _log(rng, 8, 16384), _log(rng, 1, 16384)
            if rng.random() < 0.6:
                C = -(-C // 8) * 8
            if M * C <= 16384 * 4096 and n <= max(M, 4):
                break
        if kind == "dropout":
            c = _dropout("", n, M, C, dtype, rng.choice((0.0, 0.1, 0.25, 0.5, 0.9)), rng.random() < 0.5, spread)
        else:
            c = _norm("", n, M, C, dtype, kind, offset, rng.random() < 0.8, rng.random() < 0.5, rng.random() < 0.3, spread)
    elif kind in ("affine", "affine_grad"):
        most = 4.0e10 if dtype == "f32" else 2.0e11
        while True:
            n, K, N = _log(rng, 1, 64), _log(rng, 32, 4096), _log(rng, 32, 8192)
            M = _log(rng, n, 16384)
            if rng.random() < 0.6:
                K, N = -(-K // 8) * 8, -(-N // 8) * 8
            if n * K * N <= 3e8 and 2.0 * M * K * N <= most:
                break
        act = rng.choice(("none", "relu", "gelu", "silu"))
        if kind == "affine":
            c = _affine("", n, M, K, N, dtype, act, rng.random() < 0.8, rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.3, offset, spread)
        else:
            c = _affine_grad("", n, M, K, N, dtype, act, rng.choice(("none", "relu", "gelu", "silu")), rng.random() < 0.3, offset, spread)
    else:
        most = 4.0e10 if dtype == "f32" else 2.5e11
        while True:
            sequences, M = _log(rng, 1, 64), _log(rng, 1, 16384)
            kv_heads = rng.choice((1, 2, 4, 8))
            heads = kv_heads * rng.choice((1, 1, 2, 4, 8))
            D = rng.choice((64, 64, 128, 128, rng.randrange(8, 129)))
            c = _attention("", sequences, M, heads, kv_heads, D, dtype, kind, rng.random() < 0.75, spread)
            if heads * D <= 4096 and work(c)["flops"] <= most and heads * float(M) * M / sequences <= 4e9:
                break
    del c["name"]
    return c


# ---------------------------------------------------------------- inputs


def _offsets(parts, M, spread, seed):
    """parts + 1 offsets of M rows in all; spread 0: even; larger: uneven, and from 0.5 on some parts have none."""
    r = random.Random(seed * 7919 + parts)
    share = [math.exp(3 * spread * r.uniform(-1, 1)) for _ in range(parts)]
    if spread >= 0.5 and parts >= 4:
        share[r.randrange(parts)] = 0.0
    total, acc, offs = sum(share), 0.0, [0]
    for s in share:
        acc += s
        offs.append(min(M, int(round(M * acc / total))))
    offs[parts] = M
    return offs


def _pitch(d):
    return -(-d // 64) * 64


def _randn(g, *shape, scale=1.0):
    return torch.randn(*shape, generator=g, device=DEV).mul_(scale)


def _columns(case):
    """First columns of a layer's weights or gain and of its bias, and how many columns a worker's row has."""
    offset = case["offset"]
    bias = offset + (case["N"] * case["K"] if "K" in case else case["C"])
    return offset, bias, bias + (case["N"] if "K" in case else case["C"])


def _out_type(case):
    return torch.float32 if case.get("wide") else DTYPES[case["dtype"]]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    kind, M, dt = case["kind"], case["M"], DTYPES[case["dtype"]]
    s = dict(case=case, kind=kind)
    parts = case["sequences"] if "sequences" in case else case["n"]
    s["offs"] = offs = _offsets(parts, M, case["spread"], seed)  # a program knows its batch sizes
    s["rows"] = torch.tensor(offs, dtype=torch.int32, device=DEV)
    d = 1
    if kind in ("norm", "norm_grad"):
        C = case["C"]
        gain, bias, d = _columns(case)
        P = _randn(g, case["n"], _pitch(d), scale=0.1)
        P[:, gain:gain + C] += 1.0
        # rows have levels of their own, and a few columns are larger than the others, as in a trained network
        X = _randn(g, M, C) * torch.exp(_randn(g, C, scale=0.5)) + _randn(g, M, 1)
        s.update(P=P.to(dt), X=X.to(dt))
        if kind == "norm":
            s["Y"] = torch.zeros(M, C, dtype=dt, device=DEV)
        else:
            s["dY"] = _randn(g, M, C, scale=1e-2).to(dt)
            s["add"] = _randn(g, M, C, scale=1e-2).to(dt) if case["add"] else None
            s["dX"] = torch.zeros(M, C, dtype=dt, device=DEV)
            s["G"] = _randn(g, case["n"], _pitch(d), scale=1e-2)
    elif kind in ("affine", "affine_grad"):
        K, N = case["K"], case["N"]
        at, bias, d = _columns(case)
        W = torch.empty(case["n"], _pitch(d), dtype=dt, device=DEV)
        for i in range(case["n"]):
            W[i] = _randn(g, _pitch(d), scale=K ** -0.5)
        W[:, bias:bias + N] = _randn(g, case["n"], N, scale=0.2).to(dt)
        s["W"] = W
        if kind == "affine":
            s["A"] = _randn(g, M, K).to(dt)
            s["R"] = _randn(g, M, N).to(_out_type(case)) if case["residual"] else None
            s["Z"] = torch.zeros(M, N, dtype=dt, device=DEV) if case["pre"] else None
            s["Y"] = torch.zeros(M, N, dtype=_out_type(case), device=DEV)
        else:
            s["dY"] = _randn(g, M, N, scale=1e-2).to(dt)
            s["Z"] = _randn(g, M, N).to(dt) if case["act"] != "none" else None
            s["dZ"] = torch.zeros(M, N, dtype=dt, device=DEV) if case["act"] != "none" else None
            s["below"] = _randn(g, M, K).to(dt) if case["below"] != "none" else None
            s["dA"] = torch.zeros(M, K, dtype=dt, device=DEV)
            s["G"] = _randn(g, case["n"], _pitch(d), scale=1e-2)
    elif kind == "dropout":
        s["X"] = _randn(g, M, case["C"]).to(dt)
        s["R"] = _randn(g, M, case["C"]).to(dt) if case["residual"] else None
        s["Y"] = torch.zeros(M, case["C"], dtype=dt, device=DEV)
        s["seed"] = int(seed) * 0x9E3779B9 & 0xFFFFFFFFFFFF
    else:
        H, KV, D = case["heads"], case["kv_heads"], case["D"]
        # queries, keys and values are columns of one matrix, as the layer before puts them there; some heads look sharply
        qkv = torch.empty(M, (H + 2 * KV) * D, dtype=dt, device=DEV)
        sharp = torch.exp(_randn(g, H, 1, scale=0.5)).expand(H, D).reshape(-1)
        qkv[:, :H * D] = (_randn(g, M, H * D) * sharp).to(dt)
        qkv[:, H * D:] = _randn(g, M, 2 * KV * D).to(dt)
        s.update(qkv=qkv, Q=qkv[:, :H * D], K=qkv[:, H * D:(H + KV) * D], V=qkv[:, (H + KV) * D:])
        s["O"] = torch.zeros(M, H * D, dtype=dt, device=DEV)
        s["lse"] = torch.zeros(H, M, device=DEV)
        if kind == "attention_grad":
            _plain_attention(s)  # what the forward pass left
            s["dO"] = _randn(g, M, H * D, scale=1e-2).to(dt)
            s["dqkv"] = torch.zeros_like(qkv)
    if own:
        import paper_2006_08085_amd as D
        n = case.get("n", 1)
        s["ctx"] = ctx = D.detag_create(D.Topology.ring(), n, d, _pitch(d), D.DETAG_F32)
        if kind == "norm_grad":
            ctx.reserve_layer_gradient(M, case["C"])
        elif kind == "affine_grad":
            ctx.reserve_layer_gradient(M, case["N"])
        elif kind == "attention_grad":
            ctx.reserve_attention(M, case["heads"])
    return s


# ---------------------------------------------------------------- plain forms


def _worker(s):
    r = torch.arange(s["case"]["M"], device=DEV)
    return (r[:, None] >= s["rows"][None, 1:]).sum(1)


def _per_worker(t, s):
    """M x F rows as an (n, most, F) block of floats, zeros past a worker's rows; with the place of every row in it."""
    rows, M = s["rows"].long(), t.shape[0]
    most = max(b - a for a, b in zip(s["offs"], s["offs"][1:]))
    pos = rows[:-1, None] + torch.arange(most, device=DEV)
    inside = pos < rows[1:, None]
    block = torch.where(inside[..., None], t.float()[pos.clamp(max=M - 1)], 0.0)
    worker = _worker(s)
    return block, worker, torch.arange(M, device=DEV) - rows[worker]


def _worker_sums(t, s):
    """Sums of M x F rows over every worker's."""
    out = torch.zeros(s["case"]["n"], t.shape[1], device=DEV)
    for i, (lo, hi) in enumerate(zip(s["offs"], s["offs"][1:])):
        out[i] = t[lo:hi].sum(0)
    return out


def _normalised(s):
    x = s["X"].float()
    x = x - x.mean(1, keepdim=True)
    inverse = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + EPS)
    return x * inverse, inverse


def _plain_norm(s):
    c = s["case"]
    gain, bias, _ = _columns(c)
    P, worker = s["P"].float(), _worker(s)
    y = _normalised(s)[0] * P[:, gain:gain + c["C"]][worker]
    if c["bias"]:
        y = y + P[:, bias:bias + c["C"]][worker]
    s["Y"].copy_(y)
    return s["Y"]


def _put(s, at, value):
    here = s["G"][:, at:at + value.shape[1]]
    here.copy_(here + value if s["case"]["accumulate"] else value)
    return here


def _plain_norm_grad(s):
    c = s["case"]
    gain, bias, _ = _columns(c)
    dy = s["dY"].float()
    xhat, inverse = _normalised(s)
    out = {"gain": _put(s, gain, _worker_sums(dy * xhat, s))}
    if c["bias"]:
        out["bias"] = _put(s, bias, _worker_sums(dy, s))
    dx = dy * s["P"].float()[:, gain:gain + c["C"]][_worker(s)]
    dx = (dx - dx.mean(1, keepdim=True) - xhat * (dx * xhat).mean(1, keepdim=True)) * inverse
    s["dX"].copy_(dx if s["add"] is None else dx + s["add"].float())
    return dict(out, dX=s["dX"])


def _act(z, name):
    if name == "relu":
        return torch.where(z <= 0, 0.0, z)
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * 0.5 ** 0.5))
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _slope(z, name):
    if name == "relu":
        return (z > 0).float()
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2.0 * math.pi) ** -0.5
    p = 1.0 / (1.0 + torch.exp(-z))
    return p * (1.0 + z * (1.0 - p))


def _weights(s):
    c = s["case"]
    return s["W"][:, c["offset"]:c["offset"] + c["N"] * c["K"]].float().view(c["n"], c["N"], c["K"])


def _plain_affine(s):
    c = s["case"]
    bias = _columns(c)[1]
    a, worker, place = _per_worker(s["A"], s)
    z = torch.bmm(a, _weights(s).transpose(1, 2))[worker, place]
    if c["bias"]:
        z = z + s["W"][:, bias:bias + c["N"]].float()[worker]
    y = _act(z, c["act"])
    s["Y"].copy_(y if s["R"] is None else y + s["R"].float())
    if c["pre"]:
        s["Z"].copy_(z)
        return {"Y": s["Y"], "Z": s["Z"]}
    return s["Y"]


def _plain_affine_grad(s):
    c = s["case"]
    dz = s["dY"].float()
    out = {}
    if c["act"] != "none":
        dz = dz * _slope(s["Z"].float(), c["act"])
        out["bias"] = _put(s, _columns(c)[1], _worker_sums(dz, s))
        s["dZ"].copy_(dz)
        out["dZ"] = s["dZ"]
        dz = s["dZ"]
    else:
        out["bias"] = _put(s, _columns(c)[1], _worker_sums(dz, s))
    block, worker, place = _per_worker(dz, s)
    da = torch.bmm(block, _weights(s))[worker, place]
    s["dA"].copy_(da if c["below"] == "none" else da * _slope(s["below"].float(), c["below"]))
    return dict(out, dA=s["dA"])


def _philox(c0, c1, c2, c3, seed):
    """Four 32-bit words for every counter (Philox-4x32-10; Salmon et al., SC'11)."""
    mask = 0xFFFFFFFF
    k0, k1 = seed & mask, seed >> 32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & mask) ^ c1 ^ k0, p1 & mask, ((p0 >> 32) & mask) ^ c3 ^ k1, p0 & mask
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    return torch.stack(torch.broadcast_tensors(c0, c1, c2, c3), dim=2)


def _plain_dropout(s):
    c = s["case"]
    M, C = c["M"], c["C"]
    worker = _worker(s)
    place = torch.arange(M, device=DEV) - s["rows"].long()[worker]
    words = _philox(torch.arange(-(-C // 8), device=DEV)[None, :], (place + 2 ** 31)[:, None], worker[:, None],
                    torch.full((1, 1), STEP, dtype=torch.int64, device=DEV), s["seed"])
    halves = torch.stack((words & 0xFFFF, words >> 16), dim=3).flatten(1)[:, :C]
    border = int(math.floor(c["p"] * 65536 + 0.5))
    y = torch.where(halves >= border, s["X"].float() * (65536.0 / (65536 - border)), 0.0)
    s["Y"].copy_(y if s["R"] is None else y + s["R"].float())
    return s["Y"]


def _heads(t, lo, hi, heads, D, dtype=torch.float32):
    return t[lo:hi].to(dtype).reshape(hi - lo, heads, D).transpose(0, 1).contiguous()


def _spans(s):
    return [(lo, hi) for lo, hi in zip(s["offs"], s["offs"][1:]) if hi > lo]


def _scores(s, lo, hi):
    """Probabilities of a sequence and the logarithms of their sums, and what they were made of; key heads repeated for their query heads."""
    c = s["case"]
    H, KV, D, L = c["heads"], c["kv_heads"], c["D"], hi - lo
    q = _heads(s["Q"], lo, hi, H, D)
    k, v = (_heads(s[x], lo, hi, KV, D).repeat_interleave(H // KV, 0) for x in ("K", "V"))
    z = torch.bmm(q, k.transpose(1, 2)) * D ** -0.5
    if c["causal"]:
        r = torch.arange(L, device=DEV)
        z.masked_fill_(r[None, :] > r[:, None], -math.inf)
    top = z.max(2, keepdim=True).values
    z = z.sub_(top).exp_()
    total = z.sum(2, keepdim=True)
    return z.div_(total), (top + torch.log(total))[..., 0], q, k, v


def _plain_attention(s):
    for lo, hi in _spans(s):
        p, lse, _, _, v = _scores(s, lo, hi)
        s["O"][lo:hi] = torch.bmm(p, v).transpose(0, 1).reshape(hi - lo, -1)
        s["lse"][:, lo:hi] = lse
    return {"O": s["O"], "lse": s["lse"]}


def _plain_attention_grad(s):
    c = s["case"]
    H, KV, D = c["heads"], c["kv_heads"], c["D"]
    for lo, hi in _spans(s):
        p, _, q, k, v = _scores(s, lo, hi)
        do, o = _heads(s["dO"], lo, hi, H, D), _heads(s["O"], lo, hi, H, D)
        dv = torch.bmm(p.transpose(1, 2), do)
        dz = torch.bmm(do, v.transpose(1, 2)).sub_((do * o).sum(2, keepdim=True)).mul_(p).mul_(D ** -0.5)
        dq, dk = torch.bmm(dz, k), torch.bmm(dz.transpose(1, 2), q)
        shared = [t.reshape(KV, H // KV, hi - lo, D).sum(1) for t in (dk, dv)]
        s["dqkv"][lo:hi] = torch.cat([t.transpose(0, 1).reshape(hi - lo, -1) for t in (dq, *shared)], dim=1)
    return s["dqkv"]


_PLAIN = {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "affine": _plain_affine, "affine_grad": _plain_affine_grad,
          "dropout": _plain_dropout, "attention": _plain_attention, "attention_grad": _plain_attention_grad}


# ---------------------------------------------------------------- the library's calls


def _own(s):
    import paper_2006_08085_amd as D
    c, ctx, kind, rows = s["case"], s["ctx"], s["kind"], s["rows"]
    acts = {"none": D.DETAG_ACT_NONE, "relu": D.DETAG_ACT_RELU, "gelu": D.DETAG_ACT_GELU, "silu": D.DETAG_ACT_SILU}
    if kind in ("norm", "norm_grad"):
        gain, bias, _ = _columns(c)
        at = bias if c["bias"] else None
        if kind == "norm":
            ctx.layer_norm(s["P"], gain, at, s["X"], rows, s["Y"], eps=EPS)
            return s["Y"]
        ctx.layer_norm_grad(s["P"], gain, at, s["X"], s["dY"], rows, s["dX"], s["G"], eps=EPS, add=s["add"], accumulate=c["accumulate"])
        out = {"gain": s["G"][:, gain:gain + c["C"]], "dX": s["dX"]}
        return dict(out, bias=s["G"][:, bias:bias + c["C"]]) if c["bias"] else out
    if kind == "affine":
        ctx.linear_act(s["W"], c["offset"], s["A"], rows, s["Y"], bias=_columns(c)[1] if c["bias"] else None, act=acts[c["act"]],
                       pre=s["Z"], residual=s["R"])
        return {"Y": s["Y"], "Z": s["Z"]} if c["pre"] else s["Y"]
    if kind == "affine_grad":
        bias = _columns(c)[1]
        ctx.linear_grad_bias(s["dY"], rows, s["G"], bias, act=acts[c["act"]], pre=s["Z"], dZ=s["dZ"], accumulate=c["accumulate"])
        out = {"bias": s["G"][:, bias:bias + c["N"]]}
        if c["act"] != "none":
            out["dZ"] = s["dZ"]
        ctx.linear_grad_input_act(s["W"], c["offset"], s["dY"] if c["act"] == "none" else s["dZ"], rows, s["dA"], act=acts[c["below"]],
                                  pre=s["below"])
        return dict(out, dA=s["dA"])
    if kind == "dropout":
        ctx.dropout(s["X"], rows, s["Y"], p=c["p"], seed=s["seed"], step=STEP, residual=s["R"])
        return s["Y"]
    H, KV, D = c["heads"], c["kv_heads"], c["D"]
    if kind == "attention":
        ctx.attention(s["Q"], s["K"], s["V"], rows, s["O"], H, KV, causal=c["causal"], lse=s["lse"])
        return {"O": s["O"], "lse": s["lse"]}
    d = s["dqkv"]
    ctx.attention_grad(s["Q"], s["K"], s["V"], rows, s["O"], s["lse"], s["dO"], d[:, :H * D], d[:, H * D:(H + KV) * D], d[:, (H + KV) * D:],
                       H, KV, causal=c["causal"])
    return d


def run(state):
    return _own(state) if own else _PLAIN[state["kind"]](state)


# ---------------------------------------------------------------- work and the definition in 64 bits


def work(case):
    kind, M = case["kind"], case["M"]
    e = 4 if case["dtype"] == "f32" else 2
    if kind in ("norm", "norm_grad"):
        C, n = case["C"], case["n"]
        vectors = 2 if case["bias"] else 1
        if kind == "norm":
            return {"bytes": 2 * e * M * C + vectors * e * n * C, "flops": 8.0 * M * C}
        rows = (4 if case["add"] else 3) * e * M * C
        return {"bytes": rows + e * n * C + vectors * (8 if case["accumulate"] else 4) * n * C, "flops": 16.0 * M * C}
    if kind in ("affine", "affine_grad"):
        K, N, n = case["K"], case["N"], case["n"]
        product = 2.0 * M * K * N
        if kind == "affine":
            y = 4 if case["wide"] else e
            vector = e * n * N if case["bias"] else 0
            return {"bytes": e * (n * K * N + M * K) + vector + M * N * (y * (2 if case["residual"] else 1) + (e if case["pre"] else 0)),
                    "flops": product}
        rows = M * N * (3 if case["act"] != "none" else 1) + M * K * (2 if case["below"] != "none" else 1)
        return {"bytes": e * (n * K * N + rows) + (8 if case["accumulate"] else 4) * n * N, "flops": product}
    if kind == "dropout":
        return {"bytes": (3 if case["residual"] else 2) * e * M * case["C"], "flops": 2.0 * M * case["C"]}
    H, KV, D = case["heads"], case["kv_heads"], case["D"]
    lengths = [b - a for a, b in zip(*(lambda o: (o, o[1:]))(_offsets(case["sequences"], M, case["spread"], 0)))]
    pairs = sum(x * (x + 1) / 2 if case["causal"] else x * x for x in lengths)
    rows = e * M * D * (H + 2 * KV)
    if kind == "attention":
        return {"bytes": rows + e * M * D * H + 4 * M * H, "flops": 4.0 * pairs * H * D}
    # queries, keys, values, results and their gradients in, three gradients out
    return {"bytes": 2 * rows + 2 * e * M * D * H + 4 * M * H, "flops": 10.0 * pairs * H * D}


def exact(case, seed):
    s = prepare(case, seed)
    return _EXACT[case["kind"]](case, s)


def _exact_norm(c, s):
    gain, bias, _ = _columns(c)
    y = torch.nn.functional.layer_norm(s["X"].double(), (c["C"],), eps=EPS)
    for i, (lo, hi) in enumerate(zip(s["offs"], s["offs"][1:])):
        y[lo:hi] *= s["P"][i, gain:gain + c["C"]].double()
        if c["bias"]:
            y[lo:hi] += s["P"][i, bias:bias + c["C"]].double()
    return y


def _exact_norm_grad(c, s):
    C = c["C"]
    gain, bias, _ = _columns(c)
    dX = torch.zeros(c["M"], C, dtype=torch.float64, device=DEV)
    G = s["G"].double() * (1.0 if c["accumulate"] else 0.0)
    for i, (lo, hi) in enumerate(zip(s["offs"], s["offs"][1:])):
        x, dy = s["X"][lo:hi].double(), s["dY"][lo:hi].double()
        sigma = torch.sqrt(x.var(1, unbiased=False, keepdim=True) + EPS)
        xhat = (x - x.mean(1, keepdim=True)) / sigma
        G[i, gain:gain + C] += (dy * xhat).sum(0)
        if c["bias"]:
            G[i, bias:bias + C] += dy.sum(0)
        h = dy * s["P"][i, gain:gain + C].double()
        dX[lo:hi] = (h - h.mean(1, keepdim=True) - xhat * (h * xhat).mean(1, keepdim=True)) / sigma
    if s["add"] is not None:
        dX += s["add"].double()
    out = {"gain": G[:, gain:gain + C], "dX": dX}
    return dict(out, bias=G[:, bias:bias + C]) if c["bias"] else out


def _exact_act(z, name):
    return {"none": lambda: z, "relu": lambda: torch.relu(z), "gelu": lambda: z * torch.special.ndtr(z), "silu": lambda: z * torch.sigmoid(z)}[name]()


def _exact_slope(z, name):
    z = z.detach().requires_grad_(True)
    with torch.enable_grad():
        return torch.autograd.grad(_exact_act(z, name).sum(), z)[0]


def _exact_affine(c, s):
    K, N, at = c["K"], c["N"], c["offset"]
    Z = torch.zeros(c["M"], N, dtype=torch.float64, device=DEV)
    for i, (lo, hi) in enumerate(zip(s["offs"], s["offs"][1:])):
        Z[lo:hi] = s["A"][lo:hi].double() @ s["W"][i, at:at + N * K].double().reshape(N, K).t()
        if c["bias"]:
            Z[lo:hi] += s["W"][i, at + N * K:at + N * K + N].double()
    Y = _exact_act(Z, c["act"])
    if c["residual"]:
        Y = Y + s["R"].double()
    return {"Y": Y, "Z": Z} if c["pre"] else Y


def _exact_affine_grad(c, s):
    K, N, at = c["K"], c["N"], c["offset"]
    dZ = s["dY"].double()
    out = {}
    if c["act"] != "none":
        dZ = out["dZ"] = dZ * _exact_slope(s["Z"].double(), c["act"])
    dA = torch.zeros(c["M"], K, dtype=torch.float64, device=DEV)
    b = s["G"][:, at + N * K:at + N * K + N].double() * (1.0 if c["accumulate"] else 0.0)
    for i, (lo, hi) in enumerate(zip(s["offs"], s["offs"][1:])):
        b[i] += dZ[lo:hi].sum(0)
        dA[lo:hi] = dZ[lo:hi] @ s["W"][i, at:at + N * K].double().reshape(N, K)
    if c["below"] != "none":
        dA *= _exact_slope(s["below"].double(), c["below"])
    return dict(out, bias=b, dA=dA)


def _exact_words(counters, seed):
    """The generator's words from its definition, products taken in 16-bit halves."""
    def product(a, b):  # a constant and a tensor of 32-bit numbers: (upper, lower) 32 bits
        al, ah, bl, bh = a & 0xFFFF, a >> 16, b & 0xFFFF, b >> 16
        mid = al * bh + ((al * bl) >> 16)
        mid2 = ah * bl + (mid & 0xFFFF)
        return ah * bh + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xFFFF) << 16) | ((al * bl) & 0xFFFF)
    x, key = list(counters), [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        (h0, l0), (h1, l1) = product(0xD2511F53, x[0]), product(0xCD9E8D57, x[2])
        x = [h1 ^ x[1] ^ key[0], l1, h0 ^ x[3] ^ key[1], l0]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    return x


def _exact_dropout(c, s):
    Y = s["R"].double() if c["residual"] else torch.zeros(c["M"], c["C"], dtype=torch.float64, device=DEV)
    border = int(math.floor(c["p"] * 65536 + 0.5))
    col = torch.arange(c["C"], device=DEV)
    for i, (lo, hi) in enumerate(zip(s["offs"], s["offs"][1:])):
        zero = torch.zeros(hi - lo, -(-c["C"] // 8), dtype=torch.int64, device=DEV)
        words = _exact_words([zero + torch.arange(zero.shape[1], device=DEV), zero + torch.arange(hi - lo, device=DEV)[:, None] + 2 ** 31,
                              zero + i, zero + STEP], s["seed"])
        word = torch.stack(words, dim=2).flatten(1)[:, col // 2]
        half = torch.where(col % 2 == 0, word % 65536, word // 65536)
        Y[lo:hi] += s["X"][lo:hi].double() * (half >= border) * 65536.0 / (65536 - border)
    return Y


def _exact_softmax(c, s, lo, hi, h):
    """One head of one sequence: probabilities, logarithms of the sums, queries, keys, values."""
    D, kv = c["D"], h // (c["heads"] // c["kv_heads"])
    q = s["Q"][lo:hi, h * D:(h + 1) * D].double()
    k, v = (s[x][lo:hi, kv * D:(kv + 1) * D].double() for x in ("K", "V"))
    z = q @ k.t() / math.sqrt(D)
    if c["causal"]:
        z += torch.full_like(z, -math.inf).triu_(1)
    lse = torch.logsumexp(z, 1)
    return torch.exp(z - lse[:, None]), lse, q, k, v


def _exact_attention(c, s):
    D = c["D"]
    O = torch.zeros(c["M"], c["heads"] * D, dtype=torch.float64, device=DEV)
    lse = torch.zeros(c["heads"], c["M"], dtype=torch.float64, device=DEV)
    for lo, hi in _spans(s):
        for h in range(c["heads"]):
            p, lse[h, lo:hi], _, _, v = _exact_softmax(c, s, lo, hi, h)
            O[lo:hi, h * D:(h + 1) * D] = p @ v
    return {"O": O, "lse": lse}


def _exact_attention_grad(c, s):
    H, KV, D = c["heads"], c["kv_heads"], c["D"]
    dq = torch.zeros(c["M"], H, D, dtype=torch.float64, device=DEV)
    dk, dv = (torch.zeros(c["M"], KV, D, dtype=torch.float64, device=DEV) for _ in range(2))
    for lo, hi in _spans(s):
        for h in range(H):
            p, _, q, k, v = _exact_softmax(c, s, lo, hi, h)
            kv = h // (H // KV)
            do = s["dO"][lo:hi, h * D:(h + 1) * D].double()
            dp = do @ v.t()
            dz = p * (dp - (p * dp).sum(1, keepdim=True)) / math.sqrt(D)
            dq[lo:hi, h] = dz @ k
            dk[lo:hi, kv] += dz.t() @ q
            dv[lo:hi, kv] += p.t() @ do
    return torch.cat([t.reshape(c["M"], -1) for t in (dq, dk, dv)], dim=1)


_EXACT = {"norm": _exact_norm, "norm_grad": _exact_norm_grad, "affine": _exact_affine, "affine_grad": _exact_affine_grad,
          "dropout": _exact_dropout, "attention": _exact_attention, "attention_grad": _exact_attention_grad}

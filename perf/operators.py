"""The operators of a local training step, as measurable cases.

n simulated workers learn a network of layers: every worker has its own
weights (a slice of its row of the n x ld model matrix) and its own number of
samples.  The cases are passes of

  linear   a layer's product for all workers, each on its own rows: Y = act(A W_i^T)
  lgrad    the two products of its gradient: dA = (dY W_i) [H > 0] and G_i (+)= dY^T A
  xent     softmax cross-entropy of every worker's rows (mean over its own), with the gradient of the logits
  adamw    one AdamW step over all tensors of all workers, moments in 32 bits or in 8 bits with block scales

run() computes them in elementary torch operations where `own` is false, and
through the library's entry points where it is true; exact() restates them in
64 bits.
"""
import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BETA1, BETA2, EPS, LR, STEP = 0.9, 0.999, 1e-8, 1e-3, 1000
BLOCK = 256  # columns of a tensor that share a scale of the 8-bit moments


def _linear(name, n, M, K, N, dtype="bf16", kind="linear", relu=False, offset=0, wide=False, accumulate=False, spread=0.5):
    """M rows in all, K inputs and N outputs of the layer; wide: fp32 output of bf16 operands; spread: how uneven the workers'
    numbers of rows are."""
    case = dict(name=name, kind=kind, n=n, M=M, K=K, N=N, dtype=dtype, relu=relu, offset=offset, spread=spread)
    return dict(case, wide=wide) if kind == "linear" else dict(case, accumulate=accumulate)


def _xent(name, n, M, C, dtype="f32", ignored=0.0, spread=0.5):
    return dict(name=name, kind="xent", n=n, M=M, C=C, dtype=dtype, ignored=ignored, spread=spread)


def _adamw(name, n, d, tensors, bits, dtype="f32", copy=False, odd=False):
    """copy: also writes the new models in bfloat16; odd: tensors of any length, not of multiples of 8."""
    return dict(name=name, kind="adamw", n=n, d=d, tensors=tensors, bits=bits, dtype=dtype, copy=copy, odd=odd)


def listed():
    return [
        # every worker's model answers for one sample: what a run's log asks for; the weights are all there is to read
        _linear("linear_tokens", 8, 8, 1024, 1024, spread=0.0),
        # the widening layer of a network, batches of uneven sizes (label-sorted shards), its activation in the same pass
        _linear("linear_mlp", 16, 8192, 1024, 4096, relu=True),
        # fp32 models of sizes that are no multiple of anything, as a user's own features give
        _linear("linear_odd_f32", 32, 1999, 777, 1003, dtype="f32", offset=5),
        # the largest: few workers with large models, a vocabulary-sized output in fp32 from bf16 operands
        _linear("linear_large", 8, 16384, 4096, 8192, wide=True, spread=0.25),
        # the gradient of the widening layer
        _linear("lgrad_mlp", 16, 8192, 1024, 4096, kind="lgrad", relu=True),
        # the largest gradient: few workers, square layers of 4096
        _linear("lgrad_large", 8, 16384, 4096, 4096, kind="lgrad", spread=0.25),
        # 32 workers, 128 samples each, 10 classes: the softmax workload's logits
        _xent("xent_ring32", 32, 4096, 10, spread=0.0),
        # a vocabulary in bf16; one row in ten carries no label
        _xent("xent_vocab_bf16", 8, 8192, 32000, dtype="bf16", ignored=0.1),
        # an odd vocabulary in fp32, rows that start at no multiple of 16 bytes
        _xent("xent_odd_f32", 5, 1500, 50001),
        # ResNet-20-sized models of 16 workers, moments in 8 bits
        _adamw("adamw8_ring16", 16, 272_474, 20, 8),
        # ResNet-18-sized models of 64 workers, the headline workload's state
        _adamw("adamw_torus64", 64, 11_173_962, 62, 32),
        # 256 workers, fp32 models with the bf16 copy that the next products read, moments in 8 bits
        _adamw("adamw8_regular256", 256, 1_048_576, 40, 8, copy=True),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(("linear", "linear", "lgrad", "lgrad", "xent", "xent", "adamw", "adamw"))
    if kind in ("linear", "lgrad"):
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        most = 2.0e11 if dtype == "f32" else 1.0e12
        while True:
            n, K, N = _log(rng, 1, 64), _log(rng, 32, 4096), _log(rng, 32, 8192)
            M = _log(rng, n, 16384)
            if rng.random() < 0.6:
                K, N = -(-K // 8) * 8, -(-N // 8) * 8
            if 3072 in (K, N, M) or n * K * N > 3e8 or 2.0 * M * K * N * (2 if kind == "lgrad" else 1) > most:
                continue
            break
        offset = rng.choice((0, 0, 8 * rng.randrange(1, 100), rng.randrange(1, 100)))
        common = dict(dtype=dtype, kind=kind, relu=rng.random() < 0.5, offset=offset, spread=rng.choice((0.0, 0.5, 1.0)))
        c = _linear("", n, M, K, N, wide=rng.random() < 0.3, accumulate=rng.random() < 0.3, **common)
    elif kind == "xent":
        while True:
            n, C, M = _log(rng, 1, 64), _log(rng, 2, 131072), _log(rng, 16, 16384)
            if M * C <= 8192 * 32000 and M >= n and 3072 not in (M, C):
                break
        c = _xent("", n, M, C, rng.choice(("f32", "bf16")), rng.choice((0.0, 0.1, 0.9)), rng.choice((0.0, 0.5, 1.0)))
    else:
        bits = rng.choice((8, 8, 32))
        while True:
            n, d = _log(rng, 2, 256), _log(rng, 1000, 11_173_962)
            if n * d <= (2.6e8 if bits == 8 else 7e8):
                break
        dtype = rng.choice(("f32", "f32", "bf16"))
        c = _adamw("", n, d, rng.randrange(1, 80), bits, dtype, dtype == "f32" and rng.random() < 0.5, rng.random() < 0.5)
    del c["name"]
    return c


# ---------------------------------------------------------------- inputs


def _row_offsets(n, M, spread, seed):
    """n+1 offsets of M rows in all; spread 0: even; larger: uneven, and from 0.5 on some workers have none."""
    r = random.Random(seed * 7919 + n)
    share = [math.exp(3 * spread * r.uniform(-1, 1)) for _ in range(n)]
    if spread >= 0.5 and n >= 4:
        share[r.randrange(n)] = 0.0
    total, acc, offs = sum(share), 0.0, [0]
    for s in share:
        acc += s
        offs.append(min(M, int(round(M * acc / total))))
    offs[n] = M
    return offs


def _tensors(case):
    """(offset, length) of the tensors of a row: weights of all sizes and short vectors, one after the other."""
    d, count = case["d"], min(case["tensors"], max(1, case["d"] // 16))
    r = random.Random(d * 131 + count)
    step = 1 if case["odd"] else 8
    share = [math.exp(r.uniform(0, 6)) for _ in range(count)]
    lengths = [max(step, int(d * s / sum(share)) // step * step) for s in share]
    while sum(lengths[:-1]) >= d:  # many short tensors in a short row
        lengths[lengths.index(max(lengths))] //= 2
    lengths[-1] = d - sum(lengths[:-1])
    at, out = 0, []
    for length in lengths:
        if length > 0:
            out.append((at, length))
            at += length
    return out


def _pitch(d):
    return -(-d // 64) * 64


def _randn(g, *shape, scale=1.0):
    return torch.randn(*shape, generator=g, device=DEV).mul_(scale)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    kind, n = case["kind"], case["n"]
    s = dict(case=case, kind=kind)
    if kind != "adamw":
        offs = _row_offsets(n, case["M"], case["spread"], seed)
        s["rows"] = torch.tensor(offs, dtype=torch.int32, device=DEV)
        s["most"] = max(b - a for a, b in zip(offs, offs[1:]))  # a program knows its batch sizes
    dt = DTYPES[case["dtype"]]
    if kind in ("linear", "lgrad"):
        M, K, N, off = case["M"], case["K"], case["N"], case["offset"]
        d = off + N * K
        ld = _pitch(d)
        W = torch.empty(n, ld, dtype=dt, device=DEV)
        for i in range(n):
            W[i] = _randn(g, ld, scale=K ** -0.5)
        A = _randn(g, M, K)
        A = (A.clamp_(min=0) if kind == "lgrad" and case["relu"] else A).to(dt)  # a layer after an activation has half zeros
        s.update(W=W, A=A)
        if kind == "linear":
            s["Y"] = torch.zeros(M, N, dtype=torch.float32 if case["wide"] else dt, device=DEV)
        else:
            s["dY"] = _randn(g, M, N, scale=1e-2).to(dt)
            s["dA"] = torch.zeros(M, K, dtype=dt, device=DEV)
            s["G"] = torch.empty(n, ld, device=DEV)
            for i in range(n):
                s["G"][i] = _randn(g, ld, scale=1e-2)
    elif kind == "xent":
        M, C = case["M"], case["C"]
        d, ld = 1, 1
        s["logits"] = _randn(g, M, C, scale=3.0).to(dt)
        labels = torch.randint(C, (M,), generator=g, device=DEV, dtype=torch.int32)
        labels[torch.rand(M, generator=g, device=DEV) < case["ignored"]] = -1
        s.update(labels=labels, dlogits=torch.empty_like(s["logits"]), loss=torch.empty(n, device=DEV))
    else:
        d = case["d"]
        ld = _pitch(d)
        tensors = _tensors(case)
        s["tensors"] = tensors
        s["decay"] = [0.01 if length >= 4096 else 0.0 for _, length in tensors]  # weights decay, short vectors do not
        s["scale"] = [1.0 if k % 3 else 0.5 for k in range(len(tensors))]
        X = _randn(g, n, ld, scale=0.05).to(dt)
        width = torch.exp(_randn(g, ld))
        G = _randn(g, n, ld, scale=1e-3).mul_(width)
        G.mul_(torch.rand(ld, generator=g, device=DEV) > 0.05)  # some parameters were not touched
        M = _randn(g, n, ld, scale=3e-4).mul_(width)
        V = _randn(g, n, ld, scale=1e-3).mul_(width).square_()
        s.update(X=X, G=G, seed=int(seed) & 0xFFFFFFFF)
        if case["copy"]:
            s["X16"] = torch.empty(n, ld, dtype=torch.bfloat16, device=DEV)
        if case["bits"] == 32:
            s.update(M=M, V=V, S=None)
        else:
            idx, inside, _ = _blocks(s)
            half = torch.full((1,), 32768, dtype=torch.int32, device=DEV)
            s["M"] = torch.zeros(n, ld, dtype=torch.uint8, device=DEV)
            s["V"] = torch.zeros(n, ld, dtype=torch.uint8, device=DEV)
            m, em = _encode(torch.where(inside, M[:, idx], 0), half, 7)
            v, ev = _encode(torch.where(inside, V[:, idx], 0), half, 15)
            s["M"][:, idx[inside]], s["V"][:, idx[inside]] = m[:, inside], v[:, inside]
            s["S"] = torch.stack((em, ev), dim=2).reshape(n, -1).to(torch.uint8)
            # where the moments are read back to: what the codes stand for
            s["M_values"] = torch.zeros(n, ld, dtype=torch.bfloat16, device=DEV)
            s["V_values"] = torch.zeros(n, ld, dtype=torch.bfloat16, device=DEV)
        del M, V
    if own:
        import paper_2006_08085_amd as D
        state = D.DETAG_BF16 if kind == "adamw" and case["dtype"] == "bf16" else D.DETAG_F32
        s["ctx"] = ctx = D.detag_create(D.Topology.ring(), n, d, ld, state)
        if kind == "xent":
            ctx.reserve_cross_entropy(case["M"])
        elif kind == "adamw":
            s["optimizer"] = D.AdamW(ctx, s["tensors"], s["decay"], s["scale"], bits=case["bits"])
    return s


# ---------------------------------------------------------------- plain forms


def _per_worker(t, s):
    """M x F rows as an (n, most, F) block of floats, zeros past a worker's rows; with the place of every row in it."""
    rows, most, M = s["rows"].long(), s["most"], t.shape[0]
    pos = rows[:-1, None] + torch.arange(most, device=DEV)
    inside = pos < rows[1:, None]
    block = torch.where(inside[..., None], t.float()[pos.clamp(max=M - 1)], 0.0)
    r = torch.arange(M, device=DEV)
    worker = (r[:, None] >= rows[None, 1:]).sum(1)
    return block, worker, r - rows[worker]


def _weights(s):
    c = s["case"]
    return s["W"][:, c["offset"]:c["offset"] + c["N"] * c["K"]].float().view(c["n"], c["N"], c["K"])


def _plain_linear(s):
    a, worker, place = _per_worker(s["A"], s)
    y = torch.bmm(a, _weights(s).transpose(1, 2))[worker, place]
    s["Y"].copy_(torch.where(y <= 0, 0.0, y) if s["case"]["relu"] else y)
    return s["Y"]


def _plain_lgrad(s):
    c = s["case"]
    a, worker, place = _per_worker(s["A"], s)
    dy = _per_worker(s["dY"], s)[0]
    da = torch.bmm(dy, _weights(s))[worker, place]
    s["dA"].copy_(torch.where(s["A"].float() > 0, da, 0.0) if c["relu"] else da)
    dw = torch.bmm(dy.transpose(1, 2), a).view(c["n"], -1)
    G = s["G"][:, c["offset"]:c["offset"] + c["N"] * c["K"]]
    G.copy_(G + dw if c["accumulate"] else dw)
    return {"dA": s["dA"], "G": G}


def _plain_xent(s):
    z, labels, rows, C, n = s["logits"].float(), s["labels"].long(), s["rows"], s["case"]["C"], s["case"]["n"]
    r = torch.arange(z.shape[0], device=DEV)
    worker = (r[:, None] >= rows[None, 1:]).sum(1)
    valid = (labels >= 0) & (labels < C)
    count = torch.zeros(n, device=DEV).index_add_(0, worker, valid.float())
    top = z.max(1, keepdim=True).values
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    at = labels.clamp(0, C - 1)
    row_loss = torch.log(total[:, 0]) + top[:, 0] - z[r, at]
    s["loss"].copy_(torch.zeros(n, device=DEV).index_add_(0, worker, torch.where(valid, row_loss, 0.0)) / count.clamp(min=1))
    p = e / total
    p[r, at] -= 1.0
    p = torch.where(valid[:, None], p / count.clamp(min=1)[worker][:, None], 0.0)
    s["dlogits"].copy_(p)
    return {"loss": s["loss"], "dlogits": s["dlogits"]}


def _blocks(s):
    """Columns of the blocks of 256 that each tensor is cut into: (blocks, 256) indices, which of them are inside, tensor of a block."""
    offs = torch.tensor([o for o, _ in s["tensors"]], device=DEV)
    lens = torch.tensor([length for _, length in s["tensors"]], device=DEV)
    counts = (lens + BLOCK - 1) // BLOCK
    owner = torch.repeat_interleave(torch.arange(len(counts), device=DEV), counts)
    local = torch.arange(owner.numel(), device=DEV) - (counts.cumsum(0) - counts)[owner]
    col = local[:, None] * BLOCK + torch.arange(BLOCK, device=DEV)
    inside = col < lens[owner][:, None]
    return torch.where(inside, offs[owner][:, None] + col, 0), inside, owner


def _philox(blocks, n, step, seed):
    """Four 32-bit words for every (worker, block, lane) (Philox-4x32-10; Salmon et al., SC'11), as the 16-bit halves of the 256
    columns of a block."""
    mask = 0xFFFFFFFF
    lane = torch.arange(blocks * (BLOCK // 4), device=DEV)
    c0 = lane.expand(n, -1)
    c1 = torch.full((1, 1), 0x41646157, dtype=torch.int64, device=DEV)
    c2 = torch.arange(n, device=DEV)[:, None]
    c3 = torch.full((1, 1), step, dtype=torch.int64, device=DEV)
    k0, k1 = seed & mask, seed >> 32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & mask) ^ c1 ^ k0, p1 & mask, ((p0 >> 32) & mask) ^ c3 ^ k1, p0 & mask
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    words = torch.stack(torch.broadcast_tensors(c0, c1, c2, c3), dim=2).reshape(n, blocks, BLOCK).to(torch.int32)
    return words & 0xFFFF, (words >> 16) & 0xFFFF


def _power(biased):
    """2^(biased - 127) as floats, from a biased exponent in 1..254."""
    return (biased.to(torch.int32) << 23).view(torch.float32)


def _encode(x, r, bias):
    """8-bit codes of the values of blocks (last axis) and their biased exponents.  bias 7: sign, 4 exponent bits and 3 of the
    mantissa; bias 15: no sign, 5 and 3.  r: 16 random bits a value, added below the last bit kept."""
    bits = x.view(torch.int32) & 0x7FFFFFFF
    finite = bits < 0x7F800000
    E = (torch.where(finite, bits, 0).amax(-1) >> 23).clamp(min=16)
    top = 134 if bias == 7 else 142  # the largest magnitude lands one exponent below the last
    y = bits.view(torch.float32) * _power(top + 127 - E)[..., None]
    normal = ((y.view(torch.int32) + r * 16) >> 20) - 8 * (127 - bias)
    below = (y * (2.0 ** (bias + 2)) + r.float() * 2.0 ** -16).clamp(max=8).to(torch.int32)
    code = torch.where(y < 2.0 ** (1 - bias), below, normal)
    code = torch.where(finite, code, 127 if bias == 7 else 255)
    if bias == 7:
        code = code | torch.where(x.view(torch.int32) < 0, 128, 0)
    return code.to(torch.uint8), E


def _decode(code, E, bias):
    c = code.to(torch.int32)
    mag = c & 127 if bias == 7 else c
    unit = torch.where(mag < 8, mag.float() * 2.0 ** (-bias - 2), ((mag << 20) + ((127 - bias) << 23)).view(torch.float32))
    unit = torch.where(mag == (127 if bias == 7 else 255), math.nan, unit)
    y = unit * _power(E - (7 if bias == 7 else 15))[..., None]
    return torch.where(c >= 128, -y, y) if bias == 7 else y


def _moments(m, v, g):
    return m * BETA1 + g * (1.0 - BETA1), v * BETA2 + (g * g) * (1.0 - BETA2)


def _update(x, m, v, decay, scale):
    lr = LR * scale
    step = (m / (1.0 - BETA1 ** STEP)) / (torch.sqrt(v / (1.0 - BETA2 ** STEP)) + EPS)
    return x * (1.0 - lr * decay) - lr * step


def _plain_adamw(s):
    c = s["case"]
    n, d, X, G = c["n"], c["d"], s["X"], s["G"]
    decay, scale = torch.tensor(s["decay"], device=DEV), torch.tensor(s["scale"], device=DEV)
    if c["bits"] == 32:
        lens = torch.tensor([length for _, length in s["tensors"]], device=DEV)
        m, v = _moments(s["M"][:, :d], s["V"][:, :d], G[:, :d])
        x = _update(X[:, :d].float(), m, v, torch.repeat_interleave(decay, lens), torch.repeat_interleave(scale, lens))
        X[:, :d], s["M"][:, :d], s["V"][:, :d] = x, m, v
        out = {"X": X[:, :d], "M": s["M"][:, :d], "V": s["V"][:, :d]}
    else:
        idx, inside, owner = _blocks(s)
        S = s["S"].view(n, -1, 2).to(torch.int32)
        m, v = _decode(s["M"][:, idx], S[..., 0], 7), _decode(s["V"][:, idx], S[..., 1], 15)
        g = torch.where(inside, G[:, idx], 0.0)
        m, v = _moments(torch.where(inside, m, 0.0), torch.where(inside, v, 0.0), g)
        x = _update(X[:, idx].float(), m, v, decay[owner][:, None], scale[owner][:, None])
        rm, rv = _philox(idx.shape[0], n, STEP, s["seed"])
        cm, em = _encode(m, rm, 7)
        cv, ev = _encode(v, rv, 15)
        del m, v, rm, rv
        s["S"].copy_(torch.stack((em, ev), dim=2).reshape(n, -1))
        cols = idx[inside]
        X[:, cols] = x[:, inside].to(X.dtype)
        s["M"][:, cols], s["V"][:, cols] = cm[:, inside], cv[:, inside]
        s["M_values"][:, cols] = _decode(cm, em, 7)[:, inside].to(torch.bfloat16)
        s["V_values"][:, cols] = _decode(cv, ev, 15)[:, inside].to(torch.bfloat16)
        out = {"X": X[:, :d], "M": s["M_values"][:, :d], "V": s["V_values"][:, :d]}
    if c["copy"]:
        s["X16"][:, :d] = (x if c["bits"] == 32 else X[:, :d]).to(torch.bfloat16)
        out["X16"] = s["X16"][:, :d]
    return out


_PLAIN = {"linear": _plain_linear, "lgrad": _plain_lgrad, "xent": _plain_xent, "adamw": _plain_adamw}


# ---------------------------------------------------------------- the library's calls


def _own(s):
    c, ctx = s["case"], s["ctx"]
    if s["kind"] == "linear":
        ctx.linear(s["W"], c["offset"], s["A"], s["rows"], s["Y"], relu=c["relu"])
        return s["Y"]
    if s["kind"] == "lgrad":
        ctx.linear_grad_input(s["W"], c["offset"], s["dY"], s["rows"], s["dA"], relu_of=s["A"] if c["relu"] else None)
        ctx.linear_grad_weight(s["dY"], s["A"], s["rows"], s["G"], c["offset"], accumulate=c["accumulate"])
        return {"dA": s["dA"], "G": s["G"][:, c["offset"]:c["offset"] + c["N"] * c["K"]]}
    if s["kind"] == "xent":
        ctx.cross_entropy(s["logits"], s["labels"], s["rows"], s["dlogits"], s["loss"])
        return {"loss": s["loss"], "dlogits": s["dlogits"]}
    opt, d = s["optimizer"], c["d"]
    opt.step(s["X"], s["G"], s["M"], s["V"], s["S"], lr=LR, t=STEP, beta1=BETA1, beta2=BETA2, eps=EPS, seed=s["seed"], X16=s.get("X16"))
    out = {"X": s["X"][:, :d], "M": s["M"][:, :d], "V": s["V"][:, :d]}
    if c["bits"] == 8:
        opt.values(s["M"], s["V"], s["S"], s["M_values"], s["V_values"])
        out.update(M=s["M_values"][:, :d], V=s["V_values"][:, :d])
    if c["copy"]:
        out["X16"] = s["X16"][:, :d]
    return out


def run(state):
    return _own(state) if own else _PLAIN[state["kind"]](state)


# ---------------------------------------------------------------- work and the definition in 64 bits


def work(case):
    kind, n = case["kind"], case["n"]
    e = 4 if case["dtype"] == "f32" else 2
    if kind in ("linear", "lgrad"):
        M, K, N = case["M"], case["K"], case["N"]
        product = 2.0 * M * K * N
        if kind == "linear":
            return {"bytes": e * (n * K * N + M * K) + (4 if case["wide"] else e) * M * N, "flops": product}
        # weights, dY and A in; dA and the weights' gradient out, which is read too where it is added to
        return {"bytes": e * (n * K * N + 2 * M * K + M * N) + (8 if case["accumulate"] else 4) * n * K * N, "flops": 2 * product}
    if kind == "xent":
        return {"bytes": 2 * e * case["M"] * case["C"] + 4 * case["M"] + 4 * n, "flops": 5.0 * case["M"] * case["C"]}
    elements = n * case["d"]
    # models in and out, the gradient, both moments in and out, and what is written beside them (the bf16 copy; the values
    # that 8-bit moments stand for, with the codes read once more for those)
    moments = 16 if case["bits"] == 32 else 4 + 2 + 4
    return {"bytes": elements * (2 * e + 4 + moments + (2 if case["copy"] else 0)), "flops": 15.0 * elements}


def _owner_of_rows(case, seed):
    offs = _row_offsets(case["n"], case["M"], case["spread"], seed)
    return offs, [i for i in range(case["n"]) for _ in range(offs[i + 1] - offs[i])]


def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_layer, "lgrad": _exact_layer, "xent": _exact_xent, "adamw": _exact_adamw}[case["kind"]](case, seed, s)


def _exact_layer(case, seed, s):
    """Worker by worker, in double precision."""
    K, N, off = case["K"], case["N"], case["offset"]
    offs, _ = _owner_of_rows(case, seed)
    A = s["A"].double()
    forward = case["kind"] == "linear"
    rows = torch.zeros(case["M"], N if forward else K, dtype=torch.float64, device=DEV)
    G = None if forward else torch.zeros(case["n"], N * K, dtype=torch.float64, device=DEV)
    for i in range(case["n"]):
        lo, hi = offs[i], offs[i + 1]
        W = s["W"][i, off:off + N * K].double().reshape(N, K)
        if forward:
            rows[lo:hi] = A[lo:hi] @ W.t()
        else:
            dY = s["dY"][lo:hi].double()
            rows[lo:hi] = dY @ W
            G[i] = (dY.t() @ A[lo:hi]).reshape(-1)
    if forward:
        return torch.relu(rows) if case["relu"] else rows
    if case["accumulate"]:
        G += s["G"][:, off:off + N * K].double()
    return {"dA": rows * (A > 0) if case["relu"] else rows, "G": G}


def _exact_xent(case, seed, s):
    offs, _ = _owner_of_rows(case, seed)
    loss = torch.zeros(case["n"], dtype=torch.float64, device=DEV)
    grad = torch.zeros(case["M"], case["C"], dtype=torch.float64, device=DEV)
    for i in range(case["n"]):
        mine = torch.arange(offs[i], offs[i + 1], device=DEV)
        mine = mine[s["labels"][mine] >= 0]
        if mine.numel():
            z, y = s["logits"][mine].double(), s["labels"][mine].long()[:, None]
            logp = torch.log_softmax(z, dim=1)
            loss[i] = -logp.gather(1, y).mean()
            grad[mine] = logp.exp().scatter_add(1, y, torch.full_like(y, -1, dtype=torch.float64)) / mine.numel()
    return {"loss": loss, "dlogits": grad}


def _exact_random(worker_count, lanes, step, seed):
    """The words of the rounding from the generator's definition, products taken in 16-bit halves."""
    def product(a, b):  # a constant and a tensor of 32-bit numbers: (upper, lower) 32 bits
        al, ah, bl, bh = a & 0xFFFF, a >> 16, b & 0xFFFF, b >> 16
        mid = al * bh + ((al * bl) >> 16)
        mid2 = ah * bl + (mid & 0xFFFF)
        return ah * bh + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xFFFF) << 16) | ((al * bl) & 0xFFFF)
    zero = torch.zeros(worker_count, lanes, dtype=torch.int64, device=DEV)
    x = [zero + torch.arange(lanes, device=DEV), zero + 0x41646157, zero + torch.arange(worker_count, device=DEV)[:, None], zero + step]
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        (h0, l0), (h1, l1) = product(0xD2511F53, x[0]), product(0xCD9E8D57, x[2])
        x = [h1 ^ x[1] ^ key[0], l1, h0 ^ x[3] ^ key[1], l0]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    return torch.stack(x, dim=2).reshape(worker_count, 4 * lanes)


def _exact_round(x, r, bias):
    """The 8-bit values nearest below and above x, chosen by r / 2^16, in double precision (x finite)."""
    low = -13 if bias == 7 else -29  # the least exponent of the normal numbers, relative to the largest magnitude's
    mag = x.abs()
    E = torch.floor(torch.log2(mag.amax(-1, keepdim=True).clamp(min=2.0 ** -111)))
    e = torch.maximum(torch.floor(torch.log2(mag.clamp(min=2.0 ** -300))), E + low)
    unit = torch.exp2(e - 3)
    return torch.sign(x) * torch.floor(mag / unit + r.double() / 65536.0) * unit


def _exact_value(code, E, bias):
    """What a code stands for: a table of the 128 or 256 magnitudes."""
    digits = 128 if bias == 7 else 256
    table = torch.tensor([(k % 8) * 2.0 ** (-bias - 2) if k < 8 else (1 + (k % 8) / 8) * 2.0 ** (k // 8 - bias) for k in range(digits)],
                         dtype=torch.float64, device=DEV)
    value = table[(code % digits).long()] * torch.exp2(E.double() - (134 if bias == 7 else 142))[..., None]
    return torch.where(code >= 128, -value, value) if bias == 7 else value


def _exact_adamw(case, seed, s):
    n, d = case["n"], case["d"]
    X = s["X"][:, :d].double()
    out = {"X": X}
    M = s["M_values" if case["bits"] == 8 else "M"].double()
    V = s["V_values" if case["bits"] == 8 else "V"].double()
    first = 0
    words = 0
    if case["bits"] == 8:
        count = sum(-(-length // BLOCK) for _, length in s["tensors"])
        words = _exact_random(n, count * BLOCK // 4, STEP, s["seed"])
        S = s["S"].view(n, -1, 2)
    for k, (at, length) in enumerate(s["tensors"]):
        cols = slice(at, at + length)
        blocks = -(-length // BLOCK)
        if case["bits"] == 8:
            def cut(t):  # the tensor's columns as blocks, zeros past the end
                return torch.nn.functional.pad(t, (0, blocks * BLOCK - length)).reshape(n, blocks, BLOCK)
            E = S[:, first:first + blocks]
            m = _exact_value(cut(s["M"][:, cols]), E[..., 0], 7).reshape(n, -1)[:, :length]
            v = _exact_value(cut(s["V"][:, cols]), E[..., 1], 15).reshape(n, -1)[:, :length]
        else:
            m, v = M[:, cols], V[:, cols]
        g = s["G"][:, cols].double()
        m = BETA1 * m + (1 - BETA1) * g
        v = BETA2 * v + (1 - BETA2) * g ** 2
        lr = LR * s["scale"][k]
        X[:, cols] -= lr * (s["decay"][k] * X[:, cols] + m / (1 - BETA1 ** STEP) / ((v / (1 - BETA2 ** STEP)).sqrt() + EPS))
        if case["bits"] == 8:
            w = words[:, first * BLOCK:(first + blocks) * BLOCK].reshape(n, blocks, BLOCK)
            m = _exact_round(cut(m), w % 65536, 7).reshape(n, -1)[:, :length]
            v = _exact_round(cut(v), w // 65536, 15).reshape(n, -1)[:, :length]
        M[:, cols], V[:, cols] = m, v
        first += blocks
    out.update(M=M[:, :d], V=V[:, :d])
    if case["copy"]:
        out["X16"] = X
    return out

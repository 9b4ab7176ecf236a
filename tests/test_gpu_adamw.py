"""AdamW: optimizers without tensors, numbers at the ends of fp32, every path of the rounding to 8 bits."""
import numpy as np
import pytest
import torch

import paper_2006_08085_amd as D

pytestmark = pytest.mark.gpu
DEV, BF16, F32 = "cuda:0", torch.bfloat16, torch.float32


@pytest.mark.parametrize("spans", [[], [(3, 0), (20, 0)]], ids=["no-tensors", "empty-tensors"])
@pytest.mark.parametrize("bits", [8, 32])
def test_without_columns_nothing_happens(spans, bits):
    n, d = 3, 40
    ctx = D.detag_create(D.Topology.ring(), n, d, 64)
    opt = D.AdamW(ctx, spans, bits=bits)
    assert opt.blocks == 0
    M, V, S = opt.new_moments(DEV)
    X, G = torch.ones(n, 64, device=DEV), torch.ones(n, 64, device=DEV)
    X16 = torch.full((n, 64), 3.0, dtype=BF16, device=DEV)
    opt.step(X, G, M, V, S, lr=0.1, t=1, X16=X16)
    if bits == 8:
        out = [torch.full((n, 64), 5.0, device=DEV) for _ in range(2)]
        opt.values(M, V, S, *out)
        assert (out[0] == 5).all() and (out[1] == 5).all()
    assert (X == 1).all() and (X16 == 3).all() and (M == 0).all() and (V == 0).all()


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("eps", [1e-45, 1e-40, 1e-38, 2.0 ** -126])
def test_an_eps_below_the_normal_numbers(eps, bits):
    """Columns that have never had a gradient stay where they are, however small eps is; the others step by lr."""
    n, d = 2, 300
    ctx = D.detag_create(D.Topology.ring(), n, d, 320)
    opt = D.AdamW(ctx, [(0, d)], bits=bits)
    M, V, S = opt.new_moments(DEV)
    X, G = torch.ones(n, 320, device=DEV), torch.zeros(n, 320, device=DEV)
    G[:, ::3] = 0.5
    opt.step(X, G, M, V, S, lr=0.25, t=1, eps=eps)
    # m / (1 - beta1) = g, v / (1 - beta2) = g^2, root and reciprocal within 2^-22
    want = torch.where(G > 0, 0.75, 1.0)
    want[:, d:] = 1.0
    assert torch.allclose(X, want, rtol=0, atol=2.0 ** -22)


def test_numbers_that_fp32_does_not_hold_are_refused():
    """Finite in 64 bits, infinite in the kernel: every model would be NaN."""
    n, d = 1, 300
    ctx = D.detag_create(D.Topology.ring(), n, d, 320)
    for more in (dict(weight_decay=[1e39]), dict(lr_scale=[-3.5e38])):
        with pytest.raises(D.DetagError) as e:
            D.AdamW(ctx, [(0, d)], **more)
        assert e.value.status == D.DETAG_EINVAL and "fp32" in e.value.message
    opt = D.AdamW(ctx, [(0, d)], weight_decay=[3.4e38], lr_scale=[0.0])
    M, V, S = opt.new_moments(DEV)
    X, G = torch.ones(n, 320, device=DEV), torch.zeros(n, 320, device=DEV)
    for more in (dict(lr=1e39), dict(lr=-1e39), dict(lr=0.1, eps=1e300)):
        with pytest.raises(D.DetagError) as e:
            opt.step(X, G, M, V, S, t=1, **more)
        assert e.value.status == D.DETAG_EINVAL and "fp32" in e.value.message
    opt.step(X, G, M, V, S, lr=0.1, t=1, eps=3.4e38)
    assert (X == 1).all()


# ---------------------------------------------------------------- 8-bit moments, code by code

TOP = {7: 134, 15: 142}                               # y = magnitude * 2^(TOP - E), by the codes' bias


def _random(blocks, worker, t, seed):
    """The words of a worker's columns, (blocks, 256): Philox-4x32-10 from its definition."""
    mask = np.uint64(0xFFFFFFFF)
    ident = np.arange(blocks * 64, dtype=np.uint64)
    c = [ident, np.full_like(ident, 0x41646157), np.full_like(ident, worker), np.full_like(ident, t)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), p1 & mask, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), p0 & mask]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(c, 1).reshape(blocks, 256)


def _encode(x, r, bias):
    """A block's codes, their exponent, and which of them may be one more: 2^9 y + 2^-16 r (2^17 y for v) of a denormal code is a sum in fp32
    below 16, which rounds up to a whole number from 2^-20 below it."""
    mag = np.abs(x.astype(np.float64))
    E = max(16, int(np.max(mag).astype(np.float32).view(np.int32)) >> 23)
    y = mag * 2.0 ** (TOP[bias] - E)
    normal = y >= 2.0 ** (1 - bias)
    e = np.floor(np.log2(np.where(normal, y, 1.0)))
    steps = np.where(normal, y / 2.0 ** (e - 3), y * 2.0 ** (bias + 2)) + r / 65536.0
    code = np.floor(steps) + np.where(normal, 8 * (e + bias) - 8, 0)
    tie = ~normal & (np.ceil(steps) - steps <= 2.0 ** -20) & (np.ceil(steps) > steps)
    return code.astype(np.int64) + (128 * np.signbit(x) if bias == 7 else 0), E, tie


def _decode(code, E, bias):
    """In 64 bits; works on arrays of exponents."""
    mag, E = (code % 128 if bias == 7 else code), np.maximum(E, 16)
    y = np.where(mag < 8, mag * 2.0 ** (-bias - 2), (1 + (mag % 8) / 8) * 2.0 ** (mag // 8 - bias)) * 2.0 ** (E.astype(np.float64) - TOP[bias])
    y = np.where(mag == (127 if bias == 7 else 255), np.nan, y)
    return np.where(code >= 128, -y, y) if bias == 7 else y


# magnitudes of the gradients: 2^scale at most, 2^(scale - span) at least, in every block.  With beta1 = 1/2 the first m are half of that, so
# E of m is 126 + scale; the first v are squares times 1 - beta2, E of v 125 or 126 + 2 scale.  Codes are taken together where E is
# within 30..140 and all are normal: spans of up to 13 for m, 14 for v.
@pytest.mark.parametrize("span", [3, 13, 14, 15])
@pytest.mark.parametrize("scale,beta2", [(0, 0.75), (-97, 0.75), (-96, 0.75), (-95, 0.75), (14, 0.75), (15, 0.75), (-48, 0.75), (-47, 0.75), (7, 0.75), (8, 0.75),
                                         (-48, 0.5), (7, 0.5)])
def test_codes_of_blocks_without_zeros(scale, beta2, span):
    n, spans, f = 3, [(1, 768), (770, 612), (1400, 50)], np.float32
    d, ld = 1450, 1472
    ctx = D.detag_create(D.Topology.ring(), n, d, ld)
    opt = D.AdamW(ctx, spans, bits=8)
    rng = np.random.default_rng(1000 + scale)
    blocks = [slice(c, min(c + 256, a + length)) for a, length in spans for c in range(a, a + length, 256)]
    assert opt.blocks == len(blocks) == 7
    M, V, S = opt.new_moments(DEV)
    X, seed = torch.zeros(n, ld, device=DEV), (5 << 40) + 9
    together = {7: 126 + scale in range(30, 141) and span <= 13, 15: (125 + (beta2 == 0.5) + 2 * scale) in range(30, 141) and span <= 14}
    for t in (1, 2, 3):
        G = np.exp2(scale - span * rng.random((n, ld))) * rng.choice([-1.0, 1.0], (n, ld))
        for k in blocks:
            G[:, k.start + 3], G[:, k.start + 40] = -2.0 ** scale, 2.0 ** (scale - span)
        G = G.astype(f)
        before = [a.cpu().numpy() for a in (M, V, S)]
        opt.step(X, torch.tensor(G).to(DEV), M, V, S, lr=1e-3, t=t, beta1=0.5, beta2=beta2, eps=1e-6, limit=4.0, seed=seed)
        after = [a.cpu().numpy() for a in (M, V, S)]
        for i in range(n):
            words = _random(len(blocks), i, t, seed)
            for b, k in enumerate(blocks):
                g, count = G[i, k], k.stop - k.start
                old = [_decode(before[j][i, k].astype(np.int64), before[2][i, 2 * b + j], bias).astype(f) for j, bias in ((0, 7), (1, 15))]
                new = (old[0] * f(0.5) + g * f(0.5), old[1] * f(beta2) + (g * g) * f(1 - beta2))
                for j, bias, r in ((0, 7, words[b, :count] & np.uint64(0xFFFF)), (1, 15, words[b, :count] >> np.uint64(16))):
                    code, E, tie = _encode(new[j], r.astype(np.float64), bias)
                    got, where = after[j][i, k].astype(np.int64), (t, i, b, "mv"[j])
                    assert after[2][i, 2 * b + j] == E, where
                    assert np.array_equal(got[~tie], code[~tie]), where
                    assert np.isin(got[tie] - code[tie], (0, 1)).all(), where
                    if t == 1 and count == 256:       # the case is what its numbers say
                        y = np.abs(new[j].astype(np.float64)) * 2.0 ** (TOP[bias] - E)
                        assert together[bias] == (30 <= E <= 140 and bool((y >= 2.0 ** (1 - bias)).all())), where


def test_what_small_moments_are_read_back_as():
    """Every code under every least exponent: fp32 holds all values; bf16 those of m, and of v from an exponent of 26 on, below that the
    nearest."""
    exponents = [0, 1, 15, 16, 17, 20, 24, 25, 26, 27, 60, 127, 200, 254]
    n, d = len(exponents), 512
    ctx = D.detag_create(D.Topology.ring(), n, d, d)
    opt = D.AdamW(ctx, [(0, d)], bits=8)
    codes = torch.arange(256, dtype=torch.uint8).repeat(n, 2).contiguous()
    S = torch.tensor(exponents, dtype=torch.uint8).view(n, 1).repeat(1, 4).contiguous()
    out = [torch.empty(n, d, dtype=t, device=DEV) for t in (F32, F32, BF16, BF16)]
    for pair in (out[:2], out[2:]):
        opt.values(codes.to(DEV), codes.to(DEV), S.to(DEV), *pair)
    E, c = np.array(exponents)[:, None], codes.numpy().astype(np.int64)
    for j, bias in ((0, 7), (1, 15)):
        with np.errstate(over="ignore"):
            want = _decode(c, E, bias).astype(np.float32)  # exact, or infinite: 2^128 and more under the largest exponent
        wide, narrow = out[j].cpu().numpy(), out[2 + j].float().cpu().numpy()
        assert np.array_equal(wide, want, equal_nan=True)
        assert np.array_equal(narrow, torch.tensor(want).to(BF16).float().numpy(), equal_nan=True)
        exact = (np.maximum(E, 16) >= (16 if j == 0 else 26)).repeat(d, 1)
        assert np.array_equal(narrow[exact], want[exact], equal_nan=True)
    assert (out[3].cpu().double() != out[1].cpu().double()).any()  # some are not exact


# ---------------------------------------------------------------- every form of the step

def _columns(spans, ld):
    inside = torch.zeros(ld, dtype=torch.bool, device=DEV)
    for a, length in spans:
        inside[a:a + length] = True
    return inside


@pytest.mark.parametrize("state", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("copy", [False, True], ids=["alone", "copy"])
@pytest.mark.parametrize("d", [5003, 4_000_003], ids=["stays", "streams"])
def test_a_step_in_32_bits(d, copy, state):
    """A step of fp32's roundings from given moments, and the models' own rounding: half a spacing, at most 2^-8 of a bf16 one."""
    n, spans = 3, [(3, d // 2), (d // 2 + 3, d - d // 2 - 10)]
    ctx = D.detag_create(D.Topology.ring(), n, d, d + 5, D.DETAG_BF16 if state is BF16 else D.DETAG_F32)
    opt = D.AdamW(ctx, spans, [0.1, 0.0], [1.0, 0.5])
    g = torch.Generator(device=DEV).manual_seed(d)
    X = torch.randn(n, d + 5, generator=g, device=DEV).to(state)
    G, M, V = torch.randn(n, d + 5, generator=g, device=DEV), 0.1 * torch.randn(n, d + 5, generator=g, device=DEV), torch.rand(n, d + 5, generator=g, device=DEV)
    X16 = torch.full((n, d + 5), 3.0, dtype=BF16, device=DEV) if copy else None
    was = [a.clone() for a in (X, M, V)]
    opt.step(X, G, M, V, lr=0.02, t=9, X16=X16)
    inside = _columns(spans, d + 5)
    m, v = 0.9 * was[1].double() + 0.1 * G.double(), 0.999 * was[2].double() + 0.001 * G.double() ** 2
    s, w = (torch.full((d + 5,), a, dtype=torch.float64, device=DEV) for a in (1.0, 0.1))
    s[spans[1][0]:], w[spans[1][0]:] = 0.5, 0.0
    x = was[0].double() * (1 - 0.02 * s * w) - 0.02 * s * (m / (1 - 0.9 ** 9)) / ((v / (1 - 0.999 ** 9)).sqrt() + 1e-8)
    for got, ref, old, rtol in ((X, x, was[0], 2e-6 + (2.0 ** -8 if state is BF16 else 0)), (M, m, was[1], 2e-6), (V, v, was[2], 2e-6)):
        assert torch.allclose(got[:, inside].double(), ref[:, inside], rtol=rtol, atol=2e-7)
        assert torch.equal(got[:, ~inside], old[:, ~inside])
    if copy:
        assert torch.allclose(X16[:, inside].double(), x[:, inside], rtol=2.0 ** -8 + 2e-6, atol=2e-7) and (X16[:, ~inside] == 3).all()


@pytest.mark.parametrize("state", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("copy", [False, True], ids=["alone", "copy"])
def test_a_step_in_8_bits_of_many_blocks(copy, state):
    """The models from given codes, and what so many codes are read back as."""
    n, d = 3, 5_700_000
    spans = [(1, 1_234_567), (1_234_600, 4_400_001)]
    ctx = D.detag_create(D.Topology.ring(), n, d, d + 1, D.DETAG_BF16 if state is BF16 else D.DETAG_F32)
    opt = D.AdamW(ctx, spans, [0.1, 0.1], bits=8)
    assert n * opt.blocks >= 65536 and n * opt.blocks % 4
    g = torch.Generator(device=DEV).manual_seed(1)
    # every finite m but the largest, v far enough from zero that the quotients are numbers of order one or at the limit
    M = torch.randint(0, 112, (n, d + 1), generator=g, device=DEV, dtype=torch.uint8) + 128 * torch.randint(0, 2, (n, d + 1), generator=g, device=DEV, dtype=torch.uint8)
    V = torch.randint(100, 240, (n, d + 1), generator=g, device=DEV, dtype=torch.uint8)
    S = torch.randint(100, 120, (n, 2 * opt.blocks), generator=g, device=DEV, dtype=torch.uint8)
    outs = [torch.full((n, d + 1), 7.0, dtype=t, device=DEV) for t in (F32, F32, BF16, BF16)]
    opt.values(M, V, S, *outs[:2])
    opt.values(M, V, S, *outs[2:])
    inside = _columns(spans, d + 1)
    block, b = torch.zeros(d + 1, dtype=torch.long, device=DEV), 0
    for a, length in spans:
        block[a:a + length] = b + torch.arange(length, device=DEV) // 256
        b += -(-length // 256)
    moments = []
    for j, (codes, bias) in enumerate(((M, 7), (V, 15))):
        table = torch.tensor(_decode(np.arange(256), np.array([TOP[bias]]), bias), device=DEV)
        E = S[:, j::2].double()[:, block] - TOP[bias]
        moments.append(table[codes.long()] * torch.exp2(E))
        for got in (outs[j], outs[2 + j]):
            assert torch.equal(got[:, inside].double(), moments[j][:, inside]) and (got[:, ~inside] == 7).all()
        del E
    del outs
    X = torch.randn(n, d + 1, generator=g, device=DEV).to(state)
    G = torch.randn(n, d + 1, generator=g, device=DEV) * 2.0 ** -15
    X16, was = (torch.full((n, d + 1), 3.0, dtype=BF16, device=DEV) if copy else None), X.clone()
    opt.step(X, G, M, V, S, lr=0.02, t=9, limit=4.0, X16=X16, seed=3)
    m, v = 0.9 * moments[0] + 0.1 * G.double(), 0.999 * moments[1] + 0.001 * G.double() ** 2
    del moments
    step = ((m / (1 - 0.9 ** 9)) / ((v / (1 - 0.999 ** 9)).sqrt() + 1e-8)).clamp_(-4.0, 4.0)
    x = was.double() * (1 - 0.02 * 0.1) - 0.02 * step
    assert torch.allclose(X[:, inside].double(), x[:, inside], rtol=2e-6 + (2.0 ** -8 if state is BF16 else 0), atol=5e-7)
    assert torch.equal(X[:, ~inside], was[:, ~inside])
    if copy:
        assert torch.allclose(X16[:, inside].double(), x[:, inside], rtol=2.0 ** -8 + 2e-6, atol=5e-7) and (X16[:, ~inside] == 3).all()
    del m, v, step, x
    torch.cuda.empty_cache()

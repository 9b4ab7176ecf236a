"""What the tests of a residual block's operators share: inputs in awkward places, references in 64 bits with a bound for every entry.

u = 2^-24 is half a step of fp32, r = eps / 2 of the result's type (2^-8 for bf16, u for fp32).  A sum over lanes adds at most 80 terms one
after the other (64 in a lane, six and eight levels across lanes), so it is off by at most 80 u times the sum of the magnitudes.  The bounds
are written as the kernels' formulas propagate them, and doubled for the terms of second order."""
import math

import numpy as np
import pytest
import torch

import paper_2006_08085_amd as D

DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24
ACTS = {"none": D.DETAG_ACT_NONE, "relu": D.DETAG_ACT_RELU, "gelu": D.DETAG_ACT_GELU, "silu": D.DETAG_ACT_SILU}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def context(n, d, ld=None):
    return D.detag_create(D.Topology.ring(), n, d, D.padded_ld(d) if ld is None else ld)


def offsets(counts, first=0):
    return torch.tensor(np.concatenate([[first], first + np.cumsum(counts)]), dtype=torch.int32, device=DEV)


def spans(counts, first=0):
    at = first
    for i, c in enumerate(counts):
        yield i, at, at + c
        at += c


def matrix(M, cols, dtype, seed, extra=0, shift=0, scale=1.0, around=float("nan"), values=None):
    """An M x cols view with pitch cols + extra whose first element is `shift` elements into its allocation; all else is `around`."""
    pitch = cols + extra
    buf = torch.full((shift + M * pitch + 64,), around, dtype=dtype)
    view = buf[shift:shift + M * pitch].view(M, pitch)
    if values is None and seed is not None:
        values = scale * torch.randn(M, cols, generator=torch.Generator().manual_seed(seed))
    if values is not None:
        view[:, :cols] = values.to(dtype)
    buf = buf.to(DEV)
    return buf[shift:shift + M * pitch].view(M, pitch)[:, :cols], buf


def parameters(n, ld, dtype, parts, seed):
    """n x ld, NaN but for the columns of `parts`: (first, length, mean, scale)."""
    g = torch.Generator().manual_seed(seed)
    P = torch.full((n, ld), float("nan"), dtype=dtype)
    for first, length, mean, scale in parts:
        P[:, first:first + length] = (mean + scale * torch.randn(n, length, generator=g)).to(dtype)
    return P.to(DEV)


def assert_within(got, ref, bound):
    got, ref = got.double(), ref.double()
    assert torch.isfinite(got).all()
    off = (got - ref).abs()
    worst = (off / (bound + 1e-37)).max().item() if off.numel() else 0.0
    assert worst <= 1.0, f"worst {worst:.3g} of the bound"
    return worst


def normal(z):
    """Phi, by erfc: 0.5 (1 + erf) has nothing left in the lower tail."""
    return 0.5 * torch.special.erfc(-z * 0.5 ** 0.5)


def act64(z, act):
    return {"none": lambda: z, "relu": lambda: z.clamp(min=0), "gelu": lambda: z * normal(z), "silu": lambda: z * torch.sigmoid(z)}[act]()


def slope64(z, act):
    if act == "none":
        return torch.ones_like(z)
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return normal(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    p = torch.sigmoid(z)
    return p * (1 + z * (1 - p))


def act_error(z, act, dtype):
    """Of the evaluation of an activation, or of a slope (times 1 + |z|).  fp32: the error function and exp are within 8 steps, and a rounding of
    their argument z^2 / 2 or z counts z^2 or |z| times over.  bf16: 7.1.26 is within 0.75e-7 of Phi, hardware exp2 and rcp within 2^-22 of
    the result, and of their argument's rounding."""
    if act in ("none", "relu"):
        return torch.zeros_like(z)
    size = act64(z, act).abs()
    if dtype is F32:
        return U * (16 + 4 * z * z + 4 * z.abs()) * size
    return 1e-7 * z.abs() * (act == "gelu") + U * (32 + 8 * z * z + 8 * z.abs()) * size


def slope_error(z, act, dtype):
    if act in ("none", "relu"):
        return torch.zeros_like(z)
    spread = 16 + 4 * z * z + 4 * z.abs()
    if dtype is F32:
        return U * spread * (slope64(z, act).abs() + z.abs() * torch.exp(-z * z / 2) + (act == "silu") * 2 * (1 + z.abs()) * torch.sigmoid(z))
    return 1e-7 * (act == "gelu") + 2 * U * spread * (slope64(z, act).abs() + z.abs() * torch.exp(-z * z / 2)
                                                         + (act == "silu") * 2 * (1 + z.abs()) * torch.sigmoid(z))


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2006_08085_amd.build import ensure_built
    ensure_built()
    assert torch.cuda.is_available(), "these tests need the GPU"

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

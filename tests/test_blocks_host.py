"""The operators of a residual block on the host side: what is refused before any GPU is asked."""
import ctypes as C

import pytest
import torch

import paper_2006_08085_amd as D
from paper_2006_08085_amd import build


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.ensure_built()


def test_tensors_elsewhere_are_refused_before_any_launch():
    n, inn, out, M = 4, 8, 8, 6
    ctx = D.detag_create(D.Topology.ring(), n, inn * out, inn * out)
    W, A, Y = torch.zeros(n, inn * out), torch.zeros(M, inn), torch.zeros(M, out)
    rows, lse = torch.zeros(n + 1, dtype=torch.int32), torch.zeros(2, M)
    for call in (lambda: ctx.linear_act(W, 0, A, rows, Y), lambda: ctx.linear_grad_bias(Y, rows, W, 0), lambda: ctx.linear_grad_input_act(W, 0, Y, rows, A),
                 lambda: ctx.layer_norm(W, 0, 8, A, rows, Y), lambda: ctx.layer_norm_grad(W, 0, 8, A, Y, rows, A.clone(), W),
                 lambda: ctx.dropout(A, rows, Y, p=0.1, seed=1, step=1), lambda: ctx.attention(A, A, A, rows, Y, 2, 2),
                 lambda: ctx.attention_grad(A, A, A, rows, Y, lse, Y, A, A, A, 2, 2)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_heads_that_do_not_divide_and_biases_that_are_no_columns():
    ctx = D.detag_create(D.Topology.ring(), 4, 64, 64)
    W, A, rows = torch.zeros(4, 64), torch.zeros(6, 8), torch.zeros(5, dtype=torch.int32)
    for heads in (3, 0, -2):
        with pytest.raises(ValueError, match="heads"):
            ctx.attention(A, A, A, rows, A.clone(), heads, 1)
    for bad in (-1, -64):
        with pytest.raises(ValueError, match="column"):
            D.Context._column(bad)


def test_without_a_gpu_the_calls_say_so():
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    ctx = D.detag_create(D.Topology.ring(), 4, 64, 64)
    L, at, F = D.lib(), [C.c_void_p(4096 * 1024 * k) for k in range(1, 12)], D.DETAG_F32
    for st in (L.detag_linear_act(ctx._h, at[0], 0, 32, F, at[1], 8, at[2], 6, 8, 4, 1, None, 0, None, 0, at[3], 4, F, None),
               L.detag_linear_grad_bias(ctx._h, F, at[0], 4, 0, None, 0, at[1], 6, 4, None, 0, at[2], 0, 0, None),
               L.detag_linear_grad_input_act(ctx._h, at[0], 0, F, at[1], 4, at[2], 6, 8, 4, 0, None, 0, at[3], 8, None),
               L.detag_layer_norm(ctx._h, at[0], 0, 8, F, at[1], 8, at[2], 6, 8, 1e-5, at[3], 8, None),
               L.detag_layer_norm_grad(ctx._h, at[0], 0, 8, F, at[1], 8, at[2], 8, at[3], 6, 8, 1e-5, None, 0, at[4], 8, at[5], 0, None),
               L.detag_dropout(ctx._h, at[0], 8, F, at[1], 6, 8, 0.1, 1, 1, None, 0, at[2], 8, None),
               L.detag_attention(ctx._h, at[0], 8, at[1], 8, at[2], 8, F, at[3], 4, 6, 2, 2, 4, 0.5, 1, at[4], 8, None, None),
               L.detag_attention_grad(ctx._h, at[0], 8, at[1], 8, at[2], 8, F, at[3], 4, 6, 2, 2, 4, 0.5, 1, at[4], 8, at[5], at[6], 8, at[7], 8,
                                      at[8], 8, at[9], 8, None),
               L.detag_reserve_layer_gradient(ctx._h, 6, 8), L.detag_reserve_attention(ctx._h, 6, 2)):
        assert st == D.DETAG_EHIP and b"GPU" in L.detag_last_error(ctx._h)
    for name in ("linear_act", "linear_grad_bias", "layer_norm", "layer_norm_grad", "dropout", "attention", "attention_grad"):
        assert getattr(L, "detag_" + name).restype is C.c_int and callable(getattr(D, "detag_" + name))

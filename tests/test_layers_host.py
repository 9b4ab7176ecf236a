"""Layers, loss and AdamW on the host side: what is refused before any GPU is asked, and blocks of 8-bit moments."""
import ctypes as C

import pytest
import torch

import paper_2006_08085_amd as D
from paper_2006_08085_amd import build


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.ensure_built()


@pytest.mark.parametrize("spans,blocks", [([], 0), ([(0, 0)], 0), ([(0, 1)], 1), ([(0, 256), (256, 257)], 3), ([(0, 5), (5, 5), (10, 290)], 4),
                                          ([(7, 0), (20, 512)], 2)])
def test_blocks_are_cut_from_every_tensors_own_start(spans, blocks):
    ctx = D.detag_create(D.Topology.ring(), 4, 532, 532)
    for bits in (8, 32):
        opt = D.AdamW(ctx, spans, bits=bits)
        assert opt.blocks == blocks
        opt.close()
        opt.close()                                     # once is enough


def test_tensors_that_make_no_sense_are_refused():
    ctx = D.detag_create(D.Topology.ring(), 4, 100, 104)
    for spans, more in [([(0, 101)], {}), ([(100, 1)], {}), ([(-1, 3)], {}), ([(3, -1)], {}), ([(0, 8), (7, 2)], {}), ([(50, 10), (0, 51)], {}),
                        ([(1 << 62, 1 << 62)], {}), ([(0, 4)], dict(bits=4)), ([(0, 4)], dict(weight_decay=[float("inf")])),
                        ([(0, 4)], dict(lr_scale=[float("nan")]))]:
        with pytest.raises(D.DetagError) as e:
            D.AdamW(ctx, spans, **more)
        assert e.value.status == D.DETAG_EINVAL and e.value.message
    for more in (dict(weight_decay=[]), dict(lr_scale=[1.0, 1.0])):
        with pytest.raises(ValueError, match="one number per tensor"):
            D.AdamW(ctx, [(0, 4)], **more)


def test_tensors_elsewhere_are_refused_before_any_launch():
    n, inn, out, M = 4, 8, 4, 6
    ctx = D.detag_create(D.Topology.ring(), n, inn * out, inn * out)
    W, A, Y = torch.zeros(n, inn * out), torch.zeros(M, inn), torch.zeros(M, out)
    rows, labels = torch.zeros(n + 1, dtype=torch.int32), torch.zeros(M, dtype=torch.int32)
    for call in (lambda: ctx.linear(W, 0, A, rows, Y), lambda: ctx.linear_grad_input(W, 0, Y, rows, A), lambda: ctx.linear_grad_weight(Y, A, rows, W, 0),
                 lambda: ctx.cross_entropy(Y, labels, rows, Y)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    opt = D.AdamW(ctx, [(0, inn * out)], bits=8)
    M8, V8, S8 = opt.new_moments("cpu")
    with pytest.raises(ValueError, match="GPU"):
        opt.step(W, W.clone(), M8, V8, S8, lr=0.1, t=1)
    with pytest.raises(ValueError, match="GPU"):
        opt.values(M8, V8, S8, W, W.clone())


def test_without_a_gpu_the_calls_say_so():
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    ctx = D.detag_create(D.Topology.ring(), 4, 32, 32)
    L, at = D.lib(), [C.c_void_p(4096 * 1024 * k) for k in range(1, 7)]
    opt = D.AdamW(ctx, [(0, 32)])
    for st in (L.detag_linear(ctx._h, at[0], 0, D.DETAG_F32, at[1], 8, at[2], 6, 8, 4, 0, at[3], 4, D.DETAG_F32, None),
               L.detag_linear_grad_input(ctx._h, at[0], 0, D.DETAG_F32, at[1], 4, at[2], 6, 8, 4, None, 0, at[3], 8, None),
               L.detag_linear_grad_weight(ctx._h, D.DETAG_F32, at[0], 4, at[1], 8, at[2], 6, 8, 4, at[3], 0, 0, None),
               L.detag_cross_entropy(ctx._h, at[0], 4, D.DETAG_F32, at[1], at[2], 6, 4, at[3], 4, at[4], None),
               L.detag_reserve_cross_entropy(ctx._h, 6),
               L.detag_adamw_step(ctx._h, opt._h, at[0], at[1], at[2], at[3], None, None, 0.1, 0.9, 0.999, 1e-8, 0.0, 1, 0, None)):
        assert st == D.DETAG_EHIP and b"GPU" in L.detag_last_error(ctx._h)

"""Gradients that are not wanted (frozen weights, inputs that need none): the others are right, nothing comes in their place."""
import itertools

import pytest
import torch

import paper_2511_16041_b200 as atb
from tests import operators_ref as ref
from tests.operators_ref import U16, product_bound

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _t(*shape, dtype=BF16, scale=1.0):
    return (torch.randn(shape, device="cuda") * scale).to(dtype)


def _choices(n):
    return list(itertools.product((True, False), repeat=n))


@pytest.mark.parametrize("M,N,dtype", [(5, 64, F32), (700, 1001, BF16), (40, 12288, F32), (9, 20000, BF16)])
@pytest.mark.parametrize("want", _choices(3))
def test_layer_norm(M, N, dtype, want):
    """The kernels and the order of their sums are the same: the same bits."""
    x, dy, w = _t(M, N, dtype=dtype), _t(M, N, dtype=dtype), _t(N, dtype=F32)
    _, mean, rstd = atb.atb_layer_norm(x, w, w)
    full = atb.atb_layer_norm_backward(dy, x, w, mean, rstd)
    some = atb.atb_layer_norm_backward(dy, x, w, mean, rstd, *[None if v else False for v in want])
    for a, b, v in zip(some, full, want):
        assert torch.equal(a, b) if v else a is None


def _check(got, left, right, what):
    """A product of rounded factors in FP32, rounded once."""
    res, e = left @ right, product_bound(left, right)
    ref.check(got, res, e + U16 * (res.abs() + e), what)


@pytest.mark.parametrize("M,D,F", [(1, 64, 136), (6, 1024, 520), (70, 256, 776), (640, 1024, 2736)])
@pytest.mark.parametrize("want", _choices(3))
def test_gated_ffn(M, D, F, want):
    """Products are laid out anew for each choice: each against the formula, on the dg and du that it read."""
    x, dy = _t(M, D), _t(M, D, scale=0.1)
    wg, wu, wd = _t(D, F, scale=D ** -0.5), _t(D, F, scale=D ** -0.5), _t(F, D, scale=F ** -0.5)
    _, H, G, U = atb.atb_gated_ffn(x, wg, wu, wd, save=True)
    ws = torch.empty(atb.atb_gated_ffn_backward_workspace_bytes(M, D, F), dtype=torch.uint8, device="cuda")
    dX, dW, dWd = want
    got = atb.atb_gated_ffn_backward(dy, x, wg, wu, wd, H, G, U, dX=None if dX else False, dWg=None if dW else False, dWu=None if dW else False,
                                     dWd=None if dWd else False, workspace=ws)
    assert [g is not None for g in got] == [dX, dW, dW, dWd]
    dg, du = ws[:4 * M * F].view(BF16).view(2, M, F).double()
    xd, dyd, hd = x.double(), dy.double(), H.double()
    if dX:
        _check(got[0], torch.cat([dg, du], 1), torch.cat([wg, wu], 1).double().t(), "dx")
    if dW:
        _check(got[1], xd.t(), dg, "dwg")
        _check(got[2], xd.t(), du, "dwu")
    if dWd:
        _check(got[3], hd.t(), dyd, "dwd")
    atb.atb_device_status()


@pytest.mark.parametrize("M,V,D,piece", [(1, 1000, 64, 0), (20, 5003, 128, 1024), (300, 3000, 256, 0), (300, 3000, 256, 512)])
@pytest.mark.parametrize("want", _choices(2))
def test_linear_cross_entropy(M, V, D, piece, want):
    x, w = _t(M, D), _t(V, D, scale=2 * D ** -0.5)
    labels, dloss = torch.randint(0, V, (M,), device="cuda"), torch.rand(M, device="cuda") + 0.5
    _, lse = atb.atb_linear_cross_entropy(x, w, labels)
    back = lambda *g: atb.atb_linear_cross_entropy_backward(dloss, x, w, labels, lse, -100, *g, piece=piece)  # noqa: E731
    full, some = back(), back(*[None if v else False for v in want])
    for a, b, v in zip(some, full, want):
        if not v:
            assert a is None
            continue
        # dL has the same bits (its kernel runs alone), sums of M or V products another order: within one unit of the bf16 result and
        # the FP32 sums' error, which is below it by far
        assert float((a.double() - b.double()).abs().max()) <= 2 * U16 * float(b.abs().max())
        assert float((a.double() - b.double()).norm()) <= U16 * float(b.double().norm())
    atb.atb_device_status()


def test_on_another_stream_and_refusals():
    x, wg, wd = _t(4, 16), _t(16, 24), _t(24, 16)
    _, H, G, U = atb.atb_gated_ffn(x, wg, wg, wd, save=True)
    with pytest.raises(ValueError, match="both or neither"):
        atb.atb_gated_ffn_backward(x, x, wg, wg, wd, H, G, U, dWg=False)
    with pytest.raises(ValueError):
        atb.atb_gated_ffn_backward(x, x, wg, wg, wd, H, G, U, dX=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    dX, dWg, dWu, dWd = atb.atb_gated_ffn_backward(x, x, wg, wg, wd, H, G, U, dWg=False, dWu=False, dWd=False, stream=side)
    side.synchronize()
    assert dWg is None and dWu is None and dWd is None and dX.shape == x.shape

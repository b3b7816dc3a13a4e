"""What the gated feed-forward block keeps for its backward pass: G and U in FP32, or in bf16 where the caller says so."""
import pytest
import torch

import paper_2511_16041_b200 as atb
from tests import operators_ref as ref
from tests.operators_ref import product_bound
from tests.test_gpu_gated_ffn import SHAPES, _check_backward, _check_forward, _inputs

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("keep", [F32, BF16])
@pytest.mark.parametrize("M,D,F", SHAPES + [(300, 64, 40), (300, 64, 72), (1000, 2048, 104)])
def test_forward_and_backward(M, D, F, keep):
    act = ("gelu", "gelu_tanh", "silu")[(M + D + F) // 8 % 3]
    x, wg, wu, wd, dy = _inputs(M, D, F)
    room = torch.full((2, M + 1, F), 7.0, dtype=keep, device="cuda")        # a guard row behind each
    Y, H, G, U = atb.atb_gated_ffn(x, wg, wu, wd, act=act, save=True, G=room[0, :M], U=room[1, :M])
    assert G.dtype == U.dtype == keep and bool((room[:, M] == 7).all())
    _check_forward(x, wg, wu, wd, act, Y, H, G, U)
    if keep == F32:                                            # not rounded at all
        xd = x.double()
        for got, w, name in ((G, wg, "g"), (U, wu, "u")):
            ref.check(got, xd @ w.double(), product_bound(xd, w.double()), name)
    ws = torch.empty(atb.atb_gated_ffn_backward_workspace_bytes(M, D, F), dtype=torch.uint8, device="cuda")
    grads = atb.atb_gated_ffn_backward(dy, x, wg, wu, wd, H, G, U, act=act, workspace=ws)
    atb.atb_device_status()
    _check_backward(dy, x, wg, wu, wd, act, H, G, U, *ws[:4 * M * F].view(BF16).view(2, M, F), *grads)
    # made by the call: the same bits; H and Y do not depend on what is kept
    made = atb.atb_gated_ffn(x, wg, wu, wd, act=act, save=keep)
    for a, b in zip(made, (Y, H, G, U)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("M", [2, 40, 600])
def test_gradients_are_nearer_with_fp32(M):
    D, F = 512, 1368
    x, wg, wu, wd, dy = _inputs(M, D, F)
    args = [t.double().requires_grad_() for t in (x, wg, wu, wd)]
    ref.gated_ffn(*args, "silu").backward(dy.double())
    off = {}
    for save in (True, BF16):
        _, H, G, U = atb.atb_gated_ffn(x, wg, wu, wd, save=save)
        assert G.dtype == U.dtype == (F32 if save is True else BF16) and H.dtype == BF16
        grads = atb.atb_gated_ffn_backward(dy, x, wg, wu, wd, H, G, U)
        off[save] = [float((g.double() - a.grad).norm() / a.grad.norm()) for g, a in zip(grads, args)]
    # bf16 adds the roundings of g and u, about one of 2^-9 rms, to two (dg and du, the result): 2^0.5 against 3^0.5 = 0.82
    for i, name in enumerate(("dx", "dwg", "dwu")):
        assert off[True][i] <= 0.87 * off[BF16][i], (name, off)
    assert off[True][3] == off[BF16][3]


def test_refusals():
    x, wg, wu, wd, dy = _inputs(4, 16, 24)
    _, H, G, U = atb.atb_gated_ffn(x, wg, wu, wd, save=True)
    for call in (lambda: atb.atb_gated_ffn(x, wg, wu, wd, save=torch.float16), lambda: atb.atb_gated_ffn(x, wg, wu, wd, G=G, U=U.to(BF16)),
                 lambda: atb.atb_gated_ffn(x, wg, wu, wd, G=G.double()), lambda: atb.atb_gated_ffn_backward(dy, x, wg, wu, wd, H, G, U.to(BF16)),
                 lambda: atb.atb_gated_ffn_backward(dy, x, wg, wu, wd, H.float(), G, U),
                 lambda: atb.atb_gated_ffn_backward(dy, x, wg, wu, wd, H, G.half(), U.half())):
        with pytest.raises(ValueError):
            call()
    for act in (256, 257, 512):                                # the entries' flag is no activation
        with pytest.raises(atb.AtbError) as e:
            atb.atb_gated_ffn(x, wg, wu, wd, act=act)
        assert e.value.status == 9
    # given by one of the two
    out = atb.atb_gated_ffn(x, wg, wu, wd, save=True, G=torch.empty(4, 24, dtype=BF16, device="cuda"))
    assert out[3].dtype == BF16

"""The activations of the gated feed-forward block relative to their own size, far out on the negative side, where they are
small: products of one term each, so that g, u = 1 and dh = 1 are exact and nothing but the activation is rounded."""
import math

import pytest
import torch

import paper_2511_16041_b200 as atb

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
# Before the rounding to bf16: an exponent of at most 2^7 with four roundings of 2^-24 each (2^-15 of the result), the fast exponential and
# reciprocal and the polynomial (2^-20 together).
ACT = 2.0 ** -14


def _rounded(want, err):
    """`err` and half a unit of bf16 (8 significant bits) where `want` is at most off by it."""
    return err + 2.0 ** (torch.floor(torch.log2(want.abs() + err)) - 8)


def _terms(g, act):
    """act(g), act'(g), and the sum of the magnitudes that act'(g) is made of."""
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s + g * s * torch.sigmoid(-g), s + (g * s * torch.sigmoid(-g)).abs()
    if act == "gelu":
        phi, pdf = 0.5 * torch.erfc(-g / math.sqrt(2)), torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
        return g * phi, phi + g * pdf, phi + (g * pdf).abs()
    c = math.sqrt(2 / math.pi)
    z, dz = c * (g + 0.044715 * g ** 3), c * (1 + 3 * 0.044715 * g * g)
    s, t = torch.sigmoid(2 * z), torch.sigmoid(-2 * z)
    return g * s, s + g * 2 * s * t * dz, s + (g * 2 * s * t * dz).abs()


@pytest.mark.parametrize("act,low", [("silu", -40.0), ("gelu", -12.0), ("gelu_tanh", -8.0)])
@pytest.mark.parametrize("M,D", [(1, 8), (2, 64), (5, 2048), (200, 8), (300, 1024)])
def test_relative_to_the_result(M, D, act, low):
    g = torch.cat([torch.linspace(low, 0, 900), torch.linspace(0, 12, 124)]).to(BF16)
    F = g.numel()
    x, dy = torch.zeros(M, D, dtype=BF16, device="cuda"), torch.zeros(M, D, dtype=BF16, device="cuda")
    wg, wu, wd = (torch.zeros(*s, dtype=BF16, device="cuda") for s in ((D, F), (D, F), (F, D)))
    x[:, :2], wg[0], wu[1], dy[:, 0], wd[:, 0] = 1, g.cuda(), 1, 1, 1
    _, H, G, U = atb.atb_gated_ffn(x, wg, wu, wd, act=act, save=True)
    ws = torch.empty(atb.atb_gated_ffn_backward_workspace_bytes(M, D, F), dtype=torch.uint8, device="cuda")
    atb.atb_gated_ffn_backward(dy, x, wg, wu, wd, H, G, U, act=act, workspace=ws)
    atb.atb_device_status()
    dG, dU = ws[:4 * M * F].view(BF16).view(2, M, F).double()
    assert bool((G == wg[0]).all()) and bool((U == 1).all())
    a, slope, size = _terms(wg[0].double(), act)
    for got, want, err, what in ((H.double(), a, ACT * a.abs(), "h"), (dU, a, ACT * a.abs(), "du"),
                                 (dG, slope, 2 * ACT * size, "dg")):
        over = (got - want).abs() - _rounded(want, err)
        at = int(over.max(0).values.argmax())
        assert float(over.max()) <= 0, f"{what} at g = {float(g[at])}: {float(got[0, at])} for {float(want[at])}"

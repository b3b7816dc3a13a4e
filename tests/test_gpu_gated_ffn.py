"""The gated feed-forward block against the formulas in 64 bits, stage by stage: every stage is checked on the rounded
values that it really read (H, G, U, and dG, dU in the workspace), so the bounds are those of one product."""
import pytest
import torch

import paper_2511_16041_b200 as atb
from tests import operators_ref as ref
from tests.operators_ref import U16, product_bound

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
# the activations go through the fast exponential: a few 2^-22 of the result, and of g in the exponent
ACT_REL = 2.0 ** -18


def _normal(gen, rows, cols, scale=1.0, pad=0):
    return (torch.randn((rows, cols + pad), generator=gen, device="cuda") * scale).to(BF16)[:, :cols]


def _inputs(M, D, F, pad=0, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(77 + seed)
    return (_normal(gen, M, D, 1.0, pad), _normal(gen, D, F, D ** -0.5, pad), _normal(gen, D, F, D ** -0.5, pad),
            _normal(gen, F, D, F ** -0.5, pad), _normal(gen, M, D, 0.1, pad))


def _rounded(want, err):
    return err + U16 * (want.abs() + err)


def _check_forward(x, wg, wu, wd, act, Y, H, G, U):
    x, wg, wu, wd = (t.double() for t in (x, wg, wu, wd))
    g, u = x @ wg, x @ wu
    eg, eu = product_bound(x, wg), product_bound(x, wu)
    if G is not None:
        ref.check(G, g, _rounded(g, eg), "g")
        ref.check(U, u, _rounded(u, eu), "u")
    a, _ = ref.act(g, act)
    h = a * u
    # |act'| < 1.13 for the three; |act(g)| <= |g|
    eh = 1.2 * eg * (u.abs() + eu) + a.abs() * eu + ACT_REL * (g.abs() + 1) * u.abs()
    ref.check(H, h, _rounded(h, eh), "h")
    hd = H.double()
    y = hd @ wd
    ref.check(Y, y, _rounded(y, product_bound(hd, wd)), "y")


def _check_backward(dy, x, wg, wu, wd, act, H, G, U, dG, dU, dX, dWg, dWu, dWd):
    dy, x, wg, wu, wd, H, G, U = (t.double() for t in (dy, x, wg, wu, wd, H, G, U))
    dh, e = dy @ wd.t(), product_bound(dy, wd.t())
    a, slope = ref.act(G, act)
    want = dh * a
    ref.check(dU, want, _rounded(want, e * a.abs() + ACT_REL * (G.abs() + 1) * dh.abs()), "du")
    want = dh * U * slope
    ref.check(dG, want, _rounded(want, e * (U * slope).abs() + ACT_REL * (G.abs() + 1) ** 3 * (dh * U).abs()), "dg")
    dg, du = dG.double(), dU.double()
    want = dg @ wg.t() + du @ wu.t()
    ref.check(dX, want, _rounded(want, product_bound(torch.cat([dg, du], 1), torch.cat([wg, wu], 1).t())), "dx")
    for got, left, right, name in ((dWg, x, dg, "dwg"), (dWu, x, du, "dwu"), (dWd, H, dy, "dwd")):
        want = left.t() @ right
        ref.check(got, want, _rounded(want, product_bound(left.t(), right)), name)


def _run_both(M, D, F, act, pad=0, seed=0):
    x, wg, wu, wd, dy = _inputs(M, D, F, pad, seed)
    Y, H, G, U = atb.atb_gated_ffn(x, wg, wu, wd, act=act, save=True)
    ws = torch.empty(atb.atb_gated_ffn_backward_workspace_bytes(M, D, F), dtype=torch.uint8, device="cuda")
    grads = atb.atb_gated_ffn_backward(dy, x, wg, wu, wd, H, G, U, act=act, workspace=ws)
    atb.atb_device_status()
    dG, dU = ws[:4 * M * F].view(BF16).view(2, M, F)
    return (x, wg, wu, wd, dy), (Y, H, G, U), (dG, dU) + grads


SHAPES = [(1, 8, 8), (1, 64, 64), (2, 72, 136), (3, 1024, 2736), (4, 264, 520), (7, 128, 4104), (8, 1000, 328), (9, 512, 1024), (16, 2048, 1024),
          (31, 64, 72), (64, 328, 264), (127, 128, 256), (128, 256, 128), (129, 136, 264), (256, 512, 1368), (257, 200, 520), (500, 1024, 2736),
          (1000, 320, 4104),
          # several tiles for every CTA or pair, in every product: accumulators and rings wrap round
          (20, 64, 40000), (128, 4104, 10008), (3000, 200, 4104), (2500, 2056, 520)]


@pytest.mark.parametrize("M,D,F", SHAPES)
def test_forward_and_backward(M, D, F):
    act = ("silu", "gelu", "gelu_tanh")[(M + D + F) // 8 % 3]
    ins, outs, grads = _run_both(M, D, F, act)
    _check_forward(*ins[:4], act, *outs)
    _check_backward(ins[4], *ins[:4], act, *outs[1:], *grads)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("M", [1, 5, 200, 900])
def test_every_activation(M, act):
    ins, outs, grads = _run_both(M, 256, 776, act, seed=M)
    _check_forward(*ins[:4], act, *outs)
    _check_backward(ins[4], *ins[:4], act, *outs[1:], *grads)


@pytest.mark.parametrize("M,D,F", [(1, 136, 264), (6, 136, 264), (300, 264, 776)])
def test_strided_operands(M, D, F):
    ins, outs, grads = _run_both(M, D, F, "silu", pad=24)
    _check_forward(*ins[:4], "silu", *outs)
    _check_backward(ins[4], *ins[:4], "silu", *outs[1:], *grads)


@pytest.mark.parametrize("M,D,F", [(1, 128, 136), (5, 2048, 520), (40, 128, 264), (400, 136, 520)])
def test_fused_weights_guards_and_inference(M, D, F):
    """Wg and Wu as the halves of one matrix, outputs inside larger buffers, and the call that keeps only H."""
    x, wg, wu, wd, dy = _inputs(M, D, F)
    both = torch.cat([wg, wu], 1)
    y_buf = torch.full((M + 1, D + 16), 7.0, dtype=BF16, device="cuda")
    h_buf = torch.full((M + 1, F), 7.0, dtype=BF16, device="cuda")
    Y = atb.atb_gated_ffn(x, both[:, :F], both[:, F:], wd, Y=y_buf[:M, :D], H=h_buf[:M])
    _check_forward(x, wg, wu, wd, "silu", Y, h_buf[:M], None, None)
    assert bool((y_buf[M] == 7).all()) and bool((y_buf[:, D:] == 7).all()) and bool((h_buf[M] == 7).all())
    Y2, H, G, U = atb.atb_gated_ffn(x, wg, wu, wd, save=True)
    dboth = torch.full((D, 2 * F + 8), 7.0, dtype=BF16, device="cuda")
    dX, dWg, dWu, dWd = atb.atb_gated_ffn_backward(dy, x, both[:, :F], both[:, F:], wd, H, G, U, dWg=dboth[:, :F], dWu=dboth[:, F:2 * F])
    plain = atb.atb_gated_ffn_backward(dy, x, wg, wu, wd, H, G, U)
    assert bool((dboth[:, 2 * F:] == 7).all())
    for a, b in zip((dX, dWg, dWu, dWd), plain):
        assert torch.equal(a, b)


def test_same_bits_again_and_on_another_stream():
    ins, outs, grads = _run_both(333, 512, 1368, "gelu")
    x, wg, wu, wd, dy = ins
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = atb.atb_gated_ffn(x, wg, wu, wd, act="gelu", save=True)
        back = atb.atb_gated_ffn_backward(dy, x, wg, wu, wd, *again[1:], act="gelu")
    side.synchronize()
    for a, b in zip(outs + grads[2:], again + back):
        assert torch.equal(a, b)


def test_large_pre_activations_saturate():
    """|g| up to several hundred: silu and gelu become 0 or g, their slopes 0 or 1, with no infinity or NaN on the way."""
    for M in (2, 150):
        x, wg, wu, wd, dy = _inputs(M, 64, 64)
        wg = (wg.float() * 400).to(BF16)
        for act in ("silu", "gelu", "gelu_tanh"):
            Y, H, G, U = atb.atb_gated_ffn(x, wg, wu, wd, act=act, save=True)
            _check_forward(x, wg, wu, wd, act, Y, H, G, U)
            ws = torch.empty(atb.atb_gated_ffn_backward_workspace_bytes(M, 64, 64), dtype=torch.uint8, device="cuda")
            grads = atb.atb_gated_ffn_backward(dy, x, wg, wu, wd, H, G, U, act=act, workspace=ws)
            _check_backward(dy, x, wg, wu, wd, act, H, G, U, *ws.view(BF16).view(2, M, 64), *grads)


def test_a_nan_stays_in_its_row():
    for M in (3, 140):
        x, wg, wu, wd, dy = _inputs(M, 128, 264)
        x[1, 5] = float("nan")
        Y = atb.atb_gated_ffn(x, wg, wu, wd)
        assert bool(torch.isnan(Y[1]).all())
        rest = torch.arange(M, device="cuda") != 1
        assert bool(torch.isfinite(Y[rest]).all())


def test_no_rows():
    x, wg, wu, wd, dy = _inputs(4, 64, 72)
    Y, H, G, U = atb.atb_gated_ffn(x[:0], wg, wu, wd, save=True)
    assert Y.shape == (0, 64)
    dX, dWg, dWu, dWd = atb.atb_gated_ffn_backward(dy[:0], x[:0], wg, wu, wd, H, G, U)
    assert all(bool((t == 0).all()) for t in (dWg, dWu, dWd)) and dWd.shape == (72, 64)


def test_gradient_against_differences():
    M, D, F = 6, 64, 136
    for act in ("silu", "gelu", "gelu_tanh"):
        x, wg, wu, wd, dy = _inputs(M, D, F, seed=9)
        _, H, G, U = atb.atb_gated_ffn(x, wg, wu, wd, act=act, save=True)
        grads = [t.double() for t in atb.atb_gated_ffn_backward(dy, x, wg, wu, wd, H, G, U, act=act)]
        args = [t.double() for t in (x, wg, wu, wd)]
        gen = torch.Generator(device="cuda").manual_seed(4)

        def loss(a):
            return float((ref.gated_ffn(*a, act) * dy.double()).sum())

        for i in range(4):
            d = torch.randn(args[i].shape, generator=gen, device="cuda", dtype=torch.float64)
            h = 1e-5
            up, down = list(args), list(args)
            up[i], down[i] = args[i] + h * d, args[i] - h * d
            slope = (loss(up) - loss(down)) / (2 * h)
            # five roundings to bf16 lie between (g, u, h or dg, du, the result): each element within 5 U16 of terms
            # whose signs are independent of d's
            scale = float((grads[i] * d).abs().sum())
            assert abs(slope - float((grads[i] * d).sum())) <= 5 * U16 * scale, (act, i)

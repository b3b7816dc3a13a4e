"""Layer norm, forward, BFP16 output and backward, against the formulas in 64 bits."""
import pytest
import torch

import paper_2511_16041_b200 as atb
from tests import operators_ref as ref
from tests.operators_ref import U16, U32

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _inputs(M, N, dtype, wdtype, pad=0, shift=0.5, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(1000 + seed + M * 7 + N)
    x = (torch.randn((M, N + pad), generator=gen, device="cuda") * 2 + shift).to(dtype)[:, :N]
    dy = torch.randn((M, N + pad), generator=gen, device="cuda").to(dtype)[:, :N]
    w = (torch.randn(N, generator=gen, device="cuda") * 0.2 + 1).to(wdtype)
    b = (torch.randn(N, generator=gen, device="cuda") * 0.2).to(wdtype)
    return x, dy, w, b


def _z_error(x, z, rstd):
    """Bound on |z - exact z|.  The FP32 mean of N terms, each thread adding at most 64 of them before a tree of 10 levels, is
    within 80 U32 mean|x|; rstd, from a sum of the same shape, within 100 U32 of itself; z adds two roundings."""
    a = x.abs().mean(1, keepdim=True)
    return U32 * (100 * z.abs() + rstd * (80 * a + x.abs()) + 4 * z.abs())


def _forward_bound(x, y, z, rstd, w, b, out_dtype):
    t = _z_error(x, z, rstd) * (1 if w is None else w.abs()) + 4 * U32 * (y.abs() + (0 if b is None else b.abs()))
    return t + (U16 * (y.abs() + t) if out_dtype == BF16 else 0)


SHAPES = [(1, 8), (1, 1), (3, 5), (2, 64), (5, 512), (7, 513), (4, 520), (33, 1000), (2, 1001), (9, 4096), (3, 4104), (2, 8192), (2, 8200),
          (3, 16384), (2, 16385), (2, 32768), (2, 40000), (1, 32776), (700, 72)]
# rows enough for every kernel's blocks to walk several of them
SHAPES += [(6000, 257), (3000, 520), (2500, 1001), (1500, 2048), (1400, 4095), (700, 8192), (500, 9001), (460, 16384),
           (4000, 1024), (3000, 1032), (2200, 1537), (900, 2500), (700, 3080), (500, 6144), (480, 6150), (320, 12288), (310, 12301)]


@pytest.mark.parametrize("dtype,wdtype", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("M,N", SHAPES)
def test_forward_and_backward(M, N, dtype, wdtype):
    for pad in (0, 3, 8):
        x, dy, w, b = _inputs(M, N, dtype, wdtype, pad)
        eps = 1e-5
        Y, mean, rstd = atb.atb_layer_norm(x, w, b, eps)
        xd, dyd, wd, bd = x.double(), dy.double(), w.double(), b.double()
        y, z, mu, r = ref.layer_norm(xd, wd, bd, eps)
        ref.check(Y, y, _forward_bound(xd, y, z, r, wd, bd, dtype), f"y {M}x{N} pad {pad}")
        ref.check(mean, mu[:, 0], 80 * U32 * xd.abs().mean(1), "mean")
        if N > 1:
            # a single element has variance 0 up to the rounding of its mean, which eps covers
            ref.check(rstd, r[:, 0], 120 * U32 * r[:, 0] * (1 + r[:, 0] * xd.abs().mean(1)), "rstd")
        dX, dW, dB = atb.atb_layer_norm_backward(dy, x, w, mean, rstd)
        dx, dw, db, g = ref.layer_norm_backward(dyd, z, wd, r)
        ze = _z_error(xd, z, r)
        gz, ga = (g * z).abs().mean(1, keepdim=True), g.abs().mean(1, keepdim=True)
        # each of the three terms: its sums (80 U32), z's own error, rstd's (100 U32), a few roundings
        t = r * (200 * U32 * (g.abs() + ga + z.abs() * gz) + ze * gz + z.abs() * (g.abs() * ze).mean(1, keepdim=True))
        ref.check(dX, dx, t + (U16 * (dx.abs() + t) if dtype == BF16 else 0), f"dx {M}x{N} pad {pad}")
        t = (dyd.abs() * ze).sum(0) + (M + 16) * U32 * (dyd * z).abs().sum(0)
        ref.check(dW, dw, t + (U16 * (dw.abs() + t) if wdtype == BF16 else 0), f"dw {M}x{N} pad {pad}")
        t = (M + 16) * U32 * dyd.abs().sum(0)
        ref.check(dB, db, t + (U16 * (db.abs() + t) if wdtype == BF16 else 0), f"db {M}x{N} pad {pad}")


def test_many_rows_and_repeatability():
    M, N = 5003, 1024
    x, dy, w, b = _inputs(M, N, BF16, F32)
    _, mean, rstd = atb.atb_layer_norm(x, w, b)
    first = atb.atb_layer_norm_backward(dy, x, w, mean, rstd)
    again = atb.atb_layer_norm_backward(dy, x, w, mean, rstd)
    for a, c in zip(first, again):
        assert torch.equal(a, c)
    y, z, mu, r = ref.layer_norm(x.double(), w.double(), b.double(), 1e-5)
    dx, dw, db, g = ref.layer_norm_backward(dy.double(), z, w.double(), r)
    t = (dy.double().abs() * _z_error(x.double(), z, r)).sum(0) + (M + 16) * U32 * (dy.double() * z).abs().sum(0)
    ref.check(first[1], dw, t, "dw")


def test_without_weights():
    x, dy, _, b = _inputs(6, 264, F32, F32)
    Y, mean, rstd = atb.atb_layer_norm(x)
    y, z, mu, r = ref.layer_norm(x.double(), None, None, 1e-5)
    ref.check(Y, y, _forward_bound(x.double(), y, z, r, None, None, F32), "y")
    Yb, _, _ = atb.atb_layer_norm(x, None, b)
    yb = y + b.double()
    ref.check(Yb, yb, _forward_bound(x.double(), yb, z, r, None, b.double(), F32), "y with a bias alone")
    dX, dW, dB = atb.atb_layer_norm_backward(dy, x, None, mean, rstd)
    assert dW.dtype == F32
    dx, dw, db, g = ref.layer_norm_backward(dy.double(), z, None, r)
    assert float((dX.double() - dx).abs().max()) <= 1e-4 and float((dW.double() - dw).abs().max()) <= 1e-4


def test_a_large_offset_keeps_its_digits():
    """|mean| = 3000 standard deviations: a variance from sum(x^2) would have no digit left."""
    x, _, w, b = _inputs(4, 2048, F32, F32, shift=6000.0)
    Y, mean, rstd = atb.atb_layer_norm(x, w, b)
    y, z, mu, r = ref.layer_norm(x.double(), w.double(), b.double(), 1e-5)
    ref.check(Y, y, _forward_bound(x.double(), y, z, r, w.double(), b.double(), F32), "y")


def test_constant_rows_and_special_values():
    x = torch.full((3, 40), 2.0, device="cuda")
    x[1] = 0.0
    x[2, 7] = float("nan")
    Y, mean, rstd = atb.atb_layer_norm(x, eps=1e-6)
    assert bool((Y[:2] == 0).all()) and torch.equal(mean[:2].cpu(), torch.tensor([2.0, 0.0]))
    assert float((rstd[:2] - 1e3).abs().max()) < 1e-3
    assert bool(torch.isnan(Y[2]).all())
    x[2, 7] = float("inf")
    assert bool(torch.isnan(atb.atb_layer_norm(x)[0][2]).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M,N", [(1, 8), (31, 72), (32, 64), (33, 520), (100, 4096), (5, 8200), (2, 40000)])
def test_bfp16_output_is_the_quantiser_on_the_fp32_result(M, N, dtype):
    x, _, w, b = _inputs(M, N, dtype, F32)
    x[0, :8] = 0
    mant, exp, mean, rstd = atb.atb_layer_norm_bfp16(x, w, b)
    # fp32 values of a bf16 input are exact, so the fp32 entry computes the same results from them
    Y, mean32, rstd32 = atb.atb_layer_norm(x.float(), w, b)
    want_mant, want_exp = atb.atb_quantize_bfp16(Y)
    assert torch.equal(mean, mean32) and torch.equal(rstd, rstd32)
    assert torch.equal(mant, want_mant) and torch.equal(exp, want_exp)


def test_empty():
    x = torch.empty((0, 16), device="cuda")
    w = torch.ones(16, device="cuda")
    Y, mean, rstd = atb.atb_layer_norm(x, w)
    assert Y.shape == (0, 16)
    dX, dW, dB = atb.atb_layer_norm_backward(x, x, w, mean, rstd)
    assert dX.shape == (0, 16) and bool((dW == 0).all()) and bool((dB == 0).all())


def test_on_another_stream_with_guarded_rows():
    x, dy, w, b = _inputs(37, 1000, BF16, BF16, pad=24)
    Y = torch.full((37, 1024), 7.0, dtype=BF16, device="cuda")
    dX = torch.full((37, 1024), 7.0, dtype=BF16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _, mean, rstd = atb.atb_layer_norm(x, w, b, Y=Y[:, :1000])
        atb.atb_layer_norm_backward(dy, x, w, mean, rstd, dX=dX[:, :1000])
    side.synchronize()
    assert bool((Y[:, 1000:] == 7).all()) and bool((dX[:, 1000:] == 7).all())
    assert torch.equal(Y[:, :1000], atb.atb_layer_norm(x, w, b)[0])


def test_gradient_against_differences():
    x, dy, w, b = _inputs(4, 96, F32, F32)
    _, mean, rstd = atb.atb_layer_norm(x, w, b)
    grads = [t.double() for t in atb.atb_layer_norm_backward(dy, x, w, mean, rstd)]
    args = [x.double(), w.double(), b.double()]
    gen = torch.Generator(device="cuda").manual_seed(3)

    def loss(a):
        return float((ref.layer_norm(a[0], a[1], a[2], 1e-5)[0] * dy.double()).sum())

    for i in range(3):
        d = torch.randn(args[i].shape, generator=gen, device="cuda", dtype=torch.float64)
        h = 1e-5
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + h * d, args[i] - h * d
        slope = (loss(up) - loss(down)) / (2 * h)
        # differences: h^2 of the third derivative and 1e-16 / h of the loss; the gradient: fp32
        scale = float((grads[i] * d).abs().sum())
        assert abs(slope - float((grads[i] * d).sum())) <= 1e-5 * scale + 1e-6, i

"""Matrices of more than 2^31 elements: the results that are sums over all of them, the pieces of a vocabulary that start beyond, and
a feed-forward block with as many hidden values."""
import math

import pytest
import torch

import paper_2511_16041_b200 as atb
from tests import operators_ref as ref
from tests.operators_ref import U16, U32, product_bound

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(autouse=True)
def _room():
    torch.manual_seed(7)
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 60 * 2 ** 30:
        pytest.skip("not enough free device memory")
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("N", [8192, 8191])
def test_layer_norm_weight_gradients(N):
    M = 2 ** 31 // N + 1000
    x = torch.empty((M, N), dtype=BF16, device="cuda").normal_()
    w = torch.rand(N, device="cuda") + 0.5
    _, mean, rstd = atb.atb_layer_norm(x, w, w)
    _, dW, dB = atb.atb_layer_norm_backward(x, x, w, mean, rstd)
    dw, db, size = (torch.zeros(N, dtype=torch.float64, device="cuda") for _ in range(3))
    for i in range(0, M, 1 << 14):
        part = x[i:i + (1 << 14)].double()
        z = ref.layer_norm(part, None, None, 1e-5)[1]
        dw += (part * z).sum(0)
        size += (part * z).abs().sum(0)
        db += part.sum(0)
    # a walker of at least 148 adds its rows one by one, 592 walkers at most are added up; z is off by 2^-20 at most
    adds = M / 148 + 600
    ref.check(dW, dw, (adds * U32 + 2.0 ** -20) * size, "dw")
    ref.check(dB, db, adds * U32 * (size + M), "db")


@pytest.mark.parametrize("piece", [0, 131072])
def test_linear_cross_entropy_gradients(piece):
    """Row m gives much of its probability to word V - 100 - m, beyond 2^31 elements of W; labels lie in every piece of 131072 words."""
    M, D = 9, 4096
    V = 2 ** 31 // D + 3001
    x = torch.randn((M, D), device="cuda").to(BF16)
    w = torch.empty((V, D), dtype=BF16, device="cuda").normal_(std=2.0 / D ** 0.5)
    for m in range(M):
        w[V - 100 - m] = (x[m].float() * ((math.log(V) + 2) / float(x[m].float().square().sum()))).to(BF16)
    labels = torch.tensor([3, 131071, 131072, 262144 + 7, 400000, 524287, 524288, V - 2, V - 100 - 8], device="cuda")
    dloss = torch.rand(M, device="cuda") + 0.5
    loss, lse = atb.atb_linear_cross_entropy(x, w, labels)
    dX, dW = atb.atb_linear_cross_entropy_backward(dloss, x, w, labels, lse, piece=piece)
    atb.atb_device_status()
    step = 1 << 15
    xd = x.double()
    logits = torch.cat([xd @ w[i:i + step].double().t() for i in range(0, V, step)], 1)
    want = torch.logsumexp(logits, 1)
    picked = logits.gather(1, labels[:, None])[:, 0]
    ref.check(lse, want, 1e-4 * want.abs(), "lse")
    ref.check(loss, want - picked, 1e-4 * (want.abs() + picked.abs()), "loss")
    d = torch.exp(logits - want[:, None])
    assert bool((d[torch.arange(M), V - 100 - torch.arange(M)] > 0.1).all())
    d[torch.arange(M), labels] -= 1
    d *= dloss.double()[:, None]
    dx = sum(d[:, i:i + step] @ w[i:i + step].double() for i in range(0, V, step))
    # dL's roundings: in full for the two words that carry a row (a single rounding is not evened out), in the mean square for the
    # others; its exponents (2^-14); the result's rounding
    sizes = torch.cat([w[i:i + step].double().norm(dim=1) for i in range(0, V, step)])
    terms = d.abs() * sizes
    own = torch.stack([labels, V - 100 - torch.arange(M, device="cuda")], 1)
    carried = terms.gather(1, own).sum(1)
    tol = U16 * (carried + terms.square().sum(1).sqrt() + dx.norm(dim=1)) + 2.0 ** -14 * terms.sum(1)
    off = (dX.double() - dx).norm(dim=1)
    assert bool((off <= tol).all()), (off, tol)
    for at in (0, 131072, 262144, 400000, 524288, V - 200):
        rows = slice(max(at - 200, 0), min(at + 200, V))
        dw, e = d[:, rows].t() @ xd, d[:, rows].abs().t() @ xd.abs()
        # dL rounded (U16), its exponent (2^-10), the result rounded
        ref.check(dW[rows], dw, U16 * dw.abs() + (U16 + 2.0 ** -10) * e + 1e-12, f"dw around word {at}")
    assert bool(torch.isfinite(dW.view(-1)[::4097].float()).all())


def test_gated_ffn():
    D, F = 64, 8192
    M = 2 ** 31 // F + 300
    x, dy = (torch.empty((M, D), dtype=BF16, device="cuda").normal_() for _ in range(2))
    wg, wu = ((torch.randn((D, F), device="cuda") * D ** -0.5).to(BF16) for _ in range(2))
    wd = (torch.randn((F, D), device="cuda") * F ** -0.5).to(BF16)
    Y, H, G, U = atb.atb_gated_ffn(x, wg, wu, wd, save=True)
    dX, dWg, dWu, dWd = atb.atb_gated_ffn_backward(dy, x, wg, wu, wd, H, G, U)
    atb.atb_device_status()
    xd, dyd, wgd, wud, wdd = (t.double() for t in (x, dy, wg, wu, wd))
    last = slice(M - 300, M)
    g, u = xd[last] @ wgd, xd[last] @ wud
    for got, want, b in ((G, g, wgd), (U, u, wud)):
        e = product_bound(xd[last], b)
        ref.check(got[last], want, e + U16 * (want.abs() + e), "g, u")
    y = H[last].double() @ wdd
    e = product_bound(H[last].double(), wdd)
    ref.check(Y[last], y, e + U16 * (y.abs() + e), "y")
    sums = [torch.zeros((D, F), dtype=torch.float64, device="cuda") for _ in range(2)] + [torch.zeros((F, D), dtype=torch.float64, device="cuda")]
    dx_last = None
    for i in range(0, M, 1 << 14):
        rows = slice(i, min(i + (1 << 14), M))
        a, slope = ref.act(G[rows].double(), "silu")
        dh = dyd[rows] @ wdd.t()
        dg, du = dh * U[rows].double() * slope, dh * a
        sums[0] += xd[rows].t() @ dg
        sums[1] += xd[rows].t() @ du
        sums[2] += H[rows].double().t() @ dyd[rows]
        dx_last = dg @ wgd.t() + du @ wud.t()
    # dg, du (or h) rounded and the result rounded, 2^-8 / sqrt(3) at most in the mean square each
    for got, want, name in zip((dWg, dWu, dWd, dX[-len(dx_last):]), (*sums, dx_last), ("dwg", "dwu", "dwd", "dx")):
        off = float((got.double() - want).norm() / want.norm())
        assert off <= U16, (name, off)

"""Offsets beyond 32 bits: matrices of more than 2^31 elements, checked at their far end."""
import pytest
import torch

import paper_2511_16041_b200 as atb
from tests import operators_ref as ref

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def _room(gigabytes):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gigabytes * 2 ** 30:
        pytest.skip("not enough free device memory")


@pytest.mark.parametrize("N", [8192, 8191])
def test_layer_norm(N):
    _room(24)
    M = 2 ** 31 // N + 1000
    x = torch.empty((M, N), dtype=BF16, device="cuda").normal_()
    w, b = torch.rand(N, device="cuda") + 0.5, torch.rand(N, device="cuda")
    Y, mean, rstd = atb.atb_layer_norm(x, w, b)
    dX, dW, dB = atb.atb_layer_norm_backward(x, x, w, mean, rstd)
    last = x[-300:].double()
    y, z, mu, r = ref.layer_norm(last, w.double(), b.double(), 1e-5)
    # one rounding to bf16, and 2^-16 for everything in FP32
    ref.check(Y[-300:], y, 2.0 ** -8 * y.abs() + 2.0 ** -16 * (y.abs() + z.abs() + 1), "y")
    dx = ref.layer_norm_backward(last, z, w.double(), r)[0]
    ref.check(dX[-300:], dx, 2.0 ** -8 * dx.abs() + 2.0 ** -14 * (dx.abs() + z.abs() + 1), "dx")
    # db: random signs; 2^31 / N terms of at most about 6
    want = torch.zeros(N, dtype=torch.float64, device="cuda")
    for i in range(0, M, 1 << 16):
        want += x[i:i + (1 << 16)].double().sum(0)
    ref.check(dB, want, torch.full_like(want, 2.0 ** -24 * M * 6), "db")
    del x, Y, dX
    torch.cuda.empty_cache()


def test_linear_cross_entropy():
    _room(24)
    M, D = 9, 4096
    V = 2 ** 31 // D + 3001
    x = torch.randn((M, D), device="cuda").to(BF16)
    w = torch.empty((V, D), dtype=BF16, device="cuda").normal_(std=2.0 / D ** 0.5)
    labels = V - 1 - torch.arange(M, device="cuda")
    loss, lse = atb.atb_linear_cross_entropy(x, w, labels)
    dX, dW = atb.atb_linear_cross_entropy_backward(torch.ones(M, device="cuda"), x, w, labels, lse)
    logits = torch.cat([x.double() @ w[i:i + (1 << 15)].double().t() for i in range(0, V, 1 << 15)], 1)
    want = torch.logsumexp(logits, 1)
    picked = logits.gather(1, labels[:, None])[:, 0]
    ref.check(lse, want, 1e-4 * want.abs(), "lse")
    ref.check(loss, want - picked, 1e-4 * (want.abs() + picked.abs()), "loss")
    d = torch.exp(logits[:, -2000:] - want[:, None])
    d[torch.arange(M), labels - (V - 2000)] -= 1
    dw = d.t() @ x.double()
    ref.check(dW[-2000:], dw, 2.0 ** -8 * dw.abs() + 2.0 ** -7 * (d.abs().t() @ x.double().abs()) + 1e-6, "dw")
    del w, dW
    torch.cuda.empty_cache()

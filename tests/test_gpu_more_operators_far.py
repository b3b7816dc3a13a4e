"""Matrices of more than 2^31 elements, checked at their far end: what the far rows get is what they get by themselves."""
import pytest
import torch

import paper_2511_16041_b200 as atb
from tests import operators_ref as ref
from tests.operators_ref import U16, product_bound

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
FAR = 2 ** 31


def far_rows(rows, cols, keep, dtype=BF16):
    """A matrix that is 0 but for its last `keep` rows, which are normal."""
    t = torch.zeros((rows, cols), dtype=dtype, device="cuda")
    t[-keep:] = torch.randn((keep, cols), device="cuda").to(dtype)
    return t


def test_linear():
    N, K, keep = 32768, 64, 130
    M = FAR // N + keep
    x, w, b = far_rows(M, K, keep), torch.randn((K, N), device="cuda").to(BF16), torch.randn(N, device="cuda")
    Y = atb.atb_linear(x, w, b, act="relu")
    assert torch.equal(Y[-keep:], atb.atb_linear(x[-keep:].contiguous(), w, b, act="relu"))
    dX, _, db = atb.atb_linear_backward(Y, x, w, dW=False)
    dy, wd = Y[-keep:].double(), w.double()
    want = dy @ wd.t()
    err = product_bound(dy, wd.t())
    ref.check(dX[-keep:], want, err + U16 * (want.abs() + err), "dx")
    want = dy.sum(0)                                           # all other rows of Y are the bias's
    want = want + (M - keep) * b.clamp(min=0).to(BF16).double()
    # FP32 sums of M terms, a rounding each
    ref.check(db, want, (M + 40) * 2.0 ** -24 * (dy.abs().sum(0) + (M - keep) * b.abs().double() * 1.01) + 1e-3, "db")
    del Y, dX
    torch.cuda.empty_cache()


def test_residual_norm():
    N, keep = 8192, 40
    M = FAR // N + keep
    x, f, w = far_rows(M, N, keep), far_rows(M, N, keep), torch.randn(N, device="cuda")
    H, Z, stats = atb.atb_residual_norm(x, f, w, gate=w, post_norm=True)
    near = [t[-keep:].contiguous() for t in (x, f)]
    h, z, s = atb.atb_residual_norm(*near, w, gate=w, post_norm=True)
    assert torch.equal(H[-keep:], h) and torch.equal(Z[-keep:], z) and torch.equal(stats[:, -keep:], s)
    dX, dF = atb.atb_residual_norm_backward(Z, H, x, f, stats, w, gate=w, post_norm=True)[:2]
    dx, df = atb.atb_residual_norm_backward(z, h, *near, s, w, gate=w, post_norm=True)[:2]
    assert torch.equal(dX[-keep:], dx) and torch.equal(dF[-keep:], df)
    del H, Z, dX, dF
    torch.cuda.empty_cache()


@pytest.mark.parametrize("V", [131072, 150001])
def test_sample(V):
    keep = 12
    M = FAR // V + keep
    x, u = far_rows(M, V, keep), torch.rand(M, device="cuda")
    for settings in (dict(top_k=20), dict(top_p=0.9), dict(temperature=0.0)):
        tokens, probs = atb.atb_sample(x, u, **settings)
        t, p = atb.atb_sample(x[-keep:].contiguous(), u[-keep:].contiguous(), **settings)
        assert torch.equal(tokens[-keep:], t) and torch.equal(probs[-keep:], p)
    del x
    torch.cuda.empty_cache()


def test_a_row_stride_beyond_32_bits():
    """Two rows that are 2^31 elements apart."""
    base = torch.zeros(FAR + 4096, dtype=BF16, device="cuda")
    rows = torch.as_strided(base, (2, 4096), (FAR, 1))
    rows.copy_(torch.randn((2, 4096), device="cuda"))
    near, u = rows.clone(), torch.rand(2, device="cuda")
    for a, b in zip(atb.atb_sample(rows, u, top_p=0.8), atb.atb_sample(near, u, top_p=0.8)):
        assert torch.equal(a, b)
    for a, b in zip(atb.atb_residual_norm(rows, rows), atb.atb_residual_norm(near, near)):
        assert torch.equal(a, b)
    w = torch.randn((64, 4096), device="cuda").to(BF16)
    assert torch.equal(atb.atb_linear(rows, w.t()), atb.atb_linear(near, w.t()))
    del base, rows
    torch.cuda.empty_cache()

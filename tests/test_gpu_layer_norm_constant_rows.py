"""Layer norm of rows whose elements are all one number: the mean is that number, x - mean and with it z are 0 exactly, whatever the
number, the width and the kernel that takes it."""
import pytest
import torch

import paper_2511_16041_b200 as atb

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
# Seven significant bits and at most 2^15 of them: every partial sum is exact in FP32, and so is the mean.
VALUES = [100.0, 1000.0, -0.8984375, 6016.0, 3.0, 2.0 ** -20, 1.5 * 2.0 ** 60]
WIDTHS = [1, 5, 40, 257, 513, 520, 1000, 1001, 3000, 4096, 6000, 9001, 16384, 16385, 20000]


def _rows(N, dtype):
    return torch.tensor(VALUES, device="cuda")[:, None].expand(-1, N).to(dtype).contiguous()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N", WIDTHS)
def test_forward_and_backward(N, dtype):
    x = _rows(N, dtype)
    gen = torch.Generator(device="cuda").manual_seed(N)
    w, b = (torch.randn(N, generator=gen, device="cuda") for _ in range(2))
    Y, mean, rstd = atb.atb_layer_norm(x, w, b)
    assert torch.equal(mean, torch.tensor(VALUES, device="cuda"))
    assert torch.equal(Y, b.to(dtype).expand_as(Y))
    dy = torch.randn(x.shape, generator=gen, device="cuda").to(dtype)
    dX, dW, dB = atb.atb_layer_norm_backward(dy, x, w, mean, rstd)
    assert bool((dW == 0).all()) and bool(torch.isfinite(dX).all())


@pytest.mark.parametrize("N", [8, 520, 4096, 6000, 16392])
def test_bfp16_planes(N):
    x = _rows(N, F32)
    b = torch.randn(N, device="cuda")
    mant, exp, mean, _ = atb.atb_layer_norm_bfp16(x, None, b)
    want_mant, want_exp = atb.atb_quantize_bfp16(b.expand(len(VALUES), N).contiguous())
    assert torch.equal(mean, torch.tensor(VALUES, device="cuda"))
    assert torch.equal(mant, want_mant) and torch.equal(exp, want_exp)

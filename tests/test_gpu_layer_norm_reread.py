"""Layer norm backward where a row is read from shared memory twice and its stage is filled again at once (768 and 1024 threads
per row): widths whose last warp has part of a warp's pieces, rows enough for every block to walk several."""
import pytest
import torch

import paper_2511_16041_b200 as atb
from tests import operators_ref as ref
from tests.operators_ref import U16, U32
from tests.test_gpu_layer_norm import BF16, F32, _inputs, _z_error

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,N,pad", [(F32, 8200, 0), (F32, 8712, 8), (F32, 10248, 0), (F32, 12280, 0), (F32, 12288, 8), (F32, 8201, 0), (F32, 12288, 3),
                                         (BF16, 8200, 0), (BF16, 12280, 8), (BF16, 16376, 0), (BF16, 12301, 0)])
def test_backward(dtype, N, pad):
    M = 900
    x, dy, w, b = _inputs(M, N, dtype, F32, pad)
    _, mean, rstd = atb.atb_layer_norm(x, w, b)
    dX, dW, dB = atb.atb_layer_norm_backward(dy, x, w, mean, rstd)
    xd, dyd, wd = x.double(), dy.double(), w.double()
    _, z, _, r = ref.layer_norm(xd, wd, None, 1e-5)
    dx, dw, db, g = ref.layer_norm_backward(dyd, z, wd, r)
    ze = _z_error(xd, z, r)
    # the bounds of test_gpu_layer_norm.py
    gz, ga = (g * z).abs().mean(1, keepdim=True), g.abs().mean(1, keepdim=True)
    t = r * (200 * U32 * (g.abs() + ga + z.abs() * gz) + ze * gz + z.abs() * (g.abs() * ze).mean(1, keepdim=True))
    ref.check(dX, dx, t + (U16 * (dx.abs() + t) if dtype == BF16 else 0), "dx")
    ref.check(dW, dw, (dyd.abs() * ze).sum(0) + (M + 16) * U32 * (dyd * z).abs().sum(0), "dw")
    ref.check(dB, db, (M + 16) * U32 * dyd.abs().sum(0), "db")
    again = atb.atb_layer_norm_backward(dy, x, w, mean, rstd)
    for a, c in zip((dX, dW, dB), again):
        assert torch.equal(a, c)

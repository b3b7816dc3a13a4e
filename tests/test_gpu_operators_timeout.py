"""The timeout path of the BF16 product kernels, in the form that cannot hang a GPU (see test_gpu_timeout.py): the diagnostic build,
whose waits give up after 2 ms, has one epilogue warp of CTA 0 keep back its first arrival; the issuer then waits, at the
CTA's third tile, for an accumulator that nobody frees, and gives up.  No copy and no UMMA depends on the arrival."""
import ctypes

import pytest
import torch

import paper_2511_16041_b200 as atb
from paper_2511_16041_b200 import _build

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,V,D", [(64, 128 * 148 * 3, 64),          # single CTAs: three 128 x 128 tiles each
                                   (256, 256 * 74 * 3, 64)])         # CTA pairs: three 256 x 256 tiles each
def test_a_wait_that_runs_out_is_reported_and_the_context_stays_usable(M, V, D):
    lib = ctypes.CDLL(_build.build_library(variant="timeout_test"))
    plain = atb.load_library()
    for name in ("atb_linear_cross_entropy", "atb_linear_cross_entropy_workspace_bytes", "atb_device_status", "atb_last_error_message"):
        getattr(lib, name).restype, getattr(lib, name).argtypes = getattr(plain, name).restype, getattr(plain, name).argtypes
    x, w = torch.randn(M, D, device="cuda").to(torch.bfloat16), torch.randn(V, D, device="cuda").to(torch.bfloat16)
    labels = torch.randint(0, V, (M,), device="cuda")
    loss, lse = torch.zeros(M, device="cuda"), torch.zeros(M, device="cuda")
    need = lib.atb_linear_cross_entropy_workspace_bytes(M, V, D)
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert lib.atb_device_status(stream) == atb.ATB_OK
    assert lib.atb_linear_cross_entropy(M, V, D, x.data_ptr(), D, w.data_ptr(), D, labels.data_ptr(), -100, loss.data_ptr(), lse.data_ptr(), ws.data_ptr(),
                                        need, stream) == atb.ATB_OK
    assert lib.atb_device_status(stream) == 8, lib.atb_last_error_message()
    assert b"BF16 product" in lib.atb_last_error_message()
    assert lib.atb_device_status(stream) == atb.ATB_OK               # reading the flag cleared it
    torch.cuda.synchronize()
    # the product build on the same context: tensor memory that was released is allocatable again
    got, _ = atb.atb_linear_cross_entropy(x, w, labels)
    atb.atb_device_status()
    want = torch.nn.functional.cross_entropy(x.double() @ w.double().t(), labels, reduction="none")
    assert float((got.double() - want).abs().max()) <= 1e-4 * float(want.abs().max())

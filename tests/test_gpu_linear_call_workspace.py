"""The linear layer's backward pass in a workspace of exactly what the call takes: the same results, nothing behind it written, and no more allocated."""
import pytest
import torch

import paper_2511_16041_b200 as atb

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("wanted", [(1, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 0)])
@pytest.mark.parametrize("act,y_type", [(None, BF16), (None, F32), ("gelu", BF16)])
@pytest.mark.parametrize("M,K,N", [(1, 64, 72), (5, 4104, 264), (300, 264, 4104), (700, 4104, 264)])
def test_exactly_what_a_call_takes(M, K, N, act, y_type, wanted, transposed):
    gen = torch.Generator(device="cuda").manual_seed(M)
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    x, dy = normal(M, K).to(BF16), normal(M, N).to(y_type)
    w = normal(N, K).to(BF16).t() if transposed else normal(K, N).to(BF16)
    Z = normal(M, N) if act else None
    full = atb.atb_linear_backward(dy, x, w, Z, act=act, workspace=torch.empty(atb.atb_linear_backward_workspace_bytes(M, K, N), dtype=torch.uint8, device="cuda"))
    need = atb.atb_linear_backward_call_workspace_bytes(M, K, N, act, int(y_type == BF16), int(transposed), *wanted)
    ws = torch.full((need + 4096,), 171, dtype=torch.uint8, device="cuda")
    kw = {name: None if on else False for name, on in zip(("dX", "dW", "dbias"), wanted)}
    got = atb.atb_linear_backward(dy, x, w, Z, act=act, workspace=ws[:need], **kw)
    assert bool((ws[need:] == 171).all())
    both = wanted[0] and wanted[1]
    for i, (g, f) in enumerate(zip(got, full)):
        assert (g is not None) == bool(wanted[i])
        if g is not None and (both or i == 2):                # one product alone may be split otherwise than two
            assert torch.equal(g, f)
        elif g is not None:
            assert float((g.double() - f.double()).norm()) <= 2.0 ** -8 * float(f.double().norm())
    if need > 0:
        with pytest.raises(atb.AtbError) as e:
            atb.atb_linear_backward(dy, x, w, Z, act=act, workspace=ws[:need - 1], **kw)
        assert e.value.status == 7


def test_a_projection_without_an_activation_allocates_its_results():
    M, K, N = 8192, 1024, 10944
    x, w, dy = (torch.randn(s, device="cuda").to(BF16) for s in ((M, K), (K, N), (M, N)))
    dX, dW = torch.empty_like(x), torch.empty_like(w)
    for dbias, most in ((False, 0), (None, 4 * 600 * N)):
        atb.atb_linear_backward(dy, x, w, dX=dX, dW=dW, dbias=dbias)
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        atb.atb_linear_backward(dy, x, w, dX=dX, dW=dW, dbias=dbias)
        assert torch.cuda.max_memory_allocated() - before <= most

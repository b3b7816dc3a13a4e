"""The GEMM's and the quantiser's calls with ``stream=``: results and workspaces come from that stream's memory, not from blocks that
the current stream has given up and still has to read."""
import pytest
import torch

import paper_2511_16041_b200 as atb

pytestmark = pytest.mark.gpu

M, N, K = 2048, 2048, 1024
NAMES = ["quantize", "gemm", "splitk", "bfp16_out", "config1", "config2"]


def _call(name):
    a = torch.randn(M, K, device="cuda")
    b = torch.randn(K, N, device="cuda")
    mant, exp = atb.atb_quantize_bfp16(a)
    bt_mant, bt_exp = atb.atb_quantize_bfp16(b.t().contiguous())
    a16, b16 = a.to(torch.bfloat16), b.to(torch.bfloat16)
    return {
        "quantize": lambda s: atb.atb_quantize_bfp16(a, stream=s),
        "gemm": lambda s: (atb.atb_gemm(M, N, K, 128, 128, 64, 128, mant, exp, b16, stream=s),),
        "splitk": lambda s: (atb.atb_gemm_splitk(M, N, K, 128, 128, 64, 128, mant, exp, b16, 2, stream=s),),
        "bfp16_out": lambda s: atb.atb_gemm_bfp16_out(M, N, K, 128, 256, 64, 128, mant, exp, b16, stream=s),
        "config1": lambda s: (atb.atb_gemm_config(1, M, N, K, a16, None, bt_mant, bt_exp, stream=s),),
        "config2": lambda s: atb.atb_gemm_config(2, M, N, K, mant, exp, bt_mant, bt_exp, stream=s)}[name]


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("name", NAMES)
def test_a_freed_block_that_is_still_read(name, raw):
    call, side = _call(name), torch.cuda.Stream()
    want = call(None)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    held = [torch.full((64 << 20,), 5, dtype=torch.uint8, device="cuda") for _ in range(4)]
    seen = [torch.empty_like(h) for h in held]
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)                             # about 50 ms
    for h, s in zip(held, seen):
        s.copy_(h)
    del held, h
    got = call(side.cuda_stream if raw else side)
    torch.cuda.synchronize()
    atb.atb_device_status()
    assert all(bool((s == 5).all()) for s in seen)
    for p, q in zip(got, want):
        assert torch.equal(p, q)


def test_the_names_of_the_default_stream():
    a = torch.randn(300, 512, device="cuda")
    want = atb.atb_quantize_bfp16(a)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        for handle in (0, 1, 2):
            got = atb.atb_quantize_bfp16(a, stream=handle)
            torch.cuda.synchronize()
            for p, q in zip(got, want):
                assert torch.equal(p, q)

"""Calls with ``stream=``: what they allocate comes from that stream's memory, so that a block which the current stream has given
up but still has to read, or still has to write, is not handed to kernels that do not wait for it."""
import pytest
import torch

import paper_2511_16041_b200 as atb

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
M, D, F, V = 2048, 1024, 2048, 4096


def _t(*shape, dtype=BF16):
    return torch.randn(shape, device="cuda").to(dtype)


def _calls():
    """name -> call(stream); each makes results or a workspace of several megabytes."""
    x, wg, wu, wd, dy, head, w = _t(M, D), _t(D, F), _t(D, F), _t(F, D), _t(M, D), _t(V, D), _t(D)
    labels, dloss = torch.randint(0, V, (M,), device="cuda"), torch.rand(M, device="cuda")
    _, mean, rstd = atb.atb_layer_norm(x, w, w)
    _, H, G, U = atb.atb_gated_ffn(x, wg, wu, wd, save=True)
    _, lse = atb.atb_linear_cross_entropy(x, head, labels)
    return {
        "norm": lambda s: atb.atb_layer_norm(x, w, w, stream=s),
        "norm_bfp16": lambda s: atb.atb_layer_norm_bfp16(x, w, w, stream=s),
        "norm_backward": lambda s: atb.atb_layer_norm_backward(dy, x, w, mean, rstd, stream=s),
        "ffn": lambda s: atb.atb_gated_ffn(x, wg, wu, wd, save=True, stream=s),
        "ffn_backward": lambda s: atb.atb_gated_ffn_backward(dy, x, wg, wu, wd, H, G, U, stream=s),
        "head_backward": lambda s: atb.atb_linear_cross_entropy_backward(dloss, x, head, labels, lse, stream=s)}


NAMES = ["norm", "norm_bfp16", "norm_backward", "ffn", "ffn_backward", "head_backward"]


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("name", NAMES)
def test_a_freed_block_that_is_still_read(name, raw):
    call, side = _calls()[name], torch.cuda.Stream()
    want = call(None)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    # blocks that any of the call's tensors would fit, freed while a delayed reader is queued
    held = [torch.full((64 << 20,), 5, dtype=torch.uint8, device="cuda") for _ in range(8)]
    seen = [torch.empty_like(h) for h in held]
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)                             # about 50 ms
    for h, s in zip(held, seen):
        s.copy_(h)
    del held, h
    got = call(side.cuda_stream if raw else side)
    torch.cuda.synchronize()
    assert all(bool((s == 5).all()) for s in seen)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("name", NAMES)
def test_a_freed_block_that_is_still_written(name):
    call, side = _calls()[name], torch.cuda.Stream()
    want = call(None)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    held = [torch.empty(64 << 20, dtype=torch.uint8, device="cuda") for _ in range(8)]
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)
    for h in held:
        h.fill_(255)
    del held, h
    got = call(side)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_results_freed_while_the_current_stream_reads_them():
    """The other end: a result dropped on the host while the current stream still has to read it is not handed to the next call."""
    x, other, w, side = _t(M, D), _t(M, D), _t(D), torch.cuda.Stream()
    want = atb.atb_layer_norm(x, w, w)[0]
    torch.cuda.synchronize()
    Y = atb.atb_layer_norm(x, w, w, stream=side)[0]
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(100_000_000)
    seen = Y.clone()
    del Y
    for _ in range(4):
        atb.atb_layer_norm(other, w, w, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(seen, want)


def test_the_names_of_the_default_stream():
    x, w = _t(300, 512), _t(512)
    want = atb.atb_layer_norm(x, w, w)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        for handle in (0, 1, 2):                               # default, legacy default and per-thread default
            got = atb.atb_layer_norm(x, w, w, stream=handle)
            torch.cuda.synchronize()
            for a, b in zip(got, want):
                assert torch.equal(a, b)

"""Refusals of the linear layer's entry points: checked on the host before anything is launched, so they need no GPU."""
import pytest
import torch

import paper_2511_16041_b200 as atb

P = 1 << 20                                                   # an aligned address that nothing reads
NULL, SHAPE, MISALIGNED, SMALL, ARGUMENT = 1, 2, 4, 7, 9


@pytest.mark.parametrize("layout", [0, 1])
def test_forward_refusals(layout):
    lib = atb.load_library()
    M, K, N = 4, 64, 136
    need = lib.atb_linear_workspace_bytes(M, K, N)
    assert atb.atb_linear_workspace_bytes(M, K, N) == need
    ok = dict(M=M, K=K, N=N, act=4, yt=1, x=P, ldx=K, layout=layout, w=P, ldw=K if layout else N, bt=0, b=P, r=P, ldr=N, y=P, ldy=N, zt=0, z=P, ws=P, n=need, stream=None)
    call = lambda **k: lib.atb_linear(*{**ok, **k}.values())
    assert call(act=5) == ARGUMENT and call(act=-1) == ARGUMENT and call(act=256) == ARGUMENT
    assert call(yt=2) == ARGUMENT and call(zt=-1) == ARGUMENT and call(bt=3) == ARGUMENT and call(layout=2) == ARGUMENT
    assert call(M=-1) == SHAPE and call(K=60) == SHAPE and call(K=0) == SHAPE and call(N=132) == SHAPE and call(N=0) == SHAPE and call(M=(1 << 30) + 1) == SHAPE
    for name in ("x", "w", "y"):
        assert call(**{name: None}) == NULL, name
    for name in ("x", "w", "b", "r", "y", "z", "ws"):
        assert call(**{name: P + 8}) == MISALIGNED, name
    for name in ("ldx", "ldw", "ldr", "ldy"):
        assert call(**{name: 56}) == SHAPE and call(**{name: 140}) == SHAPE, name
    assert call(yt=0, ldy=138) == SHAPE and call(yt=0, ldr=138) == SHAPE
    assert call(M=0, x=None) == 0
    if need:
        assert call(n=need - 1) == SMALL and call(ws=None) == NULL


@pytest.mark.parametrize("layout", [0, 1])
def test_backward_refusals(layout):
    lib = atb.load_library()
    M, K, N = 4, 64, 136
    need = lib.atb_linear_backward_workspace_bytes(M, K, N)
    assert need >= 2 * M * N and atb.atb_linear_backward_workspace_bytes(M, K, N) == need and lib.atb_linear_backward_workspace_bytes(0, K, N) == 0
    lw = K if layout else N
    ok = dict(M=M, K=K, N=N, act=0, yt=1, dy=P, lddy=N, x=P, ldx=K, layout=layout, w=P, ldw=lw, zt=0, z=P, dx=P, lddx=K, dw=P, lddw=lw, bt=0, db=P, ws=P, n=need, stream=None)
    call = lambda **k: lib.atb_linear_backward(*{**ok, **k}.values())
    assert call(act=5) == ARGUMENT and call(yt=9) == ARGUMENT and call(layout=-1) == ARGUMENT and call(M=-1) == SHAPE and call(K=12) == SHAPE
    for name in ("dy", "x", "w", "z", "ws"):
        assert call(**{name: None}) == NULL, name
    for name in ("dy", "x", "w", "z", "dx", "dw", "db", "ws"):
        assert call(**{name: P + 2}) == MISALIGNED, name
    for name in ("lddy", "ldx", "ldw", "lddx", "lddw"):
        assert call(**{name: 56}) == SHAPE and call(**{name: 140}) == SHAPE, name
    assert call(n=0) == SMALL


@pytest.mark.parametrize("act,error", [("swish", ValueError), ("", ValueError), ("RELU", ValueError), (0.5, TypeError), ([0], TypeError)])
def test_names_of_activations(act, error):
    x, w = torch.ones(4, 16, dtype=torch.bfloat16), torch.ones(16, 24, dtype=torch.bfloat16)
    with pytest.raises(error):
        atb.atb_linear(x, w, act=act)
    with pytest.raises(error):
        atb.atb_linear_backward(x, x, w, act=act)


def test_tensors_that_are_not_on_a_gpu():
    x, w = torch.ones(4, 16, dtype=torch.bfloat16), torch.ones(16, 24, dtype=torch.bfloat16)
    for call in (lambda: atb.atb_linear(x, w), lambda: atb.atb_linear(None, w), lambda: atb.atb_linear(x, 3), lambda: atb.atb_linear_backward(x, x, w)):
        with pytest.raises(ValueError):
            call()

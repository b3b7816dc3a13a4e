"""Refusals of the layer norm, gated feed-forward and linear cross entropy entry points: checked on the host before
anything is launched, so they need no GPU (pointers are never followed)."""
import pytest
import torch

import paper_2511_16041_b200 as atb

P = 1 << 20                                                   # an aligned address that nothing reads
NULL, SHAPE, MISALIGNED, SMALL, ARGUMENT = 1, 2, 4, 7, 9


def test_status_name():
    assert atb.atb_status_string(ARGUMENT) == "ATB_ERR_BAD_ARGUMENT"


def test_layer_norm_refusals():
    f = atb.load_library().atb_layer_norm
    ok = dict(M=4, N=64, xt=1, x=P, ldx=64, wt=0, w=P, b=P, eps=1e-5, y=P, ldy=64, mean=P, rstd=P, stream=None)
    call = lambda **k: f(*{**ok, **k}.values())
    assert call(xt=2) == ARGUMENT and call(wt=-1) == ARGUMENT
    assert call(eps=-1.0) == ARGUMENT and call(eps=float("nan")) == ARGUMENT
    assert call(M=-1) == SHAPE and call(N=-1) == SHAPE and call(M=1 << 31) == SHAPE
    assert call(ldx=63) == SHAPE and call(ldy=63) == SHAPE
    assert call(x=None) == NULL and call(y=None) == NULL
    assert call(x=P + 1) == MISALIGNED and call(w=P + 2) == MISALIGNED and call(mean=P + 2) == MISALIGNED
    assert call(M=0, x=None, y=None) == 0 and call(N=0) == 0


def test_layer_norm_bfp16_refusals():
    f = atb.load_library().atb_layer_norm_bfp16
    ok = dict(M=4, N=64, xt=1, x=P, ldx=64, wt=0, w=P, b=P, eps=1e-5, mant=P, exp=P, mean=P, rstd=P, stream=None)
    call = lambda **k: f(*{**ok, **k}.values())
    assert call(N=60) == SHAPE and call(exp=None) == NULL and call(mant=None) == NULL
    assert call(ldx=68) == MISALIGNED and call(x=P + 2) == MISALIGNED and call(w=P + 4) == MISALIGNED and call(mant=P + 8) == MISALIGNED
    assert call(M=0, exp=None) == 0


def test_layer_norm_backward_refusals():
    lib = atb.load_library()
    need = lib.atb_layer_norm_backward_workspace_bytes(4, 64)
    assert need > 0 and atb.atb_layer_norm_backward_workspace_bytes(4, 64) == need
    f = lib.atb_layer_norm_backward
    ok = dict(M=4, N=64, xt=1, dy=P, lddy=64, x=P, ldx=64, wt=0, w=P, mean=P, rstd=P, dx=P, lddx=64, dw=P, db=P, ws=P, n=need, stream=None)
    call = lambda **k: f(*{**ok, **k}.values())
    assert call(xt=7) == ARGUMENT and call(M=-1) == SHAPE
    assert call(dy=None) == NULL and call(x=None) == NULL and call(mean=None) == NULL and call(rstd=None) == NULL and call(ws=None) == NULL
    assert call(lddy=8) == SHAPE and call(ldx=8) == SHAPE and call(lddx=8) == SHAPE
    assert call(dx=P + 1) == MISALIGNED and call(ws=P + 8) == MISALIGNED
    assert call(n=need - 1) == SMALL


def test_gated_ffn_refusals():
    lib = atb.load_library()
    M, D, F = 4, 64, 136
    need = lib.atb_gated_ffn_workspace_bytes(M, D, F)
    assert atb.atb_gated_ffn_workspace_bytes(M, D, F) == need
    ok = dict(M=M, D=D, F=F, act=0, x=P, ldx=D, wg=P, wu=P, ldw=F, wd=P, ldwd=D, y=P, ldy=D, h=P, g=P, u=P, ws=P, n=need, stream=None)
    call = lambda **k: lib.atb_gated_ffn(*{**ok, **k}.values())
    assert call(act=3) == ARGUMENT and call(act=-1) == ARGUMENT
    assert call(M=-1) == SHAPE and call(D=60) == SHAPE and call(F=0) == SHAPE and call(F=132) == SHAPE and call(M=(1 << 30) + 1) == SHAPE
    for name in ("x", "wg", "wu", "wd", "y", "h", "g", "u"):
        assert call(**{name: None}) == NULL, name
        assert call(**{name: P + 8}) == MISALIGNED, name
    for name in ("ldx", "ldw", "ldwd", "ldy"):
        assert call(**{name: 56}) == SHAPE and call(**{name: 140}) == SHAPE, name
    assert call(M=0, x=None) == 0
    if need:
        assert call(n=need - 1) == SMALL and call(ws=None) == NULL


def test_gated_ffn_backward_refusals():
    lib = atb.load_library()
    M, D, F = 4, 64, 136
    need = lib.atb_gated_ffn_backward_workspace_bytes(M, D, F)
    assert need >= 4 * M * F and atb.atb_gated_ffn_backward_workspace_bytes(M, D, F) == need
    ok = dict(M=M, D=D, F=F, act=0, dy=P, lddy=D, x=P, ldx=D, wg=P, wu=P, ldw=F, wd=P, ldwd=D, h=P, g=P, u=P, dx=P, lddx=D, dwg=P, dwu=P, lddw=F,
              dwd=P, lddwd=D, ws=P, n=need, stream=None)
    call = lambda **k: lib.atb_gated_ffn_backward(*{**ok, **k}.values())
    assert call(act=9) == ARGUMENT and call(M=-1) == SHAPE and call(D=12) == SHAPE
    for name in ("dy", "x", "wg", "wu", "wd", "h", "g", "u", "dwg", "dwu", "ws"):
        assert call(**{name: None}) == NULL, name
        assert call(**{name: P + 2}) == MISALIGNED, name
    for name in ("lddy", "ldx", "ldw", "ldwd", "lddx", "lddw", "lddwd"):
        assert call(**{name: 56}) == SHAPE and call(**{name: 140}) == SHAPE, name
    assert call(n=need - 1) == SMALL


def test_linear_cross_entropy_refusals():
    lib = atb.load_library()
    M, V, D = 4, 1000, 64
    need = lib.atb_linear_cross_entropy_workspace_bytes(M, V, D)
    assert need > 0 and atb.atb_linear_cross_entropy_workspace_bytes(M, V, D) == need
    ok = dict(M=M, V=V, D=D, x=P, ldx=D, w=P, ldw=D, labels=P, ignore=-100, loss=P, lse=P, ws=P, n=need, stream=None)
    call = lambda **k: lib.atb_linear_cross_entropy(*{**ok, **k}.values())
    assert call(M=-1) == SHAPE and call(V=0) == SHAPE and call(D=60) == SHAPE and call(D=0) == SHAPE
    assert call(ldx=56) == SHAPE and call(ldw=68) == SHAPE
    for name in ("x", "w", "labels", "loss", "lse", "ws"):
        assert call(**{name: None}) == NULL, name
        assert call(**{name: P + 2}) == MISALIGNED, name
    assert call(n=need - 1) == SMALL and call(M=0, x=None) == 0


def test_linear_cross_entropy_backward_refusals():
    lib = atb.load_library()
    M, V, D = 4, 5000, 64
    need = lib.atb_linear_cross_entropy_backward_workspace_bytes(M, V, D, 0)
    assert atb.atb_linear_cross_entropy_backward_workspace_bytes(M, V, D) == need
    assert lib.atb_linear_cross_entropy_backward_workspace_bytes(M, V, D, 256) < need
    ok = dict(M=M, V=V, D=D, x=P, ldx=D, w=P, ldw=D, labels=P, ignore=-100, lse=P, dloss=P, dx=P, lddx=D, dw=P, lddw=D, piece=0, ws=P, n=need,
              stream=None)
    call = lambda **k: lib.atb_linear_cross_entropy_backward(*{**ok, **k}.values())
    assert call(M=-1) == SHAPE and call(V=0) == SHAPE and call(D=4) == SHAPE and call(piece=-1) == ARGUMENT
    for name in ("ldx", "ldw", "lddx", "lddw"):
        assert call(**{name: 56}) == SHAPE and call(**{name: 68}) == SHAPE, name
    for name in ("x", "w", "labels", "lse", "dloss", "ws"):
        assert call(**{name: None}) == NULL, name
        assert call(**{name: P + 2}) == MISALIGNED, name
    assert call(n=need - 1) == SMALL


def test_the_binding_refuses_tensors_that_are_not_on_a_gpu():
    x, v, l = torch.zeros(4, 16), torch.zeros(16), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: atb.atb_layer_norm(x, v, v), lambda: atb.atb_layer_norm_bfp16(x, v, v), lambda: atb.atb_layer_norm(None),
                 lambda: atb.atb_layer_norm_backward(x, x, v, v[:4], v[:4]), lambda: atb.atb_gated_ffn(x, x, x, x),
                 lambda: atb.atb_gated_ffn_backward(x, x, x, x, x, x, x, x), lambda: atb.atb_linear_cross_entropy(x, x, l),
                 lambda: atb.atb_linear_cross_entropy_backward(v, x, x, l, v), lambda: atb.atb_layer_norm(3), lambda: atb.atb_layer_norm(v)):
        with pytest.raises(ValueError):
            call()

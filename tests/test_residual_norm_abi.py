"""Refusals of the residual norm's entry points: checked on the host before anything is launched, so they need no GPU."""
import pytest
import torch

import paper_2511_16041_b200 as atb

P = 1 << 20                                                   # an aligned address that nothing reads
NULL, SHAPE, MISALIGNED, SMALL, ARGUMENT = 1, 2, 4, 7, 9


def test_forward_refusals():
    f = atb.load_library().atb_residual_norm
    ok = dict(M=4, N=64, kind=2, xt=0, x=P, ldx=64, ft=1, f=P, ldf=64, scale=1.0, wt=0, gate=P, pw=P, pb=P, w=P, b=P, eps=1e-5, h=P, ldh=64, z=P, ldz=64, stats=P, stream=None)
    call = lambda **k: f(*{**ok, **k}.values())
    assert call(kind=4) == ARGUMENT and call(kind=-1) == ARGUMENT and call(kind=0) == ARGUMENT and call(kind=1, pw=None) == ARGUMENT
    assert call(xt=2) == ARGUMENT and call(ft=-1) == ARGUMENT and call(wt=5) == ARGUMENT and call(xt=1, ft=0) == ARGUMENT
    assert call(eps=-1.0) == ARGUMENT and call(eps=float("nan")) == ARGUMENT
    assert call(M=-1) == SHAPE and call(N=-1) == SHAPE and call(M=1 << 31) == SHAPE
    for name in ("ldx", "ldf", "ldh", "ldz"):
        assert call(**{name: 63}) == SHAPE, name
    for name in ("x", "f", "h", "z"):
        assert call(**{name: None}) == NULL, name
    for name in ("x", "f", "h", "z", "gate", "pw", "pb", "w", "b", "stats"):
        assert call(**{name: P + 1}) == MISALIGNED, name
    assert call(x=P + 2) == MISALIGNED and call(gate=P + 2) == MISALIGNED
    assert call(M=0, x=None) == 0 and call(N=0) == 0


def test_backward_refusals():
    lib = atb.load_library()
    need = lib.atb_residual_norm_backward_workspace_bytes(4, 64)
    assert need > 0 and atb.atb_residual_norm_backward_workspace_bytes(4, 64) == need and lib.atb_residual_norm_backward_workspace_bytes(0, 64) == 0
    f = lib.atb_residual_norm_backward
    ok = dict(M=4, N=64, kind=3, xt=0, dz=P, lddz=64, dh=P, lddh=64, x=P, ldx=64, ft=1, f=P, ldf=64, scale=1.0, wt=0, gate=P, pw=P, pb=P, w=P, stats=P, dx=P, lddx=64, df=P,
              lddf=64, dgate=P, dpw=P, dpb=P, dw=P, db=P, ws=P, n=need, stream=None)
    call = lambda **k: f(*{**ok, **k}.values())
    assert call(kind=8) == ARGUMENT and call(kind=1) == ARGUMENT and call(xt=1, ft=0) == ARGUMENT and call(M=-1) == SHAPE
    assert call(kind=0, pw=None, pb=None, dpb=None) == ARGUMENT
    for name in ("dz", "x", "f", "stats", "ws"):
        assert call(**{name: None}) == NULL, name
    for name in ("lddz", "lddh", "ldx", "ldf", "lddx", "lddf"):
        assert call(**{name: 8}) == SHAPE, name
    for name in ("dz", "dh", "x", "f", "gate", "pw", "pb", "w", "stats", "dx", "df", "dgate", "dpw", "dpb", "dw", "db", "ws"):
        assert call(**{name: P + 1}) == MISALIGNED, name
    assert call(ws=P + 8) == MISALIGNED and call(n=need - 1) == SMALL


def test_the_binding():
    x = torch.zeros(4, 16)
    for call in (lambda: atb.atb_residual_norm(x, x), lambda: atb.atb_residual_norm(None, x), lambda: atb.atb_residual_norm_backward(x, x, x, x, x)):
        with pytest.raises(ValueError):
            call()
    for kind in ("l2", 0, None):
        with pytest.raises(ValueError, match="kind="):
            atb.atb_residual_norm(x, x, kind=kind)

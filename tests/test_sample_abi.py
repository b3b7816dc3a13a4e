"""Refusals of atb_sample: checked on the host before anything is launched, so they need no GPU."""
import pytest
import torch

import paper_2511_16041_b200 as atb

P = 1 << 20                                                   # an aligned address that nothing reads
NULL, SHAPE, MISALIGNED, ARGUMENT = 1, 2, 4, 9


def test_refusals():
    f = atb.load_library().atb_sample
    ok = dict(M=4, V=100, type=0, x=P, ld=100, ut=0, u=P, t=1.0, tp=None, k=0, kp=None, p=1.0, pp=None, m=0.0, mp=None, tokens=P, probs=P, stream=None)
    call = lambda **k: f(*{**ok, **k}.values())
    nan = float("nan")
    assert call(type=2) == ARGUMENT and call(type=-1) == ARGUMENT and call(ut=1) == ARGUMENT and call(ut=3) == ARGUMENT
    assert call(t=-0.5) == ARGUMENT and call(t=nan) == ARGUMENT and call(p=nan) == ARGUMENT and call(m=nan) == ARGUMENT
    assert call(M=-1) == SHAPE and call(V=0) == SHAPE and call(V=(1 << 30) + 1) == SHAPE and call(M=(1 << 27) + 1) == SHAPE and call(ld=99) == SHAPE
    for name in ("x", "u", "tokens"):
        assert call(**{name: None}) == NULL, name
    for name in ("x", "u", "tp", "kp", "pp", "mp", "tokens", "probs"):
        assert call(**{name: P + 1}) == MISALIGNED, name
    assert call(x=P + 2) == MISALIGNED and call(ut=2, u=P + 4) == MISALIGNED and call(tokens=P + 4) == MISALIGNED
    assert call(M=0, x=None) == 0


def test_the_binding():
    x, u = torch.zeros(4, 16), torch.zeros(4)
    for call in (lambda: atb.atb_sample(x, u), lambda: atb.atb_sample(None, u), lambda: atb.atb_sample(x[0], u)):
        with pytest.raises(ValueError):
            call()
    for bad in (dict(temperature="1"), dict(top_k=2.5), dict(top_p=None), dict(min_p=[0.1])):
        with pytest.raises(TypeError):
            atb.atb_sample(x, u, **bad)

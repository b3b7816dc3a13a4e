"""Scalar arguments of the operators: what is no activation is refused and not taken for one."""
import pytest
import torch

import paper_2511_16041_b200 as atb


def _block(device="cpu"):
    t = lambda *s: torch.ones(s, dtype=torch.bfloat16, device=device)  # noqa: E731
    return t(4, 16), t(16, 24), t(16, 24), t(24, 16)


@pytest.mark.parametrize("act,error", [("relu", ValueError), ("0", ValueError), ("SILU", ValueError), (0.5, TypeError), (None, TypeError), ([0], TypeError),
                                       (torch.tensor([0, 1]), TypeError)])
def test_names_of_activations(act, error):
    with pytest.raises(error, match="act=" if error is ValueError else None):
        atb.atb_gated_ffn(*_block(), act=act)
    x, wg, wu, wd = _block()
    with pytest.raises(error, match="act=" if error is ValueError else None):
        atb.atb_gated_ffn_backward(x, x, wg, wu, wd, wg, wg, wg, act=act)


def test_truth_without_a_value():
    with pytest.raises(RuntimeError, match="Boolean value"):
        atb.atb_gated_ffn(*_block(), save=torch.ones(2))


@pytest.mark.gpu
@pytest.mark.parametrize("act", [3, -1, 1 << 32, (1 << 32) + 1, -(1 << 32), 1 << 62])
def test_numbers_of_activations(act):
    x, wg, wu, wd = _block("cuda")
    _, H, G, U = atb.atb_gated_ffn(x, wg, wu, wd, save=True)
    for call in (lambda: atb.atb_gated_ffn(x, wg, wu, wd, act=act), lambda: atb.atb_gated_ffn_backward(x, x, wg, wu, wd, H, G, U, act=act)):
        with pytest.raises(atb.AtbError) as e:
            call()
        assert e.value.status == 9

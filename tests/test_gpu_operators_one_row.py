"""Matrices of one row: the distance to a next row, which is not there, refuses nothing and changes nothing."""
import pytest
import torch

import paper_2511_16041_b200 as atb

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def _row(n, pad, dtype=BF16):
    """One row out of a matrix with rows of n + pad elements, on a 16-byte boundary."""
    return torch.randn((3, n + pad), device="cuda").to(dtype)[:1, :n]


def _same(a, b):
    for p, q in zip(a, b):
        assert torch.equal(p, q)


@pytest.mark.parametrize("pad", [3, 8])
def test_one_token(pad):
    D, F = 64, 136
    x, dy, wd = _row(D, pad), _row(D, pad), torch.randn(F, D, device="cuda").to(BF16)
    wg, wu = (torch.randn(D, F, device="cuda").to(BF16) for _ in range(2))
    keep = [_row(F, pad) for _ in range(3)]                    # H, G, U
    plain = atb.atb_gated_ffn(x.clone(), wg, wu, wd, save=BF16)
    outs = atb.atb_gated_ffn(x, wg, wu, wd, save=True, Y=_row(D, pad), H=keep[0], G=keep[1], U=keep[2])
    _same(outs, plain)
    _same(atb.atb_gated_ffn_backward(dy, x, wg, wu, wd, *outs[1:], dX=_row(D, pad)),
          atb.atb_gated_ffn_backward(dy.clone(), x.clone(), wg, wu, wd, *plain[1:]))


@pytest.mark.parametrize("pad", [3, 8])
def test_one_row_of_a_norm(pad):
    x, w = _row(64, pad), torch.randn(64, device="cuda")
    _same(atb.atb_layer_norm(x, w, w), atb.atb_layer_norm(x.clone(), w, w))
    mant = torch.empty((3, 64 + pad), dtype=torch.int8, device="cuda")[:1, :64]
    _same(atb.atb_layer_norm_bfp16(x, w, w, mant=mant), atb.atb_layer_norm_bfp16(x.clone(), w, w))


@pytest.mark.parametrize("pad", [3, 8])
def test_one_row_and_one_word(pad):
    x, w, labels = _row(64, pad), _row(64, pad), torch.zeros(1, dtype=torch.int64, device="cuda")
    head = torch.randn(300, 64, device="cuda").to(BF16)
    for weights in (w, head):
        loss, lse = atb.atb_linear_cross_entropy(x, weights, labels)
        _same((loss, lse), atb.atb_linear_cross_entropy(x.clone(), weights.clone(), labels))
        args = (weights, labels, lse)
        _same(atb.atb_linear_cross_entropy_backward(torch.ones(1, device="cuda"), x, *args, dX=_row(64, pad)),
              atb.atb_linear_cross_entropy_backward(torch.ones(1, device="cuda"), x.clone(), *args))

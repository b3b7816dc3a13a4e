"""Softmax cross entropy of a linear head against the formulas in 64 bits."""
import pytest
import torch

import paper_2511_16041_b200 as atb
from tests import operators_ref as ref
from tests.operators_ref import U16, U32, product_bound

pytestmark = pytest.mark.gpu

BF16, IGNORE = torch.bfloat16, -100


def _inputs(M, V, D, scale=2.0, pad=0, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(5 + seed)
    x = torch.randn((M, D + pad), generator=gen, device="cuda").to(BF16)[:, :D]
    w = (torch.randn((V, D + pad), generator=gen, device="cuda") * scale / D ** 0.5).to(BF16)[:, :D]
    labels = torch.randint(0, V, (M,), generator=gen, device="cuda")
    if M > 2:
        labels[1::5] = IGNORE
    labels[0], labels[-1] = 0, V - 1
    dloss = torch.rand(M, generator=gen, device="cuda") + 0.5
    return x, w, labels, dloss


def _logit_error(x, w):
    return product_bound(x, w.t()).max(1).values


def _check_forward(x, w, labels, loss, lse, ignore=IGNORE):
    xd, wd = x.double(), w.double()
    want_loss, want_lse, _ = ref.cross_entropy(xd, wd, labels, ignore)
    # lse: the logits' error; 128 terms added one by one, the join, and the fast exponential on arguments below 2^7: 2^-15
    # at most of terms that far below the maximum, 2^-22 of those that count; log and the last addition
    tol = _logit_error(xd, wd) + 600 * U32 + 8 * U32 * want_lse.abs()
    ref.check(lse, want_lse, tol, "lse")
    ref.check(loss, want_loss, 2 * tol + 2 * U32 * want_loss.abs(), "loss")
    assert bool((loss[labels == ignore] == 0).all())


def _check_backward(x, w, labels, dloss, lse, dl, dX, dW, ignore=IGNORE):
    """dl: the workspace's dL, in units of the largest dloss that counts, where the vocabulary is one piece, else None."""
    M, V = x.shape[0], w.shape[0]
    xd, wd = x.double(), w.double()
    _, want_lse, p = ref.cross_entropy(xd, wd, labels, ignore)
    scale = torch.where(labels != ignore, dloss.double(), torch.zeros_like(dloss, dtype=torch.float64))[:, None]
    hot = torch.zeros_like(p).scatter_(1, labels.clamp(min=0)[:, None], 1.0)
    want = (p - hot) * scale
    # exp(l - lse): both exponents' errors, the fast exponential as above
    err = scale * (p * (3 * _logit_error(xd, wd)[:, None] + 2.0 ** -14 + 16 * U32 * want_lse.abs()[:, None]) + 3 * U32)
    err = err + U16 * (want.abs() + err)
    if dl is not None:
        exact = dl.double() * scale.max()
        ref.check(exact, want, err, "dl")
        for got, left, right, name in ((dX, exact, wd, "dx"), (dW, exact.t(), xd, "dw")):
            res, e = left @ right, product_bound(left, right)
            ref.check(got, res, e + U16 * (res.abs() + e), name)
    else:
        for got, left, right, e, name in ((dX, want, wd, err, "dx"), (dW, want.t(), xd, err.t(), "dw")):
            res, e = left @ right, product_bound(left, right) + e @ right.abs()
            ref.check(got, res, e + U16 * (res.abs() + e), name)


SHAPES = [(1, 1, 8), (1, 7, 64), (2, 130, 72), (3, 1000, 256), (16, 3200, 512), (33, 63, 136), (100, 129, 64), (128, 513, 200), (129, 257, 64),
          (200, 5003, 128), (300, 2048, 1024), (600, 1025, 96),
          # several tiles for every CTA or pair
          (20, 60011, 64), (100, 60011, 72), (900, 30011, 136)]


@pytest.mark.parametrize("M,V,D", SHAPES)
def test_forward_and_backward(M, V, D):
    for pad in (0, 16):
        x, w, labels, dloss = _inputs(M, V, D, pad=pad)
        loss, lse = atb.atb_linear_cross_entropy(x, w, labels)
        _check_forward(x, w, labels, loss, lse)
        need = atb.atb_linear_cross_entropy_backward_workspace_bytes(M, V, D)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        dX, dW = atb.atb_linear_cross_entropy_backward(dloss, x, w, labels, lse, workspace=ws)
        atb.atb_device_status()
        words = -(-V // 256) * 256                             # one piece: rows of whole tiles
        assert atb.atb_linear_cross_entropy_backward_workspace_bytes(M, V, D, V) == need
        dl = ws[:2 * M * words].view(BF16).view(M, words)[:, :V]
        _check_backward(x, w, labels, dloss, lse, dl, dX, dW)


@pytest.mark.parametrize("M,V,D,piece", [(5, 1000, 64, 256), (150, 2000, 72, 300), (300, 5003, 128, 1024), (64, 513, 64, 512)])
def test_pieces_of_the_vocabulary(M, V, D, piece):
    x, w, labels, dloss = _inputs(M, V, D)
    loss, lse = atb.atb_linear_cross_entropy(x, w, labels)
    dX, dW = atb.atb_linear_cross_entropy_backward(dloss, x, w, labels, lse, piece=piece)
    _check_backward(x, w, labels, dloss, lse, None, dX, dW)


def test_large_logits_and_one_dominant_word():
    """Logits of several hundred, one word far above the others: probabilities of exactly 0 and 1 in fp32."""
    M, V, D = 140, 700, 64
    x, w, labels, dloss = _inputs(M, V, D, scale=60.0)
    w[123] = (x[3].float() * 20).to(BF16)
    labels[3] = 123
    loss, lse = atb.atb_linear_cross_entropy(x, w, labels)
    xd, wd = x.double(), w.double()
    want_loss, want_lse, p = ref.cross_entropy(xd, wd, labels, IGNORE)
    tol = 2 * _logit_error(xd, wd) + 600 * U32 + 16 * U32 * want_lse.abs()
    ref.check(lse, want_lse, tol, "lse")
    ref.check(loss, want_loss, 2 * tol, "loss")
    dX, dW = atb.atb_linear_cross_entropy_backward(dloss, x, w, labels, lse)
    assert bool(torch.isfinite(dX).all()) and bool(torch.isfinite(dW).all())


def test_every_row_ignored():
    x, w, labels, dloss = _inputs(20, 300, 64)
    labels[:] = IGNORE
    loss, lse = atb.atb_linear_cross_entropy(x, w, labels)
    assert bool((loss == 0).all()) and bool(torch.isfinite(lse).all())
    dX, dW = atb.atb_linear_cross_entropy_backward(dloss, x, w, labels, lse)
    assert bool((dX == 0).all()) and bool((dW == 0).all())


def test_ignore_index_may_be_a_word_and_labels_outside_are_nan():
    x, w, labels, dloss = _inputs(9, 300, 64)
    labels[labels == IGNORE] = 4
    labels[2], labels[5] = 300, -7
    labels[6] = 4
    loss, lse = atb.atb_linear_cross_entropy(x, w, labels, ignore_index=4)
    assert bool(torch.isnan(loss[[2, 5]]).all()) and bool(torch.isnan(lse[[2, 5]]).all())
    rest = [0, 1, 3, 4, 6, 7, 8]
    assert float(loss[6]) == 0
    _check_forward(x[rest], w, labels[rest], loss[rest], lse[rest], ignore=4)
    dX, dW = atb.atb_linear_cross_entropy_backward(dloss, x, w, labels, lse, ignore_index=4)
    assert bool(torch.isnan(dX[[2, 5]]).all()) and bool(torch.isfinite(dX[rest]).all()) and bool((dX[6] == 0).all())


def test_an_ignored_row_of_infinities_has_no_gradient():
    x, w, labels, dloss = _inputs(6, 300, 64)
    labels[:] = 3
    labels[4] = IGNORE
    x[4] = float("inf")
    loss, lse = atb.atb_linear_cross_entropy(x, w, labels)
    dX, _ = atb.atb_linear_cross_entropy_backward(dloss, x, w, labels, lse)
    assert float(loss[4]) == 0 and bool((dX[4] == 0).all())


def test_no_rows_guards_and_same_bits():
    x, w, labels, dloss = _inputs(150, 777, 128)
    loss, lse = atb.atb_linear_cross_entropy(x[:0], w, labels[:0])
    dX, dW = atb.atb_linear_cross_entropy_backward(dloss[:0], x[:0], w, labels[:0], lse)
    assert loss.shape == (0,) and dX.shape == (0, 128) and bool((dW == 0).all())
    loss, lse = atb.atb_linear_cross_entropy(x, w, labels)
    buf_x = torch.full((151, 144), 7.0, dtype=BF16, device="cuda")
    buf_w = torch.full((778, 144), 7.0, dtype=BF16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        loss2, lse2 = atb.atb_linear_cross_entropy(x, w, labels)
        atb.atb_linear_cross_entropy_backward(dloss, x, w, labels, lse2, dX=buf_x[:150, :128], dW=buf_w[:777, :128])
    side.synchronize()
    dX, dW = atb.atb_linear_cross_entropy_backward(dloss, x, w, labels, lse)
    assert torch.equal(loss, loss2) and torch.equal(lse, lse2)
    assert torch.equal(dX, buf_x[:150, :128]) and torch.equal(dW, buf_w[:777, :128])
    for buf, r in ((buf_x, 150), (buf_w, 777)):
        assert bool((buf[r] == 7).all()) and bool((buf[:, 128:] == 7).all())


def test_gradient_against_differences():
    M, V, D = 12, 300, 64
    x, w, labels, dloss = _inputs(M, V, D)
    _, lse = atb.atb_linear_cross_entropy(x, w, labels)
    grads = [t.double() for t in atb.atb_linear_cross_entropy_backward(dloss, x, w, labels, lse)]
    args = [x.double(), w.double()]
    gen = torch.Generator(device="cuda").manual_seed(4)

    def loss(a):
        return float((ref.cross_entropy(a[0], a[1], labels, IGNORE)[0] * dloss.double()).sum())

    for i in range(2):
        d = torch.randn(args[i].shape, generator=gen, device="cuda", dtype=torch.float64)
        h = 1e-5
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + h * d, args[i] - h * d
        slope = (loss(up) - loss(down)) / (2 * h)
        # two roundings to bf16: dl and the result
        assert abs(slope - float((grads[i] * d).sum())) <= 3 * U16 * float((grads[i] * d).abs().sum()), i


@pytest.mark.parametrize("M,V,D,piece", [(255, 3000, 256, 0), (255, 3000, 256, 1024), (12, 5003, 512, 0)])
def test_a_mean_is_not_rounded(M, V, D, piece):
    """dloss = 1 / 255, half way between two bf16 numbers, in every row: rounded as it is it would move both gradients by
    2^-8 of their size.  Left are dL's other roundings and the result's, of 2^-8 / sqrt(3) at most in the mean square each; along the
    result only a label's p - 1 counts, which is off by at most 2^-9."""
    x, w, labels, _ = _inputs(M, V, D)
    dloss = torch.full((M,), 1 / 255, device="cuda")
    dloss[labels == IGNORE] = 1e30                             # does not count
    _, lse = atb.atb_linear_cross_entropy(x, w, labels)
    dX, dW = atb.atb_linear_cross_entropy_backward(dloss, x, w, labels, lse, piece=piece)
    _, _, p = ref.cross_entropy(x.double(), w.double(), labels, IGNORE)
    d = (p - torch.zeros_like(p).scatter_(1, labels.clamp(min=0)[:, None], 1.0)) * ((labels != IGNORE) * float(dloss[0]))[:, None]
    for got, want, name in ((dX, d @ w.double(), "dx"), (dW, d.t() @ x.double(), "dw")):
        off = float((got.double() - want).norm() / want.norm())
        along = float((got.double() * want).sum() / (want * want).sum()) - 1
        assert off <= 2.0 ** -8 * (2 / 3) ** 0.5, (name, off)
        assert abs(along) <= 2.0 ** -9, (name, along)


def test_scales_of_every_kind():
    """0 in every row, numbers near the ends of FP32, an infinite and a NaN one beside finite ones."""
    x, w, labels, dloss = _inputs(40, 300, 64)
    labels[:] = torch.arange(40, device="cuda")
    _, lse = atb.atb_linear_cross_entropy(x, w, labels)
    back = lambda s: atb.atb_linear_cross_entropy_backward(s, x, w, labels, lse)  # noqa: E731
    dX, dW = back(torch.zeros_like(dloss))
    assert bool((dX == 0).all()) and bool((dW == 0).all())
    one = back(dloss)
    for power in (-60, 60):                                    # a power of two changes no rounding
        dX, dW = back(dloss * 2.0 ** power)
        assert torch.equal(dX.double(), one[0].double() * 2.0 ** power) and torch.equal(dW.double(), one[1].double() * 2.0 ** power)
    dloss[7], dloss[9] = float("inf"), float("nan")
    dX, dW = back(dloss)
    rest = [i for i in range(40) if i not in (7, 9)]
    assert not bool(torch.isfinite(dX[[7, 9]]).any()) and bool(torch.isfinite(dX[rest]).all())
    assert bool(torch.isnan(dW).all())
    _check_backward(x[rest], w, labels[rest], dloss[rest], lse[rest], None, dX[rest], back(torch.where(torch.isfinite(dloss), dloss, 0.0))[1])

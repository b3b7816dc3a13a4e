"""Plain 64-bit forms of layer norm, the gated feed-forward block and the linear cross entropy, and the error bounds
that the GPU tests hold the kernels to.

U32 = 2^-24 and U16 = 2^-8 are the relative errors of one rounding to fp32 and bf16.  ``product_bound`` covers an FP32
sum of K products in any order with truncating additions: K * 2^-23 of the sum of magnitudes."""
import math

import torch

U32, U16 = 2.0 ** -24, 2.0 ** -8


def product_bound(a, b):
    """Bound on the error of the FP32 accumulation of a @ b (a, b exact, double)."""
    return (a.shape[1] + 32) * 2.0 ** -23 * (a.abs() @ b.abs())


def check(got, want, tol, what):
    """Every element within its bound; NaN and infinity only where wanted."""
    got = got.double()
    assert got.shape == want.shape, what
    assert bool(torch.isfinite(got).all()), f"{what}: not finite"
    over = (got - want).abs() - tol
    worst = int(over.argmax()) if over.numel() else 0
    assert over.numel() == 0 or float(over.max()) <= 0, \
        f"{what}: element {worst}: {float(got.reshape(-1)[worst])} for {float(want.reshape(-1)[worst])}, allowed {float(tol.expand_as(want).reshape(-1)[worst])}"


def act(g, name):
    """act(g), act'(g)."""
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    if name == "gelu":
        phi = 0.5 * torch.erfc(-g / math.sqrt(2))
        return g * phi, phi + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def layer_norm(x, w, b, eps):
    """y, z, rstd of the rows of x; w, b may be None."""
    mu = x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((x - mu) ** 2).mean(1, keepdim=True) + eps)
    z = (x - mu) * rstd
    return z * (1 if w is None else w) + (0 if b is None else b), z, mu, rstd


def layer_norm_backward(dy, z, w, rstd):
    g = dy * (1 if w is None else w)
    dx = rstd * (g - g.mean(1, keepdim=True) - z * (g * z).mean(1, keepdim=True))
    return dx, (dy * z).sum(0), dy.sum(0), g


def gated_ffn(x, wg, wu, wd, name):
    return (act(x @ wg, name)[0] * (x @ wu)) @ wd


def cross_entropy(x, w, labels, ignore):
    """loss, lse, and exp(logits - lse)."""
    logits = x @ w.t()
    lse = torch.logsumexp(logits, 1)
    keep = labels != ignore
    picked = logits.gather(1, labels.clamp(min=0)[:, None])[:, 0]
    return torch.where(keep, lse - picked, torch.zeros_like(lse)), lse, torch.exp(logits - lse[:, None])

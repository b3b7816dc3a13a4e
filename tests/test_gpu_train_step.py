"""The operators together: a block's training step against automatic differentiation in 64 bits, and the example that learns."""
import math

import pytest
import torch

import paper_2511_16041_b200 as atb
from paper_2511_16041_b200 import train_step

pytestmark = pytest.mark.gpu


def _reference(block, x, labels):
    """Loss and gradients of the same block from its rounded weights, in 64 bits."""
    w = {k: v.double().requires_grad_() for k, v in block.w.items()}
    x = x.double().requires_grad_()

    def norm(t, weight, bias):
        return torch.nn.functional.layer_norm(t, t.shape[1:], weight, bias, 1e-5)

    a = norm(x, w["n1w"], w["n1b"])
    h = x + (torch.nn.functional.silu(a @ w["wg"]) * (a @ w["wu"])) @ w["wd"]
    loss = torch.nn.functional.cross_entropy(norm(h, w["n2w"], w["n2b"]) @ w["head"].t(), labels, ignore_index=-100)
    loss.backward()
    return float(loss.detach()), {k: v.grad for k, v in w.items()}, x.grad


@pytest.mark.parametrize("tokens,model,hidden,words", [(1, 64, 136, 70), (37, 128, 344, 501), (300, 256, 688, 1000)])
def test_gradients_of_the_whole_block(tokens, model, hidden, words):
    gen = torch.Generator(device="cuda").manual_seed(3)
    block = train_step.Block(model, hidden, words)
    x = torch.randn((tokens, model), generator=gen, device="cuda").to(torch.bfloat16)
    labels = torch.randint(0, words, (tokens,), generator=gen, device="cuda")
    if tokens > 2:
        labels[1::7] = -100
    loss, g, dx = block.gradients(x, labels)
    atb.atb_device_status()
    want, wg, wdx = _reference(block, x, labels)
    # about a dozen roundings to bf16 lie between (a, g, u, h, f, x + f, z and their gradients), each 2^-9 rms of its value: 12^0.5
    # of that in the norm of a gradient, twice over for what the softmax and the norms make of it
    assert abs(float(loss) - want) <= 0.01 * max(1.0, want)
    for k in wg:
        assert float((g[k].double() - wg[k]).norm()) <= 0.03 * float(wg[k].norm()), k
    assert float((dx.double() - wdx).norm()) <= 0.03 * float(wdx.norm())


def test_the_example_learns():
    losses, right = train_step.main(["--steps", "150", "--words", "256", "--tokens", "512", "--model", "128", "--hidden", "344"])
    assert losses[0] > 0.8 * math.log(256) and losses[-1] < 0.5 * losses[0]
    assert right > 0.5

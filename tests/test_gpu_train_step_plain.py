"""The example with linear layers and the residual norm: it runs, its gradients are those of automatic differentiation in 64 bits, and its
draws are those of its logits."""
import pytest
import torch

import paper_2511_16041_b200 as atb
from paper_2511_16041_b200 import train_step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("tokens", [1, 2, 37, 300])
def test_gradients(tokens, act):
    f = torch.nn.functional
    block = train_step.Block(96, 264, 500, act=act, plain=True)
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    for k in ("b1", "b2", "gate", "n1w", "n2w"):
        block.master[k] += 0.3 * torch.randn(block.master[k].shape, generator=gen, device="cuda")
    block._round()
    x = torch.randn((tokens, 96), generator=gen, device="cuda").to(torch.bfloat16)
    labels = torch.randint(0, 500, (tokens,), generator=gen, device="cuda")
    if tokens > 2:
        labels[1] = -100
    loss, grads, dx = block.gradients(x, labels)
    atb.atb_device_status()
    w = {k: v.double().requires_grad_() for k, v in block.w.items()}
    xd = x.double().requires_grad_()
    acts = {"silu": f.silu, "gelu": f.gelu, "gelu_tanh": lambda t: f.gelu(t, approximate="tanh")}
    a = f.layer_norm(xd, (96,), w["n1w"], w["n1b"])
    h = xd + w["gate"] * (acts[act](a @ w["w1"] + w["b1"]) @ w["w2"] + w["b2"])
    want = f.cross_entropy(f.layer_norm(h, (96,), w["n2w"], w["n2b"]) @ w["head"].t(), labels, ignore_index=-100)
    want.backward()
    # about a dozen roundings to bf16 of 2^-8 each at most on the way to a gradient
    assert abs(float(loss) - float(want.detach())) <= 0.01 * max(1.0, float(want.detach()))
    assert set(grads) == set(w)
    for k, g in (*grads.items(), ("x", dx)):
        ref = xd.grad if k == "x" else w[k].grad
        assert float((g.double() - ref).norm()) <= 0.03 * float(ref.norm()), k


def test_answers():
    block = train_step.Block(64, 136, 336, plain=True)
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((50, 64), generator=gen, device="cuda").to(torch.bfloat16)
    u = torch.rand(50, generator=gen, device="cuda")
    logits = block.logits(x)
    assert torch.equal(block.sample(x, u, temperature=0.0), logits.float().argmax(1))
    for settings in (dict(temperature=0.9, top_k=7), dict(top_p=0.5), dict()):
        assert torch.equal(block.sample(x, u, **settings), atb.atb_sample(logits, u, **settings)[0])


@pytest.mark.parametrize("flags", [[], ["--plain"]])
def test_the_command_runs(flags, capsys):
    losses, right = train_step.main(["--steps", "3", "--tokens", "64", "--model", "64", "--hidden", "136", "--words", "104", *flags])
    assert len(losses) == 3 and all(v == v for v in losses) and 0 <= right <= 1
    assert "drawn" in capsys.readouterr().out


def test_a_step_captured_and_replayed():
    """Forward, backward and a draw as one graph, replayed on other inputs: the same as eager calls."""
    block = train_step.Block(64, 136, 200, plain=True)
    gen = torch.Generator(device="cuda").manual_seed(4)
    make = lambda: (torch.randn((80, 64), generator=gen, device="cuda").to(torch.bfloat16), torch.randint(0, 200, (80,), generator=gen, device="cuda"),  # noqa: E731
                    torch.rand(80, generator=gen, device="cuda"))
    x, labels, u = make()

    def work(x, labels, u):
        loss, grads, dx = block.gradients(x, labels)
        z, _ = block.forward_plain(x)
        logits = atb.atb_linear(z, block.w["head"].t(), dtype=torch.float32)
        return [loss, dx, *grads.values(), *atb.atb_sample(logits, u, temperature=0.8, top_k=20, top_p=0.95)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work(x, labels, u)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = work(x, labels, u)
    for _ in range(3):
        x2, labels2, u2 = make()
        x.copy_(x2), labels.copy_(labels2), u.copy_(u2)
        graph.replay()
        want = work(x2, labels2, u2)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)

"""A training step of a small block, made of the library's operators, and what it has learned, through the BFP16 GEMM.

    python -m paper_2511_16041_b200.train_step [--steps 60] [--tokens 512] [--model 256] [--hidden 688] [--words 1024]

The block is ``h = x + ffn(norm1(x))`` with the gated feed-forward block, the head ``softmax(norm2(h) W^T)`` with its cross
entropy.  ``Block.step`` is one training step: forward, backward and plain gradient descent on FP32 copies of the weights;
activations and the weights that the kernels read are bf16.  ``Block.logits`` is the path for answers: the last norm leaves
as BFP16 planes, which are the A operand of ``atb_gemm``.  The task is synthetic: every word has one successor.
"""
from __future__ import annotations

import argparse

import paper_2511_16041_b200 as atb


class Block:
    """Weights in FP32 (``master``) and as the kernels read them (``w``): matrices bf16, norm parameters FP32."""

    MATRICES = ("wg", "wu", "wd", "head")

    def __init__(self, model: int, hidden: int, words: int, act: str = "silu", device="cuda", seed: int = 0):
        import torch
        gen = torch.Generator(device=device).manual_seed(seed)

        def normal(rows, cols, scale):
            return torch.randn((rows, cols), generator=gen, device=device) * scale

        self.act = act
        self.master = {
            "wg": normal(model, hidden, model ** -0.5), "wu": normal(model, hidden, model ** -0.5), "wd": normal(hidden, model, hidden ** -0.5),
            "head": normal(words, model, model ** -0.5),
            "n1w": torch.ones(model, device=device), "n1b": torch.zeros(model, device=device),
            "n2w": torch.ones(model, device=device), "n2b": torch.zeros(model, device=device)}
        self._round()

    def _round(self):
        import torch
        self.w = {k: v.to(torch.bfloat16) if k in self.MATRICES else v for k, v in self.master.items()}

    def forward(self, x):
        """``x`` bf16 [tokens, model] -> the last norm's result and what the backward pass needs."""
        w = self.w
        a, mean1, rstd1 = atb.atb_layer_norm(x, w["n1w"], w["n1b"])
        f, H, G, U = atb.atb_gated_ffn(a, w["wg"], w["wu"], w["wd"], act=self.act, save=True)
        h = x + f
        z, mean2, rstd2 = atb.atb_layer_norm(h, w["n2w"], w["n2b"])
        return z, (x, a, mean1, rstd1, H, G, U, h, mean2, rstd2)

    def gradients(self, x, labels, ignore_index: int = -100):
        """Mean loss over the counted tokens, and the gradients of the weights and of ``x``."""
        w = self.w
        z, (x, a, mean1, rstd1, H, G, U, h, mean2, rstd2) = self.forward(x)
        loss, lse = atb.atb_linear_cross_entropy(z, w["head"], labels, ignore_index=ignore_index)
        counts = (labels != ignore_index).float()
        dloss = counts / counts.sum().clamp(min=1.0)
        g = {}
        dz, g["head"] = atb.atb_linear_cross_entropy_backward(dloss, z, w["head"], labels, lse, ignore_index=ignore_index)
        dh, g["n2w"], g["n2b"] = atb.atb_layer_norm_backward(dz, h, w["n2w"], mean2, rstd2)
        da, g["wg"], g["wu"], g["wd"] = atb.atb_gated_ffn_backward(dh, a, w["wg"], w["wu"], w["wd"], H, G, U, act=self.act)
        dx, g["n1w"], g["n1b"] = atb.atb_layer_norm_backward(da, x, w["n1w"], mean1, rstd1)
        return (loss * dloss).sum(), g, dx + dh

    def step(self, x, labels, rate: float, ignore_index: int = -100):
        """One step of gradient descent; returns the loss before it."""
        loss, g, _ = self.gradients(x, labels, ignore_index)
        for k, v in g.items():
            self.master[k] -= rate * v.float()
        self._round()
        return loss

    def logits(self, x):
        """bf16 logits [tokens, words]: the last norm in BFP16, times the head, by the library's BFP16 x BF16 GEMM."""
        w = self.w
        a, _, _ = atb.atb_layer_norm(x, w["n1w"], w["n1b"])
        h = x + atb.atb_gated_ffn(a, w["wg"], w["wu"], w["wd"], act=self.act)
        mant, exp, _, _ = atb.atb_layer_norm_bfp16(h, w["n2w"], w["n2b"])
        M, K, N = h.shape[0], h.shape[1], w["head"].shape[0]
        tiling, _ = atb.atb_select_tiling(M, N, K)
        return atb.atb_gemm(M, N, K, *tiling, mant, exp, w["head"].t().contiguous())


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--tokens", type=int, default=512)
    p.add_argument("--model", type=int, default=256)
    p.add_argument("--hidden", type=int, default=688)
    p.add_argument("--words", type=int, default=1024)
    p.add_argument("--rate", type=float, default=2.0)
    a = p.parse_args(argv)
    import torch
    gen = torch.Generator(device="cuda").manual_seed(1)
    embedding = torch.randn((a.words, a.model), generator=gen, device="cuda").to(torch.bfloat16)
    successor = torch.randperm(a.words, generator=gen, device="cuda")
    block = Block(a.model, a.hidden, a.words)
    losses = []
    for i in range(a.steps):
        words = torch.randint(0, a.words, (a.tokens,), generator=gen, device="cuda")
        losses.append(block.step(embedding[words], successor[words], a.rate))
        if i % 10 == 0 or i == a.steps - 1:
            print(f"step {i:4d}  loss {float(losses[-1]):.4f}")
    words = torch.arange(a.words, device="cuda")
    right = float((block.logits(embedding[words]).argmax(1) == successor[words]).float().mean())
    atb.atb_device_status()
    print(f"words whose successor the block knows (BFP16 GEMM): {right:.1%}")
    return [float(v) for v in losses], right


if __name__ == "__main__":
    main()

"""A training step of a small block, made of the library's operators, and what it has learned, through the BFP16 GEMM.

    python -m paper_2511_16041_b200.train_step [--steps 60] [--tokens 512] [--model 256] [--hidden 688] [--words 1024] [--plain]

The block is ``h = x + ffn(norm1(x))`` with the gated feed-forward block, the head ``softmax(norm2(h) W^T)`` with its cross
entropy; with ``plain`` the branch is two linear layers with biases instead, and joins the stream through a learned gate and
the residual norm: ``h = x + gate * (act(norm1(x) W1 + b1) W2 + b2)``.  ``Block.step`` is one training step: forward, backward and plain
gradient descent on FP32 copies of the weights; activations and the weights that the kernels read are bf16.  ``Block.logits`` is
the path for answers: the last norm leaves as BFP16 planes, which are the A operand of ``atb_gemm``; ``Block.sample`` draws from them.
The task is synthetic: every word has one successor.
"""
from __future__ import annotations

import argparse

import paper_2511_16041_b200 as atb


class Block:
    """Weights in FP32 (``master``) and as the kernels read them (``w``): matrices bf16, norm parameters FP32."""

    MATRICES = ("wg", "wu", "wd", "w1", "w2", "head")

    def __init__(self, model: int, hidden: int, words: int, act: str = "silu", device="cuda", seed: int = 0, plain: bool = False):
        import torch
        gen = torch.Generator(device=device).manual_seed(seed)

        def normal(rows, cols, scale):
            return torch.randn((rows, cols), generator=gen, device=device) * scale

        self.act, self.plain = act, plain
        if plain:
            branch = {"w1": normal(model, hidden, model ** -0.5), "b1": torch.zeros(hidden, device=device),
                      "w2": normal(hidden, model, hidden ** -0.5), "b2": torch.zeros(model, device=device), "gate": torch.ones(model, device=device)}
        else:
            branch = {"wg": normal(model, hidden, model ** -0.5), "wu": normal(model, hidden, model ** -0.5), "wd": normal(hidden, model, hidden ** -0.5)}
        self.master = {
            **branch, "head": normal(words, model, model ** -0.5),
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

    def forward_plain(self, x):
        """The same with the plain branch."""
        w = self.w
        a, mean1, rstd1 = atb.atb_layer_norm(x, w["n1w"], w["n1b"])
        u, s = atb.atb_linear(a, w["w1"], w["b1"], act=self.act, save=True)
        f = atb.atb_linear(u, w["w2"], w["b2"])
        h, z, stats = atb.atb_residual_norm(x, f, w["n2w"], w["n2b"], gate=w["gate"])
        return z, (x, a, mean1, rstd1, s, u, f, h, stats)

    def _head_gradients(self, z, labels, ignore_index):
        """Mean loss, the gradient of z, and that of the head."""
        loss, lse = atb.atb_linear_cross_entropy(z, self.w["head"], labels, ignore_index=ignore_index)
        counts = (labels != ignore_index).float()
        dloss = counts / counts.sum().clamp(min=1.0)
        return ((loss * dloss).sum(), *atb.atb_linear_cross_entropy_backward(dloss, z, self.w["head"], labels, lse, ignore_index=ignore_index))

    def _gradients_plain(self, x, labels, ignore_index):
        w, g = self.w, {}
        z, (x, a, mean1, rstd1, s, u, f, _, stats) = self.forward_plain(x)
        loss, dz, g["head"] = self._head_gradients(z, labels, ignore_index)
        dx, df, g["gate"], g["n2w"], g["n2b"], _, _ = atb.atb_residual_norm_backward(dz, None, x, f, stats, w["n2w"], gate=w["gate"])
        du, g["w2"], g["b2"] = atb.atb_linear_backward(df, u, w["w2"])
        da, g["w1"], g["b1"] = atb.atb_linear_backward(du, a, w["w1"], s, act=self.act)
        dx1, g["n1w"], g["n1b"] = atb.atb_layer_norm_backward(da, x, w["n1w"], mean1, rstd1)
        return loss, g, dx + dx1

    def gradients(self, x, labels, ignore_index: int = -100):
        """Mean loss over the counted tokens, and the gradients of the weights and of ``x``."""
        if self.plain:
            return self._gradients_plain(x, labels, ignore_index)
        w = self.w
        z, (x, a, mean1, rstd1, H, G, U, h, mean2, rstd2) = self.forward(x)
        g = {}
        loss, dz, g["head"] = self._head_gradients(z, labels, ignore_index)
        dh, g["n2w"], g["n2b"] = atb.atb_layer_norm_backward(dz, h, w["n2w"], mean2, rstd2)
        da, g["wg"], g["wu"], g["wd"] = atb.atb_gated_ffn_backward(dh, a, w["wg"], w["wu"], w["wd"], H, G, U, act=self.act)
        dx, g["n1w"], g["n1b"] = atb.atb_layer_norm_backward(da, x, w["n1w"], mean1, rstd1)
        return loss, g, dx + dh

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
        if self.plain:
            h = self.forward_plain(x)[1][7]
        else:
            a, _, _ = atb.atb_layer_norm(x, w["n1w"], w["n1b"])
            h = x + atb.atb_gated_ffn(a, w["wg"], w["wu"], w["wd"], act=self.act)
        mant, exp, _, _ = atb.atb_layer_norm_bfp16(h, w["n2w"], w["n2b"])
        M, K, N = h.shape[0], h.shape[1], w["head"].shape[0]
        tiling, _ = atb.atb_select_tiling(M, N, K)
        return atb.atb_gemm(M, N, K, *tiling, mant, exp, w["head"].t().contiguous())

    def sample(self, x, u, **settings):
        """One word for each row of ``x``, drawn from the logits with the random numbers ``u``; the settings of ``atb_sample``."""
        return atb.atb_sample(self.logits(x), u, **settings)[0]


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--tokens", type=int, default=512)
    p.add_argument("--model", type=int, default=256)
    p.add_argument("--hidden", type=int, default=688)
    p.add_argument("--words", type=int, default=1024)
    p.add_argument("--rate", type=float, default=2.0)
    p.add_argument("--plain", action="store_true", help="linear layers and the residual norm instead of the gated feed-forward block")
    a = p.parse_args(argv)
    import torch
    gen = torch.Generator(device="cuda").manual_seed(1)
    embedding = torch.randn((a.words, a.model), generator=gen, device="cuda").to(torch.bfloat16)
    successor = torch.randperm(a.words, generator=gen, device="cuda")
    block = Block(a.model, a.hidden, a.words, plain=a.plain)
    losses = []
    for i in range(a.steps):
        words = torch.randint(0, a.words, (a.tokens,), generator=gen, device="cuda")
        losses.append(block.step(embedding[words], successor[words], a.rate))
        if i % 10 == 0 or i == a.steps - 1:
            print(f"step {i:4d}  loss {float(losses[-1]):.4f}")
    words = torch.arange(a.words, device="cuda")
    right = float((block.logits(embedding[words]).argmax(1) == successor[words]).float().mean())
    drawn = block.sample(embedding[words], torch.rand(a.words, generator=gen, device="cuda"), temperature=0.7, top_k=20, top_p=0.9)
    atb.atb_device_status()
    print(f"words whose successor is drawn at temperature 0.7 from the best 20 and 0.9 of the probability: {float((drawn == successor[words]).float().mean()):.1%}")
    print(f"words whose successor the block knows (BFP16 GEMM): {right:.1%}")
    return [float(v) for v in losses], right


if __name__ == "__main__":
    main()

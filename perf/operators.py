"""Layer norm, the gated feed-forward block and the softmax cross entropy of a linear head: what is measured of them.

``run`` computes an operator either in its plain form (elementary torch operations in fp32, rounded once at the
end) or, with ``own`` set, through the library's entry points.  ``exact`` computes the same from the definitions in
64 bits.
"""
import math

import torch

own = False

IGNORE = -100
BF16, F32 = "bf16", "f32"
TYPES = {BF16: torch.bfloat16, F32: torch.float32}


# ------------------------------------------------------------------------------------------------ cases
def _norm(name, step, M, N, dtype, weights, pad=0):
    return {"name": name, "op": "norm", "step": step, "M": M, "N": N, "type": dtype, "weights": weights, "pad": pad}


def _ffn(name, step, M, D, F, act):
    return {"name": name, "op": "ffn", "step": step, "M": M, "D": D, "F": F, "act": act}


def _head(name, step, M, V, D):
    return {"name": name, "op": "head", "step": step, "M": M, "V": V, "D": D}


def listed():
    return [
        # one token's norm while an answer is written: latency
        _norm("norm, one token", "forward", 1, 4096, BF16, BF16),
        # the norm in front of a product, over a batch of prompts
        _norm("norm, prompts", "forward", 8192, 4096, BF16, BF16),
        # a small fp32 model with an odd width, its rows a slice of a wider buffer
        _norm("norm, odd fp32 training step", "train", 1021, 1001, F32, F32, pad=6),
        # a training step's norm of a wide model, parameters in fp32
        _norm("norm, wide training step", "train", 16384, 8192, BF16, F32),
        # one token through the block while an answer is written: every weight is read for one row
        _ffn("ffn, one token", "forward", 1, 4096, 10944, "silu"),
        # a prompt of odd length
        _ffn("ffn, prompt", "forward", 509, 2048, 5464, "gelu_tanh"),
        # a small model's step on a small batch
        _ffn("ffn, small training step", "train", 640, 1024, 2736, "gelu"),
        # a training step of one card's batch
        _ffn("ffn, training step", "train", 8192, 4096, 10944, "silu"),
        # the loss of a few answers (their scores), small vocabulary
        _head("head, few answers", "forward", 16, 32000, 2048),
        # perplexity over a text
        _head("head, evaluation", "forward", 4096, 131072, 2048),
        # fine-tuning a small model with an odd vocabulary
        _head("head, odd training step", "train", 1500, 50003, 1024),
        # a training step of one card's batch with a large vocabulary
        _head("head, training step", "train", 8192, 131072, 4096),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _eights(rng, low, high):
    return 8 * _log_int(rng, low // 8, high // 8)


def draw(rng):
    op = rng.choice(["norm", "ffn", "head"])
    step = rng.choice(["forward", "train"])
    if op == "norm":
        c = _norm("", step, _log_int(rng, 1, 16384), _log_int(rng, 64, 8192), rng.choice([BF16, F32]), rng.choice([BF16, F32]),
                  rng.choice([0, 0, 8, 5]))
    elif op == "ffn":
        c = _ffn("", step, _log_int(rng, 1, 8192), _eights(rng, 512, 4096), _eights(rng, 1024, 10944),
                 rng.choice(["silu", "gelu", "gelu_tanh"]))
    else:
        c = _head("", step, _log_int(rng, 1, 8192), _log_int(rng, 4000, 131072), _eights(rng, 512, 4096))
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0, shift=0.0, dtype=torch.bfloat16):
        return torch.randn(shape, generator=gen, device="cuda").mul_(scale).add_(shift).to(dtype)

    s = dict(case)
    M = case["M"]
    if case["op"] == "norm":
        N, dtype, wtype = case["N"], TYPES[case["type"]], TYPES[case["weights"]]
        # a residual stream: a few columns are much larger than the others, rows are off centre
        x = torch.randn((M, N + case["pad"]), generator=gen, device="cuda")
        x = x * (1.0 + 6.0 * (torch.rand((1, N + case["pad"]), generator=gen, device="cuda") > 0.995)) + 0.25
        s["x"] = x.to(dtype)[:, :N]
        s["w"] = normal(N, scale=0.1, shift=1.0, dtype=wtype)
        s["b"] = normal(N, scale=0.1, dtype=wtype)
        s["eps"] = 1e-5
        if case["step"] == "train":
            s["dy"] = normal(M, N, dtype=dtype)
    elif case["op"] == "ffn":
        D, F = case["D"], case["F"]
        s["x"] = normal(M, D)
        s["wg"] = normal(D, F, scale=1.0 / math.sqrt(D))
        s["wu"] = normal(D, F, scale=1.0 / math.sqrt(D))
        s["wd"] = normal(F, D, scale=1.0 / math.sqrt(F))
        if case["step"] == "train":
            s["dy"] = normal(M, D, scale=1e-2)
    else:
        V, D = case["V"], case["D"]
        s["x"] = normal(M, D)
        s["w"] = normal(V, D, scale=2.0 / math.sqrt(D))
        labels = torch.randint(0, V, (M,), generator=gen, device="cuda")
        # the prompt's part and the padding do not count; the first row always does
        keep = torch.rand((M,), generator=gen, device="cuda") > 0.1
        keep[0] = True
        s["labels"] = torch.where(keep, labels, torch.full_like(labels, IGNORE))
        s["dloss"] = keep.float() / keep.sum()
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _act_plain(g, act):
    """act(g) and act'(g)."""
    if act == "silu":
        sig = 1.0 / (1.0 + torch.exp(-g))
        return g * sig, sig * (1.0 + g * (1.0 - sig))
    if act == "gelu":
        phi = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return g * phi, phi + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    c = math.sqrt(2.0 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * c * (1.0 + 3.0 * 0.044715 * g * g)


def _norm_plain(s):
    dtype, wtype = s["x"].dtype, s["w"].dtype
    x, w, b = s["x"].float(), s["w"].float(), s["b"].float()
    d = x - x.mean(1, keepdim=True)
    rstd = torch.rsqrt((d * d).mean(1, keepdim=True) + s["eps"])
    xh = d * rstd
    out = {"y": (xh * w + b).to(dtype)}
    if s["step"] == "train":
        dy = s["dy"].float()
        g = dy * w
        out["dx"] = (rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))).to(dtype)
        out["dw"] = (dy * xh).sum(0).to(wtype)
        out["db"] = dy.sum(0).to(wtype)
    return out


def _ffn_plain(s):
    x, wg, wu, wd = s["x"].float(), s["wg"].float(), s["wu"].float(), s["wd"].float()
    g, u = x @ wg, x @ wu
    a, da = _act_plain(g, s["act"])
    h = a * u
    out = {"y": (h @ wd).bfloat16()}
    if s["step"] == "train":
        dy = s["dy"].float()
        dh = dy @ wd.t()
        dg, du = dh * u * da, dh * a
        out["dx"] = (dg @ wg.t() + du @ wu.t()).bfloat16()
        out["dwg"] = (x.t() @ dg).bfloat16()
        out["dwu"] = (x.t() @ du).bfloat16()
        out["dwd"] = (h.t() @ dy).bfloat16()
    return out


def _head_plain(s):
    x, w, labels = s["x"].float(), s["w"].float(), s["labels"]
    keep = labels != IGNORE
    at = torch.where(keep, labels, torch.zeros_like(labels))[:, None]
    logits = x @ w.t()
    top = logits.max(1, keepdim=True).values
    lse = top + torch.log(torch.exp(logits - top).sum(1, keepdim=True))
    loss = torch.where(keep[:, None], lse - logits.gather(1, at), torch.zeros_like(lse))
    out = {"loss": loss[:, 0], "lse": lse[:, 0]}
    if s["step"] == "train":
        scale = (s["dloss"] * keep)[:, None]
        dlogits = torch.exp(logits - lse) * scale
        dlogits.scatter_add_(1, at, -scale)
        out["dx"] = (dlogits @ w).bfloat16()
        out["dw"] = (dlogits.t() @ x).bfloat16()
    return out


# ------------------------------------------------------------------------------------------------ the library's calls
def _norm_own(s):
    import paper_2511_16041_b200 as atb
    y, mean, rstd = atb.atb_layer_norm(s["x"], s["w"], s["b"], s["eps"])
    if s["step"] != "train":
        return {"y": y}
    dx, dw, db = atb.atb_layer_norm_backward(s["dy"], s["x"], s["w"], mean, rstd)
    return {"y": y, "dx": dx, "dw": dw, "db": db}


def _ffn_own(s):
    import paper_2511_16041_b200 as atb
    if s["step"] != "train":
        return {"y": atb.atb_gated_ffn(s["x"], s["wg"], s["wu"], s["wd"], act=s["act"])}
    y, H, G, U = atb.atb_gated_ffn(s["x"], s["wg"], s["wu"], s["wd"], act=s["act"], save=True)
    dx, dwg, dwu, dwd = atb.atb_gated_ffn_backward(s["dy"], s["x"], s["wg"], s["wu"], s["wd"], H, G, U, act=s["act"])
    return {"y": y, "dx": dx, "dwg": dwg, "dwu": dwu, "dwd": dwd}


def _head_own(s):
    import paper_2511_16041_b200 as atb
    loss, lse = atb.atb_linear_cross_entropy(s["x"], s["w"], s["labels"], ignore_index=IGNORE)
    if s["step"] != "train":
        return {"loss": loss, "lse": lse}
    dx, dw = atb.atb_linear_cross_entropy_backward(s["dloss"], s["x"], s["w"], s["labels"], lse, ignore_index=IGNORE)
    return {"loss": loss, "lse": lse, "dx": dx, "dw": dw}


def run(state):
    forms = {"norm": _norm_own, "ffn": _ffn_own, "head": _head_own} if own else \
            {"norm": _norm_plain, "ffn": _ffn_plain, "head": _head_plain}
    return forms[state["op"]](state)


# ------------------------------------------------------------------------------------------------ work
def work(case):
    M, train = case["M"], case["step"] == "train"
    if case["op"] == "norm":
        N = case["N"]
        s, w = (2 if case["type"] == BF16 else 4), (2 if case["weights"] == BF16 else 4)
        # forward: x in, y out; training: dy in and dx, dw, db out as well (x once for both)
        return {"bytes": M * N * s * (4 if train else 2) + N * w * (4 if train else 2), "flops": M * N * (20 if train else 8)}
    if case["op"] == "ffn":
        D, F = case["D"], case["F"]
        return {"bytes": 2 * (M * D * (4 if train else 2) + D * F * (6 if train else 3)), "flops": M * D * F * (18 if train else 6)}
    V, D = case["V"], case["D"]
    return {"bytes": 2 * (M * D + V * D) * (2 if train else 1) + M * (20 if train else 16), "flops": M * V * D * (6 if train else 2)}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    train = case["step"] == "train"
    if case["op"] == "norm":
        x, w, b = (s[k].double() for k in ("x", "w", "b"))
        N = case["N"]
        mu = x.sum(1) / N
        var = ((x - mu[:, None]) ** 2).sum(1) / N
        r = (var + s["eps"]) ** -0.5
        z = torch.einsum("mn,m->mn", x - mu[:, None], r)
        out = {"y": torch.addcmul(b, z, w)}
        if train:
            dy = s["dy"].double()
            # dx through the mean and the variance one after the other
            dz = dy * w
            dvar = -0.5 * r ** 3 * (dz * (x - mu[:, None])).sum(1)
            dmu = -(dz.sum(1) * r)
            out["dx"] = dz * r[:, None] + (2.0 / N) * dvar[:, None] * (x - mu[:, None]) + dmu[:, None] / N
            out["dw"] = torch.einsum("mn,mn->n", dy, z)
            out["db"] = torch.einsum("mn->n", dy)
        return out
    if case["op"] == "ffn":
        x, wg, wu, wd = (s[k].double() for k in ("x", "wg", "wu", "wd"))
        g, u = torch.mm(x, wg), torch.mm(x, wu)
        if case["act"] == "silu":
            p = torch.sigmoid(g)
            a, slope = g * p, p + g * p * (1 - p)
        elif case["act"] == "gelu":
            p = 0.5 * torch.erfc(-g / 2 ** 0.5)
            a, slope = g * p, p + g * torch.exp(-g * g / 2) / (2 * math.pi) ** 0.5
        else:
            # x sigmoid(2 z) is x (1 + tanh z) / 2
            z = (2 / math.pi) ** 0.5 * (g + 0.044715 * g ** 3)
            p = torch.sigmoid(2 * z)
            a, slope = g * p, p + g * 2 * p * (1 - p) * (2 / math.pi) ** 0.5 * (1 + 0.134145 * g ** 2)
        out = {"y": torch.mm(a * u, wd)}
        if train:
            dy = s["dy"].double()
            dh = torch.mm(dy, wd.T)
            dg, du = slope * u * dh, a * dh
            out["dx"] = torch.mm(torch.cat([dg, du], 1), torch.cat([wg, wu], 1).T)
            out["dwg"], out["dwu"] = torch.mm(x.T, dg), torch.mm(x.T, du)
            out["dwd"] = torch.mm((a * u).T, dy)
        return out
    x, w, labels = s["x"].double(), s["w"].double(), s["labels"]
    M, V = case["M"], case["V"]
    loss, lse = torch.empty(M, dtype=torch.float64, device="cuda"), torch.empty(M, dtype=torch.float64, device="cuda")
    dx = torch.zeros_like(x) if train else None
    dw = torch.zeros_like(w) if train else None
    rows = max(1, (1 << 28) // V)                      # rows at a time: the logits stay below 2 GB
    for i in range(0, M, rows):
        part, lab = x[i:i + rows], labels[i:i + rows]
        counts = lab != IGNORE
        logits = torch.mm(part, w.T)
        lse[i:i + rows] = torch.logsumexp(logits, 1)
        logp = torch.log_softmax(logits, 1)
        loss[i:i + rows] = torch.where(counts, -logp[torch.arange(len(lab), device="cuda"), lab.clamp(min=0)], 0.0)
        if train:
            d = logp.exp_()
            d[torch.arange(len(lab), device="cuda"), lab.clamp(min=0)] -= 1.0
            d *= torch.where(counts, s["dloss"][i:i + rows].double(), 0.0)[:, None]
            dx[i:i + rows] = torch.mm(d, w)
            dw.addmm_(d.T, part)
    out = {"loss": loss, "lse": lse}
    if train:
        out["dx"], out["dw"] = dx, dw
    return out

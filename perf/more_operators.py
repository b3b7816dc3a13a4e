"""Products with bias, activation and residual, the residual norm, and sampling from logits: what is measured of them.

``run`` computes an operator either in its plain form (elementary torch operations in fp32, in fp64 where a draw's borders
need it, rounded once at the end) or, with ``own`` set, through the library's entry points.  ``exact`` computes the
same from the definitions in 64 bits.
"""
import math

import torch

own = False

BF16, F32 = "bf16", "f32"
TYPES = {BF16: torch.bfloat16, F32: torch.float32}


# ------------------------------------------------------------------------------------------------ cases
def _linear(name, step, M, K, N, act, out=BF16, bias=F32, residual=False, transposed=False):
    return {"name": name, "op": "linear", "step": step, "M": M, "K": K, "N": N, "act": act, "out": out, "bias": bias, "residual": residual,
            "transposed": transposed}


def _norm(name, step, M, N, stream, branch, weights, kind, gate, post, pad=0):
    return {"name": name, "op": "norm", "step": step, "M": M, "N": N, "stream": stream, "branch": branch, "weights": weights, "kind": kind, "gate": gate,
            "post": post, "pad": pad}


def _sample(name, M, V, dtype, temperature, top_k=0, top_p=1.0, min_p=0.0, per_row=False, masked=0.0):
    return {"name": name, "op": "sample", "M": M, "V": V, "type": dtype, "temperature": temperature, "top_k": top_k, "top_p": top_p, "min_p": min_p,
            "per_row": per_row, "masked": masked}


def listed():
    return [
        # one token through a block's last projection while an answer is written, added to the residual stream: latency, memory
        _linear("linear: one token", "forward", 1, 10944, 4096, "none", residual=True),
        # FP32 logits of a few answers from a head that is stored word by word, with a bias
        _linear("linear: logits", "forward", 16, 2048, 32000, "none", out=F32, transposed=True),
        # a prompt of odd length through a block's first projection
        _linear("linear: prompt", "forward", 509, 2048, 5464, "gelu_tanh", bias=BF16),
        # a training step of one card's batch through a block's first projection
        _linear("linear: training step", "train", 8192, 4096, 10944, "gelu"),
        # one token joins the residual stream and is normed again: latency
        _norm("residual norm: one token", "forward", 1, 4096, BF16, BF16, BF16, "rms", True, False),
        # prompts through a network that norms a block's result before it is added and after
        _norm("residual norm: prompts", "forward", 8192, 4096, BF16, BF16, BF16, "rms", False, True),
        # a small model's step with an FP32 stream of odd width, rows a slice of a wider buffer
        _norm("residual norm: odd training step", "train", 1021, 1001, F32, BF16, F32, "layer", True, True, pad=6),
        # a training step of a wide model with a gate
        _norm("residual norm: wide training step", "train", 16384, 8192, BF16, BF16, F32, "layer", True, False),
        # one answer's next word from a large vocabulary: latency
        _sample("sample: one answer", 1, 131072, F32, 0.8, top_k=50, top_p=0.95),
        # a few answers from bf16 logits, where many words tie
        _sample("sample: few answers", 16, 32000, BF16, 0.7, top_p=0.9),
        # a server's batch: every request with its own settings, some of them greedy, an odd vocabulary, forbidden words
        _sample("sample: batch", 64, 50003, F32, 1.0, top_k=100, top_p=0.95, min_p=0.02, per_row=True, masked=0.1),
        # answers drawn for training
        _sample("sample: many answers", 512, 131072, F32, 1.0, top_p=0.99),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _eights(rng, low, high):
    return 8 * _log_int(rng, low // 8, high // 8)


def draw(rng):
    op = rng.choice(["linear", "norm", "sample"])
    step = rng.choice(["forward", "train"])
    if op == "linear":
        act = rng.choice(["none", "relu", "silu", "gelu", "gelu_tanh"])
        transposed = rng.random() < 0.3
        c = _linear("", step, _log_int(rng, 1, 8192), _eights(rng, 512, 4096), _eights(rng, 1024, 10944), act, rng.choice([BF16, BF16, F32]),
                    rng.choice([BF16, F32, ""]), rng.random() < 0.4, transposed)
    elif op == "norm":
        stream = rng.choice([BF16, F32])
        branch = rng.choice([BF16, stream])
        c = _norm("", step, _log_int(rng, 1, 16384), _log_int(rng, 64, 8192), stream, branch, rng.choice([BF16, F32]), rng.choice(["layer", "rms"]),
                  rng.random() < 0.5, rng.random() < 0.5, rng.choice([0, 0, 8, 5]))
    else:
        per_row = rng.random() < 0.3
        c = _sample("", _log_int(rng, 1, 512), _log_int(rng, 1000, 131072), rng.choice([BF16, F32]), round(rng.uniform(0.3, 1.5), 2),
                    rng.choice([0, 0, _log_int(rng, 1, 200)]), rng.choice([1.0, round(rng.uniform(0.5, 0.99), 2)]),
                    rng.choice([0.0, 0.0, round(rng.uniform(0.01, 0.2), 3)]), per_row, rng.choice([0.0, 0.1, 0.6]))
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0, shift=0.0, dtype=torch.bfloat16):
        return torch.randn(shape, generator=gen, device="cuda").mul_(scale).add_(shift).to(dtype)

    def uniform(*shape, dtype=torch.float32):
        return torch.rand(shape, generator=gen, device="cuda", dtype=dtype)

    s = dict(case)
    M = case["M"]
    if case["op"] == "linear":
        K, N, out = case["K"], case["N"], TYPES[case["out"]]
        s["x"] = normal(M, K)
        s["w"] = normal(N, K, scale=1.0 / math.sqrt(K)).t() if case["transposed"] else normal(K, N, scale=1.0 / math.sqrt(K))
        s["b"] = normal(N, scale=0.2, dtype=TYPES[case["bias"]]) if case["bias"] else None
        s["r"] = normal(M, N, dtype=out) if case["residual"] else None
        if case["step"] == "train":
            s["dy"] = normal(M, N, scale=1e-2, dtype=out)
    elif case["op"] == "norm":
        N, stream, branch, weights = case["N"], TYPES[case["stream"]], TYPES[case["branch"]], TYPES[case["weights"]]

        def rows(dtype, scale, big):
            # a few columns of a residual stream are much larger than the others
            v = torch.randn((M, N + case["pad"]), generator=gen, device="cuda") * scale
            v = v * (1.0 + big * (uniform(1, N + case["pad"]) > 0.995)) + 0.25 * scale
            return v.to(dtype)[:, :N]

        s["x"], s["f"] = rows(stream, 1.0, 6.0), rows(branch, 0.5, 2.0)
        s["w"] = normal(N, scale=0.1, shift=1.0, dtype=weights)
        s["b"] = normal(N, scale=0.1, dtype=weights) if case["kind"] == "layer" else None
        s["g"] = normal(N, scale=0.2, shift=0.5, dtype=weights) if case["gate"] else None
        s["pw"] = normal(N, scale=0.1, shift=1.0, dtype=weights) if case["post"] else None
        s["pb"] = normal(N, scale=0.1, dtype=weights) if case["post"] and case["kind"] == "layer" else None
        s["scale"] = 1.25
        s["eps"] = 1e-5
        if case["step"] == "train":
            s["dz"], s["dh"] = normal(M, N, dtype=branch), normal(M, N, dtype=stream)
    else:
        V = case["V"]
        x = torch.randn((M, V), generator=gen, device="cuda").mul_(2.0)
        # the words that a model has in mind
        at = torch.randint(0, V, (M, 40), generator=gen, device="cuda")
        x.scatter_add_(1, at, 10.0 * uniform(M, 40))
        if case["masked"]:
            x.masked_fill_(uniform(M, V) < case["masked"], -math.inf)
        s["x"] = x.to(TYPES[case["type"]])
        s["u"] = uniform(M)
        if case["per_row"]:
            greedy = uniform(M) < 0.1
            s["temperature"] = torch.where(greedy, torch.zeros_like(s["u"]), case["temperature"] * (0.5 + uniform(M)))
            s["top_k"] = torch.randint(0, max(case["top_k"], 1) + 1, (M,), generator=gen, device="cuda", dtype=torch.int32)
            s["top_p"] = 1.0 - (1.0 - case["top_p"]) * 2.0 * uniform(M)
            s["min_p"] = case["min_p"] * 2.0 * uniform(M)
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _act_plain(z, act):
    """act(z) and act'(z)."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z * (z > 0), (z > 0).float()
    if act == "silu":
        sig = 1.0 / (1.0 + torch.exp(-z))
        return z * sig, sig * (1.0 + z * (1.0 - sig))
    if act == "gelu":
        phi = 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
        return z * phi, phi + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    c = math.sqrt(2.0 / math.pi)
    t = torch.tanh(c * (z + 0.044715 * z * z * z))
    return 0.5 * z * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3.0 * 0.044715 * z * z)


def _linear_plain(s):
    x, w, out_type = s["x"].float(), s["w"].float(), TYPES[s["out"]]
    z = x @ w
    if s["b"] is not None:
        z = z + s["b"].float()
    a, slope = _act_plain(z, s["act"])
    y = a if s["r"] is None else a + s["r"].float()
    out = {"y": y.to(out_type)}
    if s["step"] == "train":
        dz = s["dy"].float() * slope
        out["dx"] = (dz @ w.t()).bfloat16()
        out["dw"] = (x.t() @ dz).bfloat16()
        if s["b"] is not None:
            out["db"] = dz.sum(0).to(s["b"].dtype)
    return out


def _normed(v, kind, eps):
    """norm(v) and 1 / its spread."""
    d = v - v.mean(1, keepdim=True) if kind == "layer" else v
    r = torch.rsqrt((d * d).mean(1, keepdim=True) + eps)
    return d * r, r


def _normed_backward(g, n, r, kind):
    out = g - n * (g * n).mean(1, keepdim=True)
    return r * (out - g.mean(1, keepdim=True)) if kind == "layer" else r * out


def _norm_plain(s):
    kind, eps, stream, branch = s["kind"], s["eps"], s["x"].dtype, s["f"].dtype
    x, f, w = s["x"].float(), s["f"].float(), s["w"].float()
    u = f
    if s["pw"] is not None:
        fn, fr = _normed(f, kind, eps)
        u = fn * s["pw"].float()
        if s["pb"] is not None:
            u = u + s["pb"].float()
    h = s["scale"] * x + (u if s["g"] is None else s["g"].float() * u)
    hn, hr = _normed(h, kind, eps)
    z = hn * w
    if s["b"] is not None:
        z = z + s["b"].float()
    out = {"h": h.to(stream), "z": z.to(branch)}
    if s["step"] == "train":
        dz = s["dz"].float()
        t = s["dh"].float() + _normed_backward(dz * w, hn, hr, kind)
        out["dx"] = (s["scale"] * t).to(stream)
        du = t
        if s["g"] is not None:
            out["dgate"] = (t * u).sum(0).to(s["g"].dtype)
            du = t * s["g"].float()
        if s["pw"] is not None:
            out["dpw"] = (du * fn).sum(0).to(s["pw"].dtype)
            if s["pb"] is not None:
                out["dpb"] = du.sum(0).to(s["pb"].dtype)
            du = _normed_backward(du * s["pw"].float(), fn, fr, kind)
        out["df"] = du.to(branch)
        out["dw"] = (dz * hn).sum(0).to(s["w"].dtype)
        if s["b"] is not None:
            out["db"] = dz.sum(0).to(s["b"].dtype)
    return out


def _column(v, like):
    """A setting of every row, or one for all, as a column in 64 bits."""
    return v.double()[:, None] if torch.is_tensor(v) else torch.full((like.shape[0], 1), float(v), dtype=torch.float64, device=like.device)


def _sample_plain(s):
    x = s["x"].double()
    M, V = x.shape
    t, k, p, least = (_column(s[n], x) for n in ("temperature", "top_k", "top_p", "min_p"))
    greedy = t <= 0
    t = torch.where(greedy, torch.ones_like(t), t)
    k = torch.where(k <= 0, torch.full_like(k, V), k)
    k = torch.where(greedy, torch.ones_like(k), k)
    top, order = torch.sort(x, dim=1, descending=True, stable=True)
    weight = torch.exp((top - top[:, :1]) / t)
    rank = torch.arange(V, device=x.device, dtype=torch.float64)[None]
    weight = torch.where(rank < k, weight, torch.zeros_like(weight))
    before = torch.cumsum(weight, 1) - weight
    weight = torch.where((before < p * weight.sum(1, keepdim=True)) & (weight >= least), weight, torch.zeros_like(weight))
    del before
    # back to the vocabulary's order
    weight = torch.zeros_like(x).scatter_(1, order, weight)
    total = torch.cumsum(weight, 1)
    token = (total <= _column(s["u"], x) * total[:, -1:]).sum(1, keepdim=True).clamp(max=V - 1)
    return {"tokens": token[:, 0], "probs": (weight.gather(1, token) / total[:, -1:])[:, 0].float()}


# ------------------------------------------------------------------------------------------------ the library's calls
def _linear_own(s):
    import paper_2511_16041_b200 as atb
    act, out_type = s["act"], TYPES[s["out"]]
    if s["step"] != "train":
        return {"y": atb.atb_linear(s["x"], s["w"], s["b"], act=act, residual=s["r"], dtype=out_type)}
    y, z = atb.atb_linear(s["x"], s["w"], s["b"], act=act, residual=s["r"], dtype=out_type, save=True)
    wanted = False if s["b"] is None else torch.empty_like(s["b"])
    dx, dw, db = atb.atb_linear_backward(s["dy"], s["x"], s["w"], z, act=act, dbias=wanted)
    out = {"y": y, "dx": dx, "dw": dw}
    if db is not None:
        out["db"] = db
    return out


def _norm_own(s):
    import paper_2511_16041_b200 as atb
    given = dict(gate=s["g"], scale=s["scale"], post_norm=s["pw"] is not None, post_W=s["pw"], post_B=s["pb"], kind=s["kind"])
    h, z, stats = atb.atb_residual_norm(s["x"], s["f"], s["w"], s["b"], eps=s["eps"], **given)
    out = {"h": h, "z": z}
    if s["step"] == "train":
        no = {} if s["b"] is not None else {"dB": False}
        if s["pb"] is None:
            no["dpost_B"] = False
        dx, df, dgate, dw, db, dpw, dpb = atb.atb_residual_norm_backward(s["dz"], s["dh"], s["x"], s["f"], stats, s["w"], **given, **no)
        out.update({k: v for k, v in (("dx", dx), ("df", df), ("dgate", dgate), ("dw", dw), ("db", db), ("dpw", dpw), ("dpb", dpb)) if v is not None})
    return out


def _sample_own(s):
    import paper_2511_16041_b200 as atb
    tokens, probs = atb.atb_sample(s["x"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
    return {"tokens": tokens, "probs": probs}


def run(state):
    forms = {"linear": _linear_own, "norm": _norm_own, "sample": _sample_own} if own else \
            {"linear": _linear_plain, "norm": _norm_plain, "sample": _sample_plain}
    return forms[state["op"]](state)


# ------------------------------------------------------------------------------------------------ work
def work(case):
    M, size = case["M"], {BF16: 2, F32: 4, "": 0}
    train = case.get("step") == "train"
    if case["op"] == "linear":
        K, N, out, bias = case["K"], case["N"], size[case["out"]], size[case["bias"]]
        moved = 2 * M * K + 2 * K * N + N * bias + M * N * out * (2 if case["residual"] else 1)
        if train:                          # dy in; dx, dw, db out
            moved += M * N * out + 2 * M * K + 2 * K * N + N * bias
        return {"bytes": moved, "flops": 2 * M * K * N * (3 if train else 1)}
    if case["op"] == "norm":
        N, stream, branch = case["N"], size[case["stream"]], size[case["branch"]]
        vectors = size[case["weights"]] * N * (1 + case["gate"] + case["post"] + (case["kind"] == "layer") * (1 + case["post"]))
        # x, f in, h, z out; training: dz, dh in, dx, df out
        return {"bytes": (2 if train else 1) * (2 * M * N * (stream + branch) + vectors), "flops": M * N * (50 if train else 20)}
    return {"bytes": M * case["V"] * size[case["type"]] + M * (4 + 12 + (16 if case["per_row"] else 0)), "flops": M * case["V"] * 10}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _exact_linear(s):
    x, w = s["x"].double(), s["w"].double()
    z = torch.mm(x, w) if s["b"] is None else torch.addmm(s["b"].double(), x, w)
    act = s["act"]
    if act == "none":
        a, slope = z, torch.ones((), dtype=z.dtype, device=z.device)
    elif act == "relu":
        a, slope = torch.clamp(z, min=0.0), torch.where(z > 0, 1.0, 0.0).to(z.dtype)
    else:
        if act == "silu":
            q, dq = torch.sigmoid(z), None
        elif act == "gelu":
            q, dq = 0.5 * torch.erfc(-z / 2 ** 0.5), torch.exp(-z * z / 2) / (2 * math.pi) ** 0.5
        else:
            # z (1 + tanh v) / 2 is z sigmoid(2 v)
            q = torch.sigmoid(2 * (2 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3))
            dq = q * (1 - q) * 2 * (2 / math.pi) ** 0.5 * (1 + 0.134145 * z ** 2)
        if dq is None:
            dq = q * (1 - q)
        a, slope = z * q, q + z * dq
    out = {"y": a if s["r"] is None else torch.add(a, s["r"].double())}
    if s["step"] == "train":
        dz = torch.mul(s["dy"].double(), slope)
        out["dx"], out["dw"] = torch.mm(dz, w.T), torch.mm(x.T, dz)
        if s["b"] is not None:
            out["db"] = torch.einsum("mn->n", dz)
    return out


def _exact_norm(s):
    layer, eps, N = s["kind"] == "layer", s["eps"], s["N"]

    def norm(v):
        c = v - (v.sum(1) / N)[:, None] if layer else v
        r = (torch.einsum("mn,mn->m", c, c) / N + eps) ** -0.5
        return c, r

    def back(g, c, r):
        # through the spread, then through the centre
        dc = g * r[:, None] - c * (torch.einsum("mn,mn->m", g, c) * r ** 3 / N)[:, None]
        return dc - (dc.sum(1) / N)[:, None] if layer else dc

    x, f, w = s["x"].double(), s["f"].double(), s["w"].double()
    gate = torch.ones_like(w) if s["g"] is None else s["g"].double()
    u = f
    if s["pw"] is not None:
        cf, rf = norm(f)
        u = torch.einsum("mn,m,n->mn", cf, rf, s["pw"].double())
        if s["pb"] is not None:
            u = torch.add(u, s["pb"].double())
    h = torch.addcmul(s["scale"] * x, u, gate)
    ch, rh = norm(h)
    z = torch.einsum("mn,m,n->mn", ch, rh, w)
    out = {"h": h, "z": z if s["b"] is None else torch.add(z, s["b"].double())}
    if s["step"] == "train":
        dz = s["dz"].double()
        t = torch.add(s["dh"].double(), back(dz * w, ch, rh))
        out["dx"] = s["scale"] * t
        if s["g"] is not None:
            out["dgate"] = torch.einsum("mn,mn->n", t, u)
        du = t * gate
        if s["pw"] is not None:
            out["dpw"] = torch.einsum("mn,mn,m->n", du, cf, rf)
            if s["pb"] is not None:
                out["dpb"] = torch.einsum("mn->n", du)
            du = back(du * s["pw"].double(), cf, rf)
        out["df"] = du
        out["dw"] = torch.einsum("mn,mn,m->n", dz, ch, rh)
        if s["b"] is not None:
            out["db"] = torch.einsum("mn->n", dz)
    return out


def _exact_sample(s):
    """Row by row: the words in order, the first n of them by each of the settings, and the draw among those."""
    tokens, probs = [], []
    for m in range(s["M"]):
        at = lambda name: float(s[name][m]) if torch.is_tensor(s[name]) else float(s[name])  # noqa: E731
        t, k, p, least = at("temperature"), int(at("top_k")), at("top_p"), at("min_p")
        logits = s["x"][m].double()
        # rising by the negative logit; a stable sort keeps the vocabulary's order among equals
        falling, order = torch.sort(-logits, stable=True)
        if t <= 0:
            tokens.append(order[0])
            probs.append(torch.ones((), dtype=torch.float64, device=logits.device))
            continue
        weight = torch.softmax(-falling / t, 0)
        n = k if 0 < k < len(weight) else len(weight)
        weight = weight[:n]
        reach = torch.searchsorted(weight.cumsum(0), p * weight.sum()) + 1     # the word that takes the sum to p is in
        n = min(n, int(reach)) if p < 1 else n
        n = min(n, int((weight / weight[0] >= least).sum()))
        kept, by_word = torch.sort(order[:n])
        run = weight[:n][by_word].cumsum(0)
        j = min(int(torch.searchsorted(run, at("u") * run[-1], right=True)), n - 1)
        tokens.append(kept[j])
        probs.append(weight[:n][by_word][j] / run[-1])
    return {"tokens": torch.stack(tokens), "probs": torch.stack(probs)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "norm": _exact_norm, "sample": _exact_sample}[case["op"]](s)

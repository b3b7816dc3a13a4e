"""Sampling against its definition in 64 bits: sort, keep, and walk the vocabulary.

Tokens have to be equal.  Weights are exact to 2^-46 of the largest, so that a draw could fall otherwise only where u is within about V * 2^-46 of a
border: with these sizes and seeds below 1e-8 per row.  Probabilities are rounded once to FP32 (U32), from weights that are off by 2^-46 at most."""
import math

import pytest
import torch

import paper_2511_16041_b200 as atb
from tests.operators_ref import U32

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
INF, NAN = math.inf, math.nan


def reference(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Tokens and probabilities (double), and how many words are kept."""
    x = x.double()
    x = torch.where(x.isnan(), torch.full_like(x, -INF), x)
    M, V = x.shape
    col = lambda v: v.double()[:, None] if torch.is_tensor(v) else torch.full((M, 1), float(v), dtype=torch.float64, device=x.device)  # noqa: E731
    t, k, p, least, u = col(temperature), col(top_k), col(top_p), col(min_p), col(u)
    greedy = ~(t > 0)
    k = torch.where((k <= 0) | (k > V), torch.full_like(k, V), k)
    k = torch.where(greedy, torch.ones_like(k), k)
    top, order = torch.sort(x, dim=1, descending=True, stable=True)
    first = top[:, :1]
    w = torch.exp((top - first) / torch.where(greedy, torch.ones_like(t), t))
    w = torch.where(top == first, torch.ones_like(w), torch.where(top == -INF, torch.zeros_like(w), w.nan_to_num(0.0)))
    w = torch.where(first == -INF, torch.zeros_like(w), w)
    rank = torch.arange(V, device=x.device)[None]
    w = torch.where(rank < k, w, torch.zeros_like(w))
    before = w.cumsum(1) - w
    off = ~(p < 1) | greedy
    keep = (off | (before < p * w.sum(1, keepdim=True)) | (rank == 0)) & ((w >= least.clamp(max=1.0)) | ~(least > 0))
    w = torch.where(keep, w, torch.zeros_like(w))
    kept = (w > 0).sum(1)
    w = torch.zeros_like(w).scatter(1, order, w)
    run = w.cumsum(1)
    total = run[:, -1:]
    target = torch.where(u > 0, u, torch.zeros_like(u)) * total
    token = (run <= target).sum(1, keepdim=True)
    # u = 1: the last kept word
    last = V - 1 - (w.flip(1) > 0).to(torch.int8).argmax(1, keepdim=True)
    token = torch.minimum(token, last)
    prob = (w.gather(1, token) / total)[:, 0]
    none = total[:, 0] == 0
    return torch.where(none, torch.full_like(token[:, 0], -1), token[:, 0]), torch.where(none, torch.zeros_like(prob), prob), kept


def compare(x, u, **settings):
    tokens, probs = atb.atb_sample(x, u, **settings)
    want, p, kept = reference(x, u, **settings)
    bad = (tokens != want).nonzero()[:, 0].tolist()
    assert not bad, [(i, int(tokens[i]), int(want[i]), int(kept[i]), float(p[i])) for i in bad[:5]]
    over = (probs.double() - p).abs() - (U32 * p + 2.0 ** -44)
    assert float(over.max()) <= 0, (float(over.max()), int(over.argmax()))
    return tokens, probs


def logits(M, V, dtype=F32, seed=0, spread=2.0, pad=0):
    gen = torch.Generator(device="cuda").manual_seed(300 + seed)
    x = torch.randn((M, V + pad), generator=gen, device="cuda") * spread
    x[:, :: max(1, V // 20)] += 8 * torch.rand((M, 1), generator=gen, device="cuda")
    return x.to(dtype)[:, :V], torch.rand(M, generator=gen, device="cuda")


SETTINGS = [dict(), dict(top_k=1), dict(top_k=50), dict(top_p=0.9), dict(min_p=0.05), dict(temperature=0.7, top_k=200, top_p=0.95),
            dict(temperature=1.4, top_p=0.99, min_p=0.001), dict(temperature=0.5, top_k=7, min_p=0.2), dict(temperature=0.0, top_p=0.5), dict(top_k=3, top_p=0.3, min_p=0.1)]
WORDS = [1, 2, 7, 31, 100, 1000, 1001, 4096, 16384, 16385, 32000, 50003, 65537, 131072, 131073, 300001]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", WORDS)
def test_vocabularies(V, dtype):
    for i, s in enumerate(SETTINGS):
        x, u = logits(5, V, dtype, seed=V + i)
        compare(x, u, **s)


@pytest.mark.parametrize("M", [1, 2, 64, 300])
@pytest.mark.parametrize("settings", SETTINGS)
def test_rows(M, settings):
    x, u = logits(M, 20000, (F32, BF16)[M % 2], seed=M)
    compare(x, u, **settings)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad,skip", [(1, 0), (3, 3), (8, 5), (0, 0), (7, 1)])
def test_strides_and_alignment(dtype, pad, skip):
    gen = torch.Generator(device="cuda").manual_seed(8)
    base = (torch.randn((9, 33000 + pad), generator=gen, device="cuda") * 2).to(dtype)
    x = base[:, skip:skip + 33000 - skip]
    compare(x, torch.rand(9, generator=gen, device="cuda"), top_k=40, top_p=0.9)
    compare(x, torch.rand(9, generator=gen, device="cuda"), top_p=0.99)


@pytest.mark.parametrize("V", [50, 1000, 40000])
def test_every_row_its_own_settings(V):
    x, u = logits(200, V, F32, seed=4)
    gen = torch.Generator(device="cuda").manual_seed(4)
    r = lambda: torch.rand(200, generator=gen, device="cuda")  # noqa: E731
    t, p, least = 0.3 + 1.2 * r(), r() * 1.2, r() * 0.3 - 0.1
    k = torch.randint(-3, 60, (200,), generator=gen, device="cuda", dtype=torch.int32)
    t[::7], t[3], t[5] = 0.0, -1.0, NAN
    p[11], least[12], p[13], least[14] = NAN, NAN, -0.5, 3.0
    compare(x, u, temperature=t, top_k=k, top_p=p, min_p=least)
    compare(x, u.double(), temperature=0.9, top_k=k, top_p=p)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_ties(dtype):
    """Few values, so that every border falls among equals: the lowest indices are kept."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    for V in (40, 3000, 70000):
        x = torch.randint(-3, 4, (12, V), generator=gen, device="cuda").to(dtype)
        u = torch.rand(12, generator=gen, device="cuda")
        for s in (dict(top_k=V // 3), dict(top_k=5), dict(top_p=0.5), dict(top_p=0.93, top_k=V // 2), dict(min_p=0.3), dict(min_p=1.0), dict(top_p=0.0), dict(top_k=1)):
            compare(x, u, **s)


def test_one_value():
    """All logits alike: weights and sums are whole numbers, and the borders exact."""
    for V in (8, 1000, 40000):
        x = torch.full((6, V), 1.5, device="cuda")
        u = torch.tensor([0.0, 0.25, 0.5, 0.75, 1 - 2.0 ** -24, 1.0], device="cuda")
        assert atb.atb_sample(x, u)[0].tolist() == [0, V // 4, V // 2, 3 * V // 4, math.floor((1 - 2.0 ** -24) * V), V - 1]
        # half of the weight: the first half of the words
        assert atb.atb_sample(x, u, top_p=0.5)[0].tolist() == [0, V // 8, V // 4, 3 * V // 8, V // 2 - 1, V // 2 - 1]
        tokens, probs = atb.atb_sample(x, u, top_k=4)
        assert tokens.tolist() == [0, 1, 2, 3, 3, 3] and probs.tolist() == [0.25] * 6


def test_random_numbers_outside_their_range():
    x, _ = logits(6, 5000)
    u = torch.tensor([-1.0, NAN, 0.0, 1.0, 7.0, INF], device="cuda")
    compare(x, torch.where(u.isnan(), torch.zeros_like(u), u).clamp(0, 1))
    got = atb.atb_sample(x, u)[0]
    want = atb.atb_sample(x, torch.tensor([0.0, 0.0, 0.0, 1.0, 1.0, 1.0], device="cuda"))[0]
    assert torch.equal(got, want)


@pytest.mark.parametrize("V", [33, 5000, 40000, 140000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_masked_and_infinite_logits(V, dtype):
    x, u = logits(16, V, dtype, seed=9)
    x[0] = -INF
    x[1] = NAN
    x[2], x[2, V // 2] = -INF, -3.0
    x[3, : V // 2] = -INF
    x[4, 1::2] = NAN
    x[5, 3] = x[5, V - 1] = INF
    x[6, 2], x[6, 5] = INF, NAN
    x[7] = torch.finfo(dtype).min
    x[8], x[8, 7] = torch.finfo(dtype).min, torch.finfo(dtype).max
    x[9] = -0.0
    x[9, ::3] = 0.0
    x[10] = x[10] * 1e-30
    x[11] = x[11] * 1e30
    x[12, 5:] = -INF
    for s in (dict(), dict(top_k=4), dict(top_p=0.6), dict(top_k=30, top_p=0.8, min_p=0.01), dict(temperature=0.0), dict(temperature=INF), dict(temperature=1e-4), dict(min_p=1.0),
              dict(temperature=INF, top_k=9), dict(temperature=1e30, top_p=0.5), dict(temperature=1e38, top_p=0.7), dict(temperature=1e38, top_k=V // 3)):
        tokens, probs = compare(x, u, **s)
        assert tokens[:3].tolist() == [-1, -1, V // 2] and probs[:3].tolist() == [0.0, 0.0, 1.0]


def test_the_weights_floor():
    """What weighs less than 2^-46 of the largest is not drawn, however small u is; what weighs more is."""
    x = torch.full((2, 100), -200.0, device="cuda")
    x[:, 50] = 0.0
    x[1, 3] = -30.0                                           # e^-30 = 2^-43.3
    tokens, probs = atb.atb_sample(x, torch.zeros(2, device="cuda"))
    assert tokens.tolist() == [50, 3]


def test_the_drawn_distribution():
    """u on an even grid: every word comes up in proportion to its probability, within one."""
    x, _ = logits(1, 300, spread=1.5)
    n = 4096
    u = (torch.arange(n, device="cuda").double() + 0.5) / n
    for s in (dict(), dict(temperature=0.6, top_k=20), dict(top_p=0.8), dict(min_p=0.1)):
        tokens, probs = atb.atb_sample(x.expand(n, 300).contiguous(), u, **s)
        counts = torch.bincount(tokens, minlength=300)
        for word in counts.nonzero()[:, 0].tolist():
            p = float(probs[tokens == word][0])
            assert abs(float(counts[word]) - n * p) <= 1.001
        assert abs(sum(float(probs[tokens == w][0]) for w in counts.nonzero()[:, 0].tolist()) - 1) <= 300 / n + 1e-6


def test_places_streams_and_graphs():
    x, u = logits(40, 32000)
    want, p = atb.atb_sample(x, u, top_p=0.9)
    tokens, probs = torch.full((41,), 7, device="cuda"), torch.full((41,), 7.0, device="cuda")
    got = atb.atb_sample(x, u, top_p=0.9, tokens=tokens[:40], probs=probs[:40])
    assert torch.equal(got[0], want) and torch.equal(got[1], p) and int(tokens[40]) == 7 and float(probs[40]) == 7
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = atb.atb_sample(x, u, top_p=0.9, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want) and torch.equal(got[1], p)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = atb.atb_sample(x, u, top_p=0.9)
    for seed in (1, 2, 3):
        x2, u2 = logits(40, 32000, seed=seed)
        x.copy_(x2)
        u.copy_(u2)
        graph.replay()
        torch.cuda.synchronize()
        again = atb.atb_sample(x2, u2, top_p=0.9)
        assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])

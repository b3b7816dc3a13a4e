"""Sampling where a border or a draw hangs on the weights' and the borders' own arithmetic."""
import math

import pytest
import torch

import paper_2511_16041_b200 as atb
from tests.test_gpu_sample import compare

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1e-47, 2e-47, 1e-46, 1e-45, 1e-30])
@pytest.mark.parametrize("settings", [dict(), dict(top_k=5), dict(top_k=300), dict(top_p=0.9), dict(top_k=300, top_p=0.5), dict(min_p=0.01)])
@pytest.mark.parametrize("V", [40, 5000, 40000])
def test_temperatures_near_the_least_distance_of_logits(V, settings, T):
    """The largest logit is 0, subnormal or little more, and its neighbour may lie one subnormal number below it."""
    gen = torch.Generator(device="cuda").manual_seed(V)
    x = -torch.rand((6, V), generator=gen, device="cuda") - 1e-3
    at = torch.randint(0, V, (6,), generator=gen, device="cuda")
    x[torch.arange(6), at] = 0.0
    x[1] *= 1e-36
    x[2] *= 1e-40
    x[3, (int(at[3]) + 7) % V] = -2.0 ** -149
    x[4] -= 2.0 ** -126
    x[5] += 2.0 ** -120
    compare(x, torch.rand(6, generator=gen, device="cuda"), temperature=T, **settings)


# A temperature at which a logit is its word's power of 2.
POWERS = 1.4426950408889634


def test_weights_that_round_to_nothing():
    """2^25 words, units of 2^-37: 2^-38.001 rounds to 0, and 2^-13 of the largest weight with it, in all.  The largest word alone reaches the goal,
    which is a millionth of its weight below it; all other weights are whole numbers of units."""
    V = 1 << 25
    x = torch.full((1, V), -38.001, device="cuda")
    x[0, 10], x[0, 20] = 0.0, -14.0
    x[0, 30:62] = -15.0
    p = 2 ** 37 / (2 ** 37 + 2 ** 23 + 32 * 2 ** 22) * (1 - 1e-6)
    for u in (0.0, 0.5, 0.99999):
        tokens, probs = atb.atb_sample(x, torch.tensor([u], device="cuda", dtype=torch.float64), temperature=POWERS, top_p=p)
        assert int(tokens) == 10 and float(probs) == 1.0


def test_weights_that_round_to_a_unit():
    """2^29 words, units of 2^-33: 2^-33.999 rounds to one, and all of them weigh 1/16 of the largest instead of 1/32.  Sums are whole numbers of units,
    and what is kept is the largest word and the first few per cent of the others."""
    V = 1 << 29
    x = torch.full((2, V), -34.0, device="cuda", dtype=torch.bfloat16)
    x[:, 0] = 0.0
    p, u = 0.945, torch.tensor([0.0, 0.9999], device="cuda", dtype=torch.float64)
    tokens, probs = atb.atb_sample(x, u, temperature=POWERS * 34.0 / 33.999, top_p=p, min_p=1e-12)
    goal = p * float(2 ** 33 + V - 1)
    total = 2 ** 33 + math.ceil(goal - 2.0 ** 33)
    # the word behind the largest that u lies in; the j-th of them has 2^33 + j units up to its own
    target = int(float(u[1]) * float(total)) + 1
    assert tokens.tolist() == [0, target - 2 ** 33]
    want = torch.tensor([2.0 ** 33 / total, 1.0 / total], dtype=torch.float64).float()
    assert torch.equal(probs.cpu(), want)


@pytest.mark.parametrize("V", [1000, 131072, 500000])
@pytest.mark.parametrize("top_k", [0, 1, 4, 300])
@pytest.mark.parametrize("top_p", [-math.inf, -1.0, 0.0])
def test_top_p_of_nothing_and_less(V, top_k, top_p):
    """The first word in the order is kept, also where top-k cuts through so many equals that what it leaves is lost in the weight of all."""
    x = torch.zeros((3, V), device="cuda")
    x[1, :V // 2] = -1.0
    u = torch.tensor([0.0, 0.5, 0.999], device="cuda")
    for p in (top_p, torch.full((3,), top_p, device="cuda")):
        tokens, probs = atb.atb_sample(x, u, top_k=top_k, top_p=p)
        assert tokens.tolist() == [0, V // 2, 0] and probs.tolist() == [1.0] * 3

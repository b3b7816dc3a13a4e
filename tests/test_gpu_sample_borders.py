"""Sampling where a border or a draw hangs on the weights' and the borders' own arithmetic."""
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

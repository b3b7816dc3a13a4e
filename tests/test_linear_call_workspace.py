"""What one call of the linear layer's backward pass takes of its workspace: host arithmetic."""
import pytest

import paper_2511_16041_b200 as atb

F32, BF16 = 0, 1
SHAPES = [(1, 8, 8), (3, 1024, 2736), (16, 2048, 32000), (500, 1024, 2736), (8192, 4096, 10944)]


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_a_call_takes_what_it_uses(M, K, N, layout):
    most = atb.atb_linear_backward_workspace_bytes(M, K, N)
    need = lambda act, y, *wanted: atb.atb_linear_backward_call_workspace_bytes(M, K, N, act, y, layout, *wanted)  # noqa: E731
    dz = -(-2 * M * N // 256) * 256
    for wanted in ((1, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 0), (0, 1, 1)):
        for act, y in (("gelu", BF16), ("relu", F32), (None, F32), (None, BF16)):
            is_dy, products = act is None and y == BF16, wanted[0] or wanted[1]
            n = need(act, y, *wanted)
            assert n <= most and n == need(None, BF16, *wanted) + (dz if products and not is_dy else 0)
    assert need(None, BF16, 0, 0, 0) == 0 and 0 < need("silu", BF16, 0, 0, 1) < dz + 4 * 592 * N + 512
    assert need(None, BF16, 1, 1, 1) - need(None, BF16, 1, 1, 0) == need("gelu", F32, 0, 0, 1)      # the sums over rows
    assert atb.atb_linear_backward_call_workspace_bytes(0, K, N, None, BF16, layout) == 0


def test_a_projection_without_an_activation():
    """8192 x 4096 x 10944, no product of which is split: nothing at all without a bias, and never room for dZ."""
    need = lambda *w: atb.atb_linear_backward_call_workspace_bytes(8192, 4096, 10944, None, BF16, 0, *w)  # noqa: E731
    assert need(True, True, False) == 0 and need() < 4 * 592 * 10944

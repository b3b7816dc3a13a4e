"""The smoke run reaches the operators between the products beside the GEMM kernels."""
import pytest

import __graft_entry__

pytestmark = pytest.mark.gpu


def test_smoke_runs_everything(capsys):
    __graft_entry__.smoke()
    out = capsys.readouterr().out
    for part in ("tiling (128, 128, 64, 128) ok", "CTA-pair tiling and BFP16 output ok", "head loss and gradients of 1 token ok",
                 "head loss and gradients of 40 tokens ok"):
        assert part in out

"""Linear layer, residual norm and sampling: what the binding refuses on a GPU, calls on other streams, two calls at once, repeated bits."""
import pytest
import torch

import paper_2511_16041_b200 as atb

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def _t(*shape, dtype=BF16):
    return torch.randn(shape, device="cuda").to(dtype)


def _status(call):
    with pytest.raises(atb.AtbError) as e:
        call()
    return e.value.status


def test_linear_refusals():
    x, w, b, dy = _t(4, 16), _t(16, 24), _t(24), _t(4, 24)
    Y, Z = atb.atb_linear(x, w, b, act="silu", save=True)
    for call in (lambda: atb.atb_linear(x.float(), w), lambda: atb.atb_linear(x, w.float()), lambda: atb.atb_linear(x, _t(24, 16)), lambda: atb.atb_linear(x[0], w),
                 lambda: atb.atb_linear(x, _t(16, 48)[:, ::2]),                   # neither rows nor columns contiguous
                 lambda: atb.atb_linear(x, w, b.half()), lambda: atb.atb_linear(x, w, b[:8]), lambda: atb.atb_linear(x, w, b.cpu()),
                 lambda: atb.atb_linear(x, w, residual=x), lambda: atb.atb_linear(x, w, residual=dy.float(), dtype=BF16),
                 lambda: atb.atb_linear(x, w, dtype=torch.float16), lambda: atb.atb_linear(x, w, dtype=3), lambda: atb.atb_linear(x, w, save=torch.float16),
                 lambda: atb.atb_linear(x, w, Y=dy.t()), lambda: atb.atb_linear(x, w, Z=_t(4, 32)[:, :24]), lambda: atb.atb_linear(x, w, act="swish"),
                 lambda: atb.atb_linear_backward(dy[:2], x, w), lambda: atb.atb_linear_backward(None, x, w), lambda: atb.atb_linear_backward(dy.half(), x, w),
                 lambda: atb.atb_linear_backward(dy, x, w, Z[:2], act="silu"), lambda: atb.atb_linear_backward(dy, x, w, dW=_t(24, 16).t()),
                 lambda: atb.atb_linear_backward(dy, x, w.t().contiguous().t(), dW=w), lambda: atb.atb_linear_backward(dy, x, w, dbias=b.half())):
        with pytest.raises(ValueError):
            call()
    assert _status(lambda: atb.atb_linear(_t(4, 12), _t(12, 24))) == 2 and _status(lambda: atb.atb_linear(x, w, act=9)) == 9
    assert _status(lambda: atb.atb_linear_backward(dy, x, w, act="silu")) == 1    # no Z
    assert _status(lambda: atb.atb_linear_backward(dy, x, w, workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))) == 7
    assert _status(lambda: atb.atb_linear(_t(4, 20)[:, 1:17], w)) in (2, 4)       # rows off 16-byte boundaries
    for act in (5, -1, 256, 1 << 40):
        assert _status(lambda: atb.atb_linear(x, w, act=act)) == 9


def test_residual_norm_refusals():
    x, f, w = _t(4, 16, dtype=F32), _t(4, 16), _t(16)
    _, _, stats = atb.atb_residual_norm(x, f, w)
    for call in (lambda: atb.atb_residual_norm(x, f[:, :8], w), lambda: atb.atb_residual_norm(x.half(), f, w), lambda: atb.atb_residual_norm(x, f, w[:8]),
                 lambda: atb.atb_residual_norm(x, f, w, gate=w.float()), lambda: atb.atb_residual_norm(x, f.t(), w), lambda: atb.atb_residual_norm(x, None, w),
                 lambda: atb.atb_residual_norm(x, f, w, kind="batch"), lambda: atb.atb_residual_norm(x, f, w, stats=stats[:1]), lambda: atb.atb_residual_norm(x, f, w, Z=x),
                 lambda: atb.atb_residual_norm_backward(f, x, x, f, stats[:1], w), lambda: atb.atb_residual_norm_backward(x, x, x, f, stats, w),
                 lambda: atb.atb_residual_norm_backward(f, f, x, f, stats, w), lambda: atb.atb_residual_norm_backward(f, x, x, f, stats, w, post_norm=True)):
        with pytest.raises(ValueError):
            call()
    assert _status(lambda: atb.atb_residual_norm(f, x, w)) == 9 and _status(lambda: atb.atb_residual_norm(x, f, w, eps=-1.0)) == 9
    assert _status(lambda: atb.atb_residual_norm(x, f, w, post_W=w)) == 9
    assert _status(lambda: atb.atb_residual_norm_backward(f, x, x, f, stats, w, workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))) == 7


def test_sample_refusals():
    x, u, v = _t(4, 100, dtype=F32), torch.rand(4, device="cuda"), torch.rand(4, device="cuda")
    for call in (lambda: atb.atb_sample(x.double(), u), lambda: atb.atb_sample(x.t(), u), lambda: atb.atb_sample(x, u[:3]), lambda: atb.atb_sample(x, u.half()),
                 lambda: atb.atb_sample(x, None), lambda: atb.atb_sample(x, u, temperature=v.double()), lambda: atb.atb_sample(x, u, top_k=v),
                 lambda: atb.atb_sample(x, u, top_k=torch.ones(4, dtype=torch.int64, device="cuda")), lambda: atb.atb_sample(x, u, top_p=v[:2]),
                 lambda: atb.atb_sample(x, u, min_p=v.cpu()), lambda: atb.atb_sample(x, u, tokens=u), lambda: atb.atb_sample(x, u, probs=u.double())):
        with pytest.raises(ValueError):
            call()
    assert _status(lambda: atb.atb_sample(x, u, temperature=-1.0)) == 9 and _status(lambda: atb.atb_sample(x, u, top_p=float("nan"))) == 9
    assert _status(lambda: atb.atb_sample(x[:, :0], u)) == 2
    with pytest.raises(TypeError):
        atb.atb_sample(x, u, top_k=0.5)
    tokens, probs = atb.atb_sample(x[:0], u[:0])
    assert tokens.shape == probs.shape == (0,)


def _calls():
    x, w, b, dy, xf = _t(700, 512), _t(512, 1032), _t(1032, dtype=F32), _t(700, 1032), _t(700, 512, dtype=F32)
    head, u, v = _t(9000, 512), torch.rand(700, device="cuda"), _t(512)
    Y, Z = atb.atb_linear(x, w, b, act="gelu", save=True)
    few = _t(2, 512)
    _, _, stats = atb.atb_residual_norm(xf, x, v, gate=v, post_norm=True)
    logits = atb.atb_linear(x, head.t(), dtype=F32)
    return {
        "linear": lambda s: atb.atb_linear(x, w, b, act="gelu", save=True, stream=s),
        "linear_few": lambda s: (atb.atb_linear(few, w, b, stream=s), atb.atb_linear(few, head.t(), dtype=F32, stream=s)),
        "linear_backward": lambda s: atb.atb_linear_backward(dy, x, w, Z, act="gelu", stream=s),
        "residual_norm": lambda s: atb.atb_residual_norm(xf, x, v, gate=v, post_norm=True, stream=s),
        "residual_norm_backward": lambda s: atb.atb_residual_norm_backward(x, xf, xf, x, stats, v, gate=v, post_norm=True, stream=s),
        "sample": lambda s: atb.atb_sample(logits, u, top_p=0.9, stream=s),
        "sample_few": lambda s: atb.atb_sample(logits, u, top_k=30, stream=s)}


NAMES = ["linear", "linear_few", "linear_backward", "residual_norm", "residual_norm_backward", "sample", "sample_few"]


@pytest.mark.parametrize("name", NAMES)
def test_other_streams_and_the_same_bits(name):
    call = _calls()[name]
    want = call(None)
    torch.cuda.synchronize()
    # a block that the current stream has given up but still has to write is not handed to a call on another stream
    held = [torch.empty(64 << 20, dtype=torch.uint8, device="cuda") for _ in range(8)]
    torch.cuda.synchronize()
    torch.cuda._sleep(50_000_000)
    for h in held:
        h.fill_(255)
    del held, h
    side = torch.cuda.Stream()
    got = call(side)
    raw = call(side.cuda_stream)
    torch.cuda.synchronize()
    again = call(None)
    for a, b, c, d in zip(want, got, raw, again):
        assert torch.equal(a, b) and torch.equal(a, c) and torch.equal(a, d)


def test_calls_at_once():
    """Every operator on a stream of its own, several times over, at the same time."""
    calls = _calls()
    want = {k: f(None) for k, f in calls.items()}
    torch.cuda.synchronize()
    streams = {k: torch.cuda.Stream() for k in calls}
    got = [(k, f(streams[k])) for _ in range(6) for k, f in calls.items()]
    torch.cuda.synchronize()
    for k, r in got:
        for a, b in zip(want[k], r):
            assert torch.equal(a, b), k
    atb.atb_device_status()


def test_graphs_that_share_a_workspace():
    x, w, dy = _t(300, 4104), _t(4104, 264), _t(300, 264)
    ws = torch.empty(max(atb.atb_linear_backward_workspace_bytes(300, 4104, 264), atb.atb_linear_workspace_bytes(300, 4104, 264)), dtype=torch.uint8, device="cuda")
    want = (atb.atb_linear(x, w), *atb.atb_linear_backward(dy, x, w))
    graphs, outs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    with torch.cuda.graph(graphs[0]):
        outs.append(atb.atb_linear(x, w, workspace=ws))
    with torch.cuda.graph(graphs[1]):
        outs += atb.atb_linear_backward(dy, x, w, workspace=ws)
    for _ in range(3):
        for o in outs:
            o.zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, outs):
            assert torch.equal(a, b)

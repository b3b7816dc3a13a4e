"""What the binding of the operators refuses on a GPU, and calls on a stream that is not the current one."""
import pytest
import torch

import paper_2511_16041_b200 as atb

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def _t(*shape, dtype=BF16):
    return torch.randn(shape, device="cuda").to(dtype)


def test_layer_norm_refusals():
    x, w = _t(4, 16), _t(16)
    _, mean, rstd = atb.atb_layer_norm(x, w, w)
    for call in (lambda: atb.atb_layer_norm(x[0], w, w),                         # not a matrix
                 lambda: atb.atb_layer_norm(x.half(), w, w),                     # no such type
                 lambda: atb.atb_layer_norm(x.t(), w, w),                        # columns not next to one another
                 lambda: atb.atb_layer_norm(x, w[:8], w),                        # too short
                 lambda: atb.atb_layer_norm(x, w, w.float()),                    # W and B of two types
                 lambda: atb.atb_layer_norm(x, w.cpu(), w),                      # not on the device
                 lambda: atb.atb_layer_norm(x, w, w, Y=x.float()),               # not X's type
                 lambda: atb.atb_layer_norm(x, w, w, mean=mean.double()),
                 lambda: atb.atb_layer_norm_bfp16(x, w, w, mant=torch.zeros(4, 32, dtype=torch.int8, device="cuda")[:, :16]),
                 lambda: atb.atb_layer_norm_backward(x[:3], x, w, mean, rstd),
                 lambda: atb.atb_layer_norm_backward(x, x, w, mean, rstd, workspace=torch.zeros(1 << 20, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(atb.AtbError) as e:
        atb.atb_layer_norm(x, w, w, eps=-1.0)
    assert e.value.status == 9
    with pytest.raises(atb.AtbError) as e:
        atb.atb_layer_norm_backward(x, x, w, mean, rstd, workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 7
    with pytest.raises(atb.AtbError) as e:
        atb.atb_layer_norm_bfp16(_t(4, 12))
    assert e.value.status == 2
    with pytest.raises(TypeError):
        atb.atb_layer_norm(x, w, w, "eps")


def test_gated_ffn_refusals():
    x, wg, wd = _t(4, 16), _t(16, 24), _t(24, 16)
    _, H, G, U = atb.atb_gated_ffn(x, wg, wg, wd, save=True)
    for call in (lambda: atb.atb_gated_ffn(x.float(), wg, wg, wd), lambda: atb.atb_gated_ffn(x, wd, wg, wd), lambda: atb.atb_gated_ffn(x, wg, wg, wg),
                 lambda: atb.atb_gated_ffn(x, wg, _t(16, 32)[:, :24], wd),       # two row strides
                 lambda: atb.atb_gated_ffn(x, wg, wg, wd, H=_t(4, 32)[:, :24]), lambda: atb.atb_gated_ffn(x, wg, wg, wd, act="relu"),
                 lambda: atb.atb_gated_ffn_backward(x[:2], x, wg, wg, wd, H, G, U), lambda: atb.atb_gated_ffn_backward(x, x, wg, wg, wd, H, G, None),
                 lambda: atb.atb_gated_ffn_backward(x, x, wg, wg, wd, H, G, U, dWg=_t(16, 32)[:, :24])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(atb.AtbError) as e:
        atb.atb_gated_ffn(_t(4, 12), _t(12, 24), _t(12, 24), _t(24, 12))
    assert e.value.status == 2
    with pytest.raises(atb.AtbError) as e:
        atb.atb_gated_ffn(x, wg, wg, wd, act=7)
    assert e.value.status == 9


def test_linear_cross_entropy_refusals():
    x, w, labels = _t(4, 16), _t(40, 16), torch.zeros(4, dtype=torch.int64, device="cuda")
    loss, lse = atb.atb_linear_cross_entropy(x, w, labels)
    for call in (lambda: atb.atb_linear_cross_entropy(x, w.float(), labels), lambda: atb.atb_linear_cross_entropy(x, w[:, :8], labels),
                 lambda: atb.atb_linear_cross_entropy(x, w, labels.int()), lambda: atb.atb_linear_cross_entropy(x, w, labels[:3]),
                 lambda: atb.atb_linear_cross_entropy_backward(loss[:2], x, w, labels, lse),
                 lambda: atb.atb_linear_cross_entropy_backward(loss.double(), x, w, labels, lse)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(atb.AtbError) as e:
        atb.atb_linear_cross_entropy_backward(loss, x, w, labels, lse, piece=-1)
    assert e.value.status == 9


def test_a_stream_given_to_the_call():
    """The kernels run on the stream given, in its order, and memory that the call makes is not handed out again meanwhile."""
    side = torch.cuda.Stream()
    M, D, F, V = 200, 256, 520, 1000
    x, wg, wu, wd, dy, head = _t(M, D), _t(D, F), _t(D, F), _t(F, D), _t(M, D), _t(V, D)
    w, labels = _t(D), torch.randint(0, V, (M,), device="cuda")
    dloss = torch.rand(M, device="cuda")

    def all_of(stream):
        n = atb.atb_layer_norm(x, w, w, stream=stream)
        nb = atb.atb_layer_norm_backward(dy, x, w, n[1], n[2], stream=stream)
        f = atb.atb_gated_ffn(x, wg, wu, wd, save=True, stream=stream)
        fb = atb.atb_gated_ffn_backward(dy, x, wg, wu, wd, *f[1:], stream=stream)
        h = atb.atb_linear_cross_entropy(x, head, labels, stream=stream)
        hb = atb.atb_linear_cross_entropy_backward(dloss, x, head, labels, h[1], piece=256, stream=stream)
        return n + nb + f + fb + h + hb

    want = all_of(None)
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        got = all_of(stream)
        # the current stream allocates and writes while the other one may still be at work
        for _ in range(20):
            torch.full((1 << 20,), 7, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_calls_inside_a_graph():
    """The calls only enqueue kernels: they are captured and replayed on new inputs in the same buffers."""
    M, D, F = 130, 128, 264
    x, wg, wu, wd, w = _t(M, D), _t(D, F), _t(D, F), _t(F, D), _t(D)
    atb.atb_gated_ffn(atb.atb_layer_norm(x, w, w)[0], wg, wu, wd)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = atb.atb_gated_ffn(atb.atb_layer_norm(x, w, w)[0], wg, wu, wd)
    x.copy_(_t(M, D))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, atb.atb_gated_ffn(atb.atb_layer_norm(x, w, w)[0], wg, wu, wd))

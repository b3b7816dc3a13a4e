"""The linear layer with bias, activation and residual against the formulas in 64 bits.  Backward stages are checked on what they
really read (Z, and dZ in the workspace), so the bounds are those of one product."""
import pytest
import torch

import paper_2511_16041_b200 as atb
from tests import operators_ref as ref
from tests.operators_ref import U16, U32, product_bound

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
ACTS = [None, "relu", "silu", "gelu", "gelu_tanh"]
# the activations go through the fast exponential: a few 2^-22 of the result, and of z in the exponent
ACT_REL = 2.0 ** -18


def act_of(z, name):
    if name is None:
        return z, torch.ones_like(z)
    if name == "relu":
        return z.clamp(min=0), (z > 0).double()
    return ref.act(z, name)


def rel_of(name):
    return 0.0 if name in (None, "relu") else ACT_REL


def normal(gen, rows, cols, scale=1.0, pad=0, dtype=BF16):
    return (torch.randn((rows, cols + pad), generator=gen, device="cuda") * scale).to(dtype)[:, :cols]


def weights(gen, K, N, transposed, pad=0):
    return normal(gen, N, K, K ** -0.5, pad).t() if transposed else normal(gen, K, N, K ** -0.5, pad)


def unit(dtype):
    return U16 if dtype == BF16 else U32


def check_forward(x, w, b, r, act, Y, Z=None):
    xd, wd = x.double(), w.double()
    z = xd @ wd + (0 if b is None else b.double())
    ez = product_bound(xd, wd)
    ez = ez + U32 * (z.abs() + ez)                             # the bias
    if Z is not None:
        ref.check(Z, z, ez + unit(Z.dtype) * (z.abs() + ez), "z")
    y, _ = act_of(z, act)
    ey = 1.2 * ez + rel_of(act) * (z.abs() + 1)                # |act'| < 1.13
    if r is not None:
        y = y + r.double()
        ey = ey + U32 * (y.abs() + ey)
    ref.check(Y, y, ey + unit(Y.dtype) * (y.abs() + ey), "y")


def check_backward(dy, x, w, Z, act, dZ, dX, dW, db):
    dyd, xd, wd = dy.double(), x.double(), w.double()
    if act is None:
        want, err = dyd, torch.zeros_like(dyd)
    else:
        zd = Z.double()
        want = dyd * act_of(zd, act)[1]
        err = rel_of(act) * (zd.abs() + 1) ** 3 * dyd.abs() + U32 * want.abs()
    if dZ is None:
        dZ = dy                                                # no activation, bf16: the products read dY
    else:
        ref.check(dZ, want, err + U16 * (want.abs() + err), "dz")
    dz = dZ.double()
    if dX is not None:
        v = dz @ wd.t()
        e = product_bound(dz, wd.t())
        ref.check(dX, v, e + U16 * (v.abs() + e), "dx")
    if dW is not None:
        v = xd.t() @ dz
        e = product_bound(xd.t(), dz)
        ref.check(dW, v, e + U16 * (v.abs() + e), "dw")
    if db is not None:
        v = want.sum(0)
        e = err.sum(0) + (dy.shape[0] + 1) * U32 * (want.abs() + err).sum(0)
        ref.check(db, v, e + unit(db.dtype) * (v.abs() + e), "db")


def run_both(M, K, N, act, transposed=False, y_type=BF16, z_type=F32, bias=F32, residual=False, pad=0, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(501 + seed)
    x, w = normal(gen, M, K, 1.0, pad), weights(gen, K, N, transposed, pad)
    b = normal(gen, 1, N, 0.3, dtype=bias)[0] if bias else None
    r = normal(gen, M, N, 1.0, pad, y_type) if residual else None
    dy = normal(gen, M, N, 0.1, pad, y_type)
    Y, Z = atb.atb_linear(x, w, b, act=act, residual=r, dtype=y_type, save=z_type)
    alone = atb.atb_linear(x, w, b, act=act, residual=r, dtype=y_type)
    assert Y.dtype == y_type and Z.dtype == z_type and torch.equal(Y, alone)
    check_forward(x, w, b, r, act, Y, Z)
    ws = torch.empty(atb.atb_linear_backward_workspace_bytes(M, K, N), dtype=torch.uint8, device="cuda")
    db = torch.empty(N, dtype=bias, device="cuda") if bias else False
    dX, dW, dB = atb.atb_linear_backward(dy, x, w, Z, act=act, dbias=db, workspace=ws)
    atb.atb_device_status()
    assert dW.stride() == (torch.empty(N, K).t() if transposed else torch.empty(K, N)).stride()
    dZ = None if act is None and y_type == BF16 else ws[:2 * M * N].view(BF16).view(M, N)
    check_backward(dy, x, w, Z, act, dZ, dX, dW, dB)


SHAPES = [(1, 8, 8), (1, 2048, 1024), (1, 10944, 4096), (1, 64, 40000), (2, 72, 136), (2, 2056, 4104), (3, 1024, 2736), (4, 264, 520), (7, 128, 4104), (8, 1000, 328),
          (16, 2048, 1024), (31, 64, 72), (64, 328, 264), (65, 4104, 64), (127, 128, 256), (128, 256, 128), (129, 136, 264), (257, 200, 520),
          (500, 1024, 2736), (1000, 320, 4104),
          # several tiles for every CTA or pair: accumulators, boxes and rings wrap round
          (20, 64, 40000), (3000, 200, 4104), (2500, 2056, 520), (5000, 520, 2056)]


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_shapes(M, K, N, transposed):
    i = (M + K // 8 + N // 8) % 5
    run_both(M, K, N, ACTS[i], transposed, y_type=(BF16, F32)[i % 2], z_type=(F32, BF16)[(M + i) % 2], bias=(F32, BF16, None)[i % 3], residual=i % 2 == 0)


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("y_type,z_type", [(BF16, F32), (BF16, BF16), (F32, F32), (F32, BF16)])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M", [1, 40, 900])
def test_every_epilogue(M, act, y_type, z_type, residual):
    run_both(M, 256, 776, act, False, y_type, z_type, BF16 if M == 40 else F32, residual, seed=M)


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("M,K,N", [(1, 136, 264), (2, 4104, 264), (6, 136, 264), (300, 264, 776), (700, 4104, 264)])
@pytest.mark.parametrize("y_type", [BF16, F32])
def test_strided_operands(M, K, N, transposed, y_type):
    run_both(M, K, N, "silu", transposed, y_type, residual=True, pad=24)


@pytest.mark.parametrize("y_type", [BF16, F32])
@pytest.mark.parametrize("M,K,N", [(1, 128, 136), (2, 128, 136), (5, 2048, 520), (40, 128, 264), (400, 136, 520)])
def test_outputs_inside_larger_buffers(M, K, N, y_type):
    """Rows behind the last one and columns beside the result are left as they were; some gradients are not wanted."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    for transposed in (False, True):
        x, w, r = normal(gen, M, K), weights(gen, K, N, transposed), normal(gen, M, N, dtype=y_type)
        y = torch.full((M + 1, N + 16), 7.0, dtype=y_type, device="cuda")
        atb.atb_linear(x, w, residual=r, Y=y[:M, :N])
        check_forward(x, w, None, r, None, y[:M, :N])
        assert bool((y[M:] == 7).all()) and bool((y[:, N:] == 7).all())
        dy = normal(gen, M, N, 0.1, dtype=y_type)
        full = atb.atb_linear_backward(dy, x, w)
        dx = torch.full((M + 1, K + 8), 7.0, dtype=BF16, device="cuda")
        dw = torch.full((N + 1, K + 8) if transposed else (K + 1, N + 8), 7.0, dtype=BF16, device="cuda")
        dw_view = dw[:N, :K].t() if transposed else dw[:K, :N]
        assert atb.atb_linear_backward(dy, x, w, dX=dx[:M, :K], dW=False, dbias=False)[1:] == (None, None)
        atb.atb_linear_backward(dy, x, w, dX=False, dW=dw_view, dbias=False)
        only = atb.atb_linear_backward(dy, x, w, dX=False, dW=False)
        assert only[:2] == (None, None) and torch.equal(only[2], full[2])
        ref.check(dx[:M, :K], full[0].double(), 2 * U16 * full[0].double().abs() + 1e-6, "dx")
        ref.check(dw_view, full[1].double(), 2 * U16 * full[1].double().abs() + 1e-6, "dw")
        assert bool((dx[M:] == 7).all()) and bool((dx[:, K:] == 7).all())
        rest = dw.clone()
        (rest[:N, :K] if transposed else rest[:K, :N]).fill_(7.0)
        assert bool((rest == 7).all())


def test_no_rows():
    w, x = torch.ones((64, 72), dtype=BF16, device="cuda"), torch.empty((0, 64), dtype=BF16, device="cuda")
    dy = torch.empty((0, 72), dtype=BF16, device="cuda")
    assert atb.atb_linear(x, w).shape == (0, 72)
    for layout in (w, w.t().contiguous().t()):
        dX, dW, db = atb.atb_linear_backward(dy, x, layout)
        assert dX.shape == (0, 64) and bool((dW == 0).all()) and bool((db == 0).all())


@pytest.mark.parametrize("M", [1, 2, 3, 70, 300])
def test_the_slope_of_relu_at_zero_and_nan(M):
    """z = 0 everywhere: relu's slope there is 0; a NaN in one row stays in that row."""
    x, w = torch.zeros((M, 64), dtype=BF16, device="cuda"), torch.ones((64, 72), dtype=BF16, device="cuda")
    dy = torch.ones((M, 72), dtype=BF16, device="cuda")
    Y, Z = atb.atb_linear(x, w, act="relu", save=True)
    assert bool((Y == 0).all()) and bool((Z == 0).all())
    dX, dW, db = atb.atb_linear_backward(dy, x, w, Z, act="relu")
    assert bool((dX == 0).all()) and bool((db == 0).all())
    x[M - 1, 5] = float("nan")
    for act in ACTS:
        Y = atb.atb_linear(x, w, act=act)
        assert bool(Y[M - 1].isnan().all()) and not bool(Y[:M - 1].isnan().any())


@pytest.mark.parametrize("act", ACTS[2:])
@pytest.mark.parametrize("M", [2, 50])
def test_gradients_against_differences(M, act):
    """sum(C * Y) along one direction of each input: central differences of the FP32 result.  Every perturbed input is a bf16 number
    (multiples of 1/64 below 1).  The step h = 1/64 leaves h^2 / 6 of the third derivative (below 1.2 here, times the cube of |dz|),
    each Y is off by product_bound and ACT_REL (|z| + 1), which the differences divide by h, and the gradients are rounded
    on the way (dZ) and at their end."""
    K, N = 16, 24
    gen = torch.Generator(device="cuda").manual_seed(11)

    def grid(*shape, most=32):
        return (torch.randint(-most, most + 1, shape, generator=gen, device="cuda").float() / 64)

    x, w, b, c = grid(M, K), grid(K, N), grid(N), grid(M, N)
    Y, Z = atb.atb_linear(x.to(BF16), w.to(BF16), b, act=act, dtype=F32, save=True)
    dX, dW, db = atb.atb_linear_backward(c, x.to(BF16), w.to(BF16), Z, act=act)
    f = lambda x, w, b: float((atb.atb_linear(x.to(BF16), w.to(BF16), b, act=act, dtype=F32).double() * c.double()).sum())  # noqa: E731
    for i, (got, h) in enumerate(((dX, 1 / 64), (dW, 1 / 64), (db, 1 / 64))):
        ins = [x, w, b]
        v = torch.randint(0, 2, ins[i].shape, generator=gen, device="cuda").float() * 2 - 1
        up, down = list(ins), list(ins)
        up[i], down[i] = ins[i] + h * v, ins[i] - h * v
        want = (f(*up) - f(*down)) / (2 * h)
        along = float((got.double() * v.double()).sum())
        vd, cd = v.double(), c.double().abs()
        dz = vd @ w.double() if i == 0 else x.double() @ vd if i == 1 else vd.expand(M, N)
        third = float((1.2 * h * h / 6 * dz.abs() ** 3 * cd).sum())
        xd, wd = x.double(), w.double()
        values = float(((1.2 * product_bound(xd.abs() + h, wd.abs() + h) + ACT_REL * (Z.double().abs() + 1 + h * dz.abs())) * cd).sum()) / h
        # the roundings of dZ reach dX (through |W|), dW (through |x|) but not db, which is summed before
        reach = vd.abs() @ wd.abs() if i == 0 else xd.abs() @ vd.abs() if i == 1 else torch.zeros_like(cd)
        rounding = U16 * float((1.13 * cd * reach).sum()) + U16 * float(got.double().abs().sum())
        slopes = ACT_REL * float((((Z.double().abs() + 1) ** 3) * cd * (reach if i < 2 else 1)).sum())
        assert abs(along - want) <= third + values + rounding + slopes, (i, along, want)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("z_type", [torch.float32, torch.bfloat16])
def test_the_slopes_of_large_and_infinite_sums(act, z_type):
    """Beyond |z| = 150 the slope's distance to 1 or 0 is less than e^-140 z, below FP32's range: dZ is dY or 0.  A NaN stays one."""
    at = [150.0, 1e5, 1e10, 1e20, 1e31, 3e38, float("inf")]
    Z = torch.tensor([s * v for v in at for s in (1.0, -1.0)] + [float("nan"), 0.0], device="cuda").to(z_type).expand(3, 16).contiguous()
    dy = torch.full((3, 16), 0.5, device="cuda", dtype=torch.bfloat16)
    x = torch.ones(3, 8, device="cuda", dtype=torch.bfloat16)
    w = torch.ones(8, 16, device="cuda", dtype=torch.bfloat16)
    _, dw, db = atb.atb_linear_backward(dy, x, w, Z, act=act, dX=False)
    want = torch.tensor([1.5, 0.0] * len(at) + [float("nan"), 0.75], device="cuda")
    assert torch.equal(db.isnan(), want.isnan()) and torch.equal(db[:-2], want[:-2])
    # Phi(0) of the erf form comes from a polynomial, off by at most 4.4e-7 of it in FP32; the two additions of three rows are off by 2^-24 each:
    # 4.4e-7 + 1.2e-7 = 5.6e-7 < 2^-20 = 9.5e-7 of the sum
    assert abs(float(db[-1]) - 0.75) <= 0.75 * 2.0 ** -20
    assert torch.equal(dw.float().nan_to_num(7.0), want.nan_to_num(7.0).expand(8, 16))

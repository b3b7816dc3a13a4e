"""The residual norm against the formulas in 64 bits.

Bounds: a sum over a row is at most 16 terms one after the other in a thread and 15 levels of joining, so 40 roundings of FP32 cover a mean, a
spread and what follows from it; errors of an input of a step are carried on by its formula.  Sums over rows: a rounding per row."""
import pytest
import torch

import paper_2511_16041_b200 as atb
from tests import operators_ref as ref
from tests.operators_ref import U16, U32

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
C = 40 * U32
EPS = 1e-5


def unit(dtype):
    return U16 if dtype == BF16 else U32


def mean(v):
    return v.mean(1, keepdim=True)


def norm(v, ev, kind, eps):
    """norm(v), r, and the error of norm(v) where v itself is off by ev."""
    mu = mean(v) if kind == "layer" else torch.zeros_like(v[:, :1])
    d = v - mu
    r = (mean(d * d) + eps) ** -0.5
    n = d * r
    e = r * (ev + mean(ev) + C * (v.abs() + mean(v.abs()))) + n.abs() * (r * mean(ev * ev).sqrt() + r * C * mean(v.abs()) + C)
    return n, r, e


def back(g, eg, n, en, r, kind):
    """r (g - mean g - n mean(g n)) and its error."""
    m0, m1 = mean(g) if kind == "layer" else 0.0, mean(g * n)
    out = r * (g - m0 - n * m1)
    e = r * (eg + mean(eg) + n.abs() * mean(eg * n.abs() + g.abs() * en) + en * m1.abs() + C * (g.abs() + mean(g.abs()) + n.abs() * mean((g * n).abs()))) + C * out.abs()
    return out, e


class Case:
    def __init__(self, M, N, types=(BF16, BF16), weights=F32, kind="layer", gate=True, post=True, biases=True, pad=0, scale=1.25, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(900 + seed)
        self.M, self.N, self.kind, self.post, self.scale, self.types, self.weights = M, N, kind, post, scale, types, weights

        def rows(dtype, spread=1.0, shift=0.0):
            return (torch.randn((M, N + pad), generator=gen, device="cuda") * spread + shift).to(dtype)[:, :N]

        def vector(shift):
            return (torch.randn(N, generator=gen, device="cuda") * 0.2 + shift).to(weights)

        self.x, self.f = rows(types[0], 1.0, 0.5), rows(types[1], 0.7, -0.3)
        self.dz, self.dh = rows(types[1]), rows(types[0])
        self.w, self.b = vector(1.0), vector(0.0) if biases else None
        self.g = vector(0.5) if gate else None
        self.pw, self.pb = (vector(1.0), vector(0.0) if biases else None) if post else (None, None)
        self.given = dict(gate=self.g, scale=scale, post_norm=post, post_W=self.pw, post_B=self.pb, kind=kind)

    def reference(self):
        d = lambda t, none: none if t is None else t.double()  # noqa: E731
        x, f, w, g, pw = self.x.double(), self.f.double(), d(self.w, 1.0), d(self.g, 1.0), d(self.pw, 1.0)
        b, pb = d(self.b, 0.0), d(self.pb, 0.0)
        zero = torch.zeros_like(x)
        absolute = lambda t: abs(t) if isinstance(t, float) else t.abs()  # noqa: E731
        if self.post:
            m, rf, em = norm(f, zero, self.kind, EPS)
            u = m * pw + pb
            eu = absolute(pw) * em + 2 * U32 * ((m * pw).abs() + absolute(pb))
        else:
            m, rf, em, u, eu = f, None, zero, f, zero
        h = self.scale * x + g * u
        eh = absolute(g) * eu + 2 * U32 * ((self.scale * x).abs() + (g * u).abs())
        n, r, en = norm(h, eh, self.kind, EPS)
        z = n * w + b
        ez = absolute(w) * en + 2 * U32 * ((n * w).abs() + absolute(b))
        return dict(locals())

    def check(self, H, Z, grads, dh):
        o = self.reference()
        ref.check(H, o["h"], o["eh"] + unit(H.dtype) * (o["h"].abs() + o["eh"]), "h")
        ref.check(Z, o["z"], o["ez"] + unit(Z.dtype) * (o["z"].abs() + o["ez"]), "z")
        if grads is None:
            return
        dX, dF, dgate, dW, dB, dPW, dPB = grads
        n, en, r, m, em, g, pw, u, eu = (o[k] for k in ("n", "en", "r", "m", "em", "g", "pw", "u", "eu"))
        absolute = o["absolute"]
        dz, M = self.dz.double(), self.M
        t, et = back(dz * o["w"], U32 * (dz * o["w"]).abs(), n, en, r, self.kind)
        if dh is not None:
            t = t + dh.double()
            et = et + U32 * t.abs()

        def rounded(got, want, err, what):
            ref.check(got, want, err + unit(got.dtype) * (want.abs() + err), what)

        def total(got, terms, errs, what, weight=1.0):
            want = weight * terms.sum(0)
            err = absolute(weight) * (errs.sum(0) + (M + 40) * U32 * (terms.abs() + errs).sum(0)) + 2 * U32 * want.abs()
            rounded(got, want, err, what)

        rounded(dX, self.scale * t, self.scale * et + U32 * (self.scale * t).abs(), "dx")
        du, edu = g * t, absolute(g) * et + U32 * (g * t).abs()
        if self.post:
            q, eq = du * pw, edu * absolute(pw) + U32 * (du * pw).abs()
            want, err = back(q, eq, m, em, o["rf"], self.kind)
            rounded(dF, want, err, "df")
            total(dPW, t * m, et * m.abs() + t.abs() * em + U32 * (t * m).abs(), "dpost_w", g)
            if dPB is not None:
                total(dPB, t, et, "dpost_b", g)
        else:
            rounded(dF, du, edu, "df")
            assert dPW is None and dPB is None
        if self.g is not None:
            # pw sum(t m) + pb sum(t): the two sums' errors apart
            if self.post:
                pb = o["pb"]
                terms, errs = t * m, et * m.abs() + t.abs() * em + U32 * (t * m).abs()
                many = (M + 40) * U32
                err = absolute(pw) * (errs.sum(0) + many * (terms.abs() + errs).sum(0)) + absolute(pb) * (et.sum(0) + many * (t.abs() + et).sum(0))
                want = (t * u).sum(0)
                rounded(dgate, want, err + 2 * U32 * (absolute(pw) * terms.sum(0).abs() + absolute(pb) * t.sum(0).abs()), "dgate")
            else:
                total(dgate, t * u, et * u.abs() + U32 * (t * u).abs(), "dgate")
        else:
            assert dgate is None
        total(dW, dz * n, dz.abs() * en + U32 * (dz * n).abs(), "dw")
        total(dB, dz, torch.zeros_like(dz), "db")

    def run(self, dh=True):
        H, Z, stats = atb.atb_residual_norm(self.x, self.f, self.w, self.b, eps=EPS, **self.given)
        assert H.dtype == self.types[0] and Z.dtype == self.types[1] and stats.shape == (4 if self.post else 2, self.M)
        dH = self.dh if dh else None
        grads = atb.atb_residual_norm_backward(self.dz, dH, self.x, self.f, stats, self.w, **self.given)
        self.check(H, Z, grads, dH)
        return H, Z, stats, grads


TYPES = [(BF16, BF16), (F32, BF16), (F32, F32)]
# every width of the kernels, in one group and its border, and beyond the widest; odd ones
WIDTHS = [1, 7, 8, 64, 100, 256, 264, 333, 512, 520, 1000, 1001, 1024, 1032, 2048, 2056, 2499, 4096, 4104, 6000, 6152, 8192, 8200, 12288, 12296, 16384, 16392, 20001]


@pytest.mark.parametrize("N", WIDTHS)
@pytest.mark.parametrize("types", TYPES)
def test_widths(types, N):
    i = N + len(WIDTHS)
    Case(37, N, types, (F32, BF16)[i % 2], ("layer", "rms")[i // 2 % 2], gate=i % 3 > 0, post=True, seed=N).run()
    Case(37, N, types, (F32, BF16)[(i + 1) % 2], ("rms", "layer")[i // 2 % 2], gate=i % 3 < 2, post=False, seed=N).run()


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("weights", [F32, BF16])
@pytest.mark.parametrize("types", TYPES)
def test_every_form(types, weights, gate, post, kind):
    for N in (200, 1001, 4160):
        Case(19, N, types, weights, kind, gate, post, biases=kind == "layer").run()


@pytest.mark.parametrize("M", [1, 2, 3, 4, 5, 147, 148, 149, 600, 5000])
@pytest.mark.parametrize("N", [96, 776, 5000])
def test_rows(M, N):
    """From one row to many for every walker; without dH too."""
    if M * N > 4_000_000:
        N = 776 if N > 776 else N
    Case(M, N, TYPES[M % 3], seed=M).run()
    Case(M, N, TYPES[(M + 1) % 3], post=False, seed=M).run(dh=False)


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("N", [258, 400, 512, 6001, 6152, 8001, 8192])
def test_several_rows_of_a_walker(N, types):
    """More rows than are on their way at once, for the layouts that keep the weights in places of their own beside four sums."""
    M = 5000 if N < 1000 else 900
    Case(M, N, types, (F32, BF16)[N % 2], ("layer", "rms")[N // 2 % 2], gate=True, post=True, seed=N).run(dh=N != 6152)


@pytest.mark.parametrize("pad", [8, 24, 1, 3, 6])
@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("N", [77, 512, 4097])
def test_strides(N, types, pad):
    Case(23, N, types, pad=pad, seed=pad).run()


@pytest.mark.parametrize("N", [256, 1001, 8192, 16400])
def test_large_means_and_constant_rows(N):
    """Where all elements of h are one number its norm is 0; a row far off centre keeps its digits."""
    x = torch.full((5, N), 3.0, dtype=F32, device="cuda")
    f = torch.full((5, N), -7.25, dtype=BF16, device="cuda")
    x[3] = 1000.0 + torch.arange(N, device="cuda").float() % 7
    for post in (False, True):
        H, Z, stats = atb.atb_residual_norm(x, f, eps=EPS, post_norm=post)
        assert bool((Z[[0, 1, 2, 4]] == 0).all())
        want = x[3].double() + (0 if post else -7.25)
        want = (want - want.mean()) / (want.var(unbiased=False) + EPS).sqrt()
        # mean and distances are off by a few units of 1000; the spread is 2
        ref.check(Z[3][None], want[None], 8 * U32 * 1000 / 2 + U16 * (want.abs()[None] + 1e-3), "z")


@pytest.mark.parametrize("N", [64, 1001, 6000, 20000])
def test_bad_rows_stay_their_own(N):
    c = Case(9, N)
    H, Z, _, grads = c.run()
    x = c.x.clone()
    x[4, N // 2], x[6, 0] = float("nan"), float("inf")
    H2, Z2, stats = atb.atb_residual_norm(x, c.f, c.w, c.b, eps=EPS, **c.given)
    dX, dF = atb.atb_residual_norm_backward(c.dz, c.dh, x, c.f, stats, c.w, **c.given)[:2]
    keep = [0, 1, 2, 3, 5, 7, 8]
    for got, want in ((H2, H), (Z2, Z), (dX, grads[0]), (dF, grads[1])):
        assert torch.equal(got[keep], want[keep])
    assert bool(Z2[[4, 6]].isnan().any(1).all())


@pytest.mark.parametrize("N", [96, 1001, 4096, 9000])
def test_wanted_gradients_and_places(N):
    c = Case(50, N, (F32, BF16))
    H, Z, stats, full = c.run()
    h, z = torch.full((51, N + 8), 7.0, device="cuda"), torch.full((51, N + 8), 7.0, dtype=BF16, device="cuda")
    atb.atb_residual_norm(c.x, c.f, c.w, c.b, eps=EPS, H=h[:50, :N], Z=z[:50, :N], **c.given)
    assert torch.equal(h[:50, :N], H) and torch.equal(z[:50, :N], Z)
    assert all(bool((t[50:] == 7).all()) and bool((t[:, N:] == 7).all()) for t in (h, z))
    names = ("dX", "dF", "dgate", "dW", "dB", "dpost_W", "dpost_B")
    for i, name in enumerate(names):
        got = atb.atb_residual_norm_backward(c.dz, c.dh, c.x, c.f, stats, c.w, **c.given, **{k: False for k in names if k != name})
        for j in range(7):
            assert (got[j] is None) == (i != j)
        assert torch.equal(got[i], full[i]), name
        got = atb.atb_residual_norm_backward(c.dz, c.dh, c.x, c.f, stats, c.w, **c.given, **{name: False})
        for j in range(7):
            assert got[j] is None if i == j else torch.equal(got[j], full[j])
    assert all(g is None for g in atb.atb_residual_norm_backward(c.dz, c.dh, c.x, c.f, stats, c.w, **c.given, **{k: False for k in names}))


def test_no_vectors_at_all():
    c = Case(40, 320, (BF16, BF16), gate=False, post=False, scale=1.0)
    H, Z, stats = atb.atb_residual_norm(c.x, c.f)
    c.w = torch.ones(320, device="cuda")
    c.b = None
    dX, dF, dgate, dW, dB, dPW, dPB = atb.atb_residual_norm_backward(c.dz, None, c.x, c.f, stats)
    assert torch.equal(dX, dF) and dgate is None and dPW is None and dW.dtype == F32
    c.check(H, Z, (dX, dF, None, dW, dB, None, None), None)


def test_no_rows():
    x, w = torch.empty((0, 64), dtype=BF16, device="cuda"), torch.ones(64, device="cuda")
    H, Z, stats = atb.atb_residual_norm(x, x, w, gate=w, post_norm=True)
    assert H.shape == (0, 64) and stats.shape == (4, 0)
    grads = atb.atb_residual_norm_backward(x, x, x, x, stats, w, gate=w, post_norm=True)
    assert grads[0].shape == (0, 64) and all(bool((g == 0).all()) and g.shape == (64,) for g in grads[2:])


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("post", [False, True])
def test_gradients_against_differences(post, kind):
    """FP32, sum(C Z + D H) along one direction of each input, by central differences with step s: the third derivative leaves an s^2 part, which
    Richardson's second step (s and 2 s) takes away, and FP32 results leave their rounding over s."""
    M, N, s = 3, 24, 2.0 ** -6
    c = Case(M, N, (F32, F32), F32, kind, True, post, seed=5)
    Cz, Dh = c.dz, c.dh

    def value(**changed):
        v = {**dict(X=c.x, F=c.f, W=c.w, B=c.b, gate=c.g, post_W=c.pw, post_B=c.pb), **changed}
        H, Z, _ = atb.atb_residual_norm(**v, scale=c.scale, post_norm=post, kind=kind, eps=EPS)
        return float((Z.double() * Cz.double()).sum() + (H.double() * Dh.double()).sum())

    H, Z, stats = atb.atb_residual_norm(c.x, c.f, c.w, c.b, eps=EPS, **c.given)
    dX, dF, dgate, dW, dB, dPW, dPB = atb.atb_residual_norm_backward(Cz, Dh, c.x, c.f, stats, c.w, **c.given)
    gen = torch.Generator(device="cuda").manual_seed(6)
    pairs = [("X", c.x, dX), ("F", c.f, dF), ("gate", c.g, dgate), ("W", c.w, dW), ("B", c.b, dB)] + ([("post_W", c.pw, dPW), ("post_B", c.pb, dPB)] if post else [])
    size = float((Z.abs() * Cz.abs()).sum() + (H.abs() * Dh.abs()).sum())
    for name, at, grad in pairs:
        v = torch.randn(at.shape, generator=gen, device="cuda")
        d1, d2 = ((value(**{name: at + k * s * v}) - value(**{name: at - k * s * v})) / (2 * k * s) for k in (1, 2))
        want = (4 * d1 - d2) / 3
        along = float((grad.double() * v.double()).sum())
        # results: C of their size over s; the fifth derivative's part, s^4 (1.5e-8 of it here), is below that
        assert abs(along - want) <= 2 * C * size / s + 1e-4 * float((grad.abs() * v.abs()).sum()), (name, along, want)

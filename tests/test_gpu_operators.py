"""The operators of LocalTrain (layer norm, matrix product with epilogue, distillation loss, each with its gradients) against their
formulas in 64 bits, at the sizes, types, strides and contents where they can go wrong.

Tolerances.  u = eps / 2 of the output's type is one rounding, F = 2^-24 one of binary32.  A sum of n terms in any order is
off by at most n F times the sum of magnitudes; each bound below is that, with the terms that enter written out.
"""
import math

import numpy as np
import pytest

from paper_1709_09393_amd import binding, workloads

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F = 2.0 ** -24
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
DTYPES = ["f32", "f16", "bf16"]


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU test selected but torch.cuda.is_available() is False")
    torch.cuda.set_device(0)


@pytest.fixture(scope="module")
def ctx():
    sd = binding.SlimDP(4096, 32)
    yield sd
    sd.close()


def u(t):
    return torch.finfo(t).eps / 2


def tiny(t):
    """Half a step below the smallest normal number."""
    return torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2


class Maker:
    """Seeded tensors on the GPU; every matrix may be a view: pad elements between its rows, shift elements before its first."""

    def __init__(self, seed, pad=0, shift=0):
        self.g = np.random.default_rng(seed)
        self.pad, self.shift = pad, shift
        self.views = []

    def view(self, rows, cols, dtype, fill=None):
        ld = cols + self.pad
        flat = torch.full((self.shift + rows * ld + 7,), -77.0, dtype=dtype, device="cuda")
        m = flat[self.shift:self.shift + rows * ld].view(rows, ld)[:, :cols]
        if fill is not None:
            m.copy_(torch.from_numpy(fill).to("cuda").to(dtype))
        self.views.append((flat, rows, cols, ld))
        return m

    def normal(self, rows, cols, dtype, sigma=1.0, mean=0.0):
        return self.view(rows, cols, dtype, self.g.normal(mean, sigma, (rows, cols)).astype(np.float32))

    def vec(self, n, sigma=1.0, mean=0.0, dtype=torch.float32):
        flat = torch.empty(n + self.shift, dtype=dtype, device="cuda")
        v = flat[self.shift:]
        v.copy_(torch.from_numpy(self.g.normal(mean, sigma, n).astype(np.float32)))
        return v

    def check_gaps(self):
        """Nothing but the matrices' elements has been written."""
        for flat, rows, cols, ld in self.views:
            mask = torch.ones_like(flat, dtype=torch.bool)
            mask[self.shift:self.shift + rows * ld].view(rows, ld)[:, :cols] = False
            assert bool((flat[mask] == -77.0).all())


def close(got, want, tol, what):
    got, want = got.double(), want.double()
    assert got.shape == want.shape, what
    if got.numel() == 0:
        return
    bad = ~((got - want).abs() <= tol)
    bad &= ~(got.isnan() & want.isnan()) & (got != want)
    if bool(bad.any()):
        i = tuple(int(v) for v in bad.nonzero()[0])
        t = tol[i] if torch.is_tensor(tol) and tol.shape == got.shape else tol
        pytest.fail(f"{what}{list(i)}: got {float(got[i])!r}, want {float(want[i])!r}, tolerance {t!r}, {int(bad.sum())} of {got.numel()} off")


# ---------------------------------------------------------------------------------------------------------------
# layer norm
# ---------------------------------------------------------------------------------------------------------------
NORM_SHAPES = [
    ([1], 1), ([3], 2), ([5], 7), ([9, 0, 2], 16), ([33], 63), ([4], 64), ([17], 65), ([6, 1], 127), ([5], 128), ([7], 255), ([3], 512),
    ([2], 513), ([5], 1000), ([4, 4], 1024), ([3], 1337), ([70, 3, 0, 40], 2048), ([3], 2049), ([2], 4096), ([9], 4099), ([2], 8192),
    ([2], 8200), ([3], 16384), ([2], 16391), ([1], 32768), ([2], 32777), ([1], 65536), ([2], 65533), ([300], 48), ([1100, 700], 96),
]


def norm_tolerance(x, weight, bias, eps, dtype):
    """Depth of the sums: up to 64 elements a thread one after the other, ten steps across threads, a few roundings more."""
    n, K = x.shape[1], 96 * F
    mean = x.mean(1, keepdim=True)
    var = (x - mean).square().mean(1, keepdim=True)
    rstd = (var + eps).rsqrt()
    dmean = K * x.abs().mean(1, keepdim=True)
    drstd = K + (2 * dmean * (x - mean).abs().mean(1, keepdim=True) + dmean.square()) / (var + eps)     # relative
    xh = (x - mean) * rstd
    g = weight.abs()
    y = xh * weight + bias
    e = g * (rstd * (dmean + 2 * F * (x.abs() + mean.abs())) + xh.abs() * (drstd + 4 * F)) + 2 * F * (bias.abs() + y.abs())
    return y, mean[:, 0], rstd[:, 0], u(dtype) * y.abs() + 1.01 * e + tiny(dtype), dmean[:, 0], rstd[:, 0] * drstd[:, 0] + F * rstd[:, 0]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
def test_layer_norm_matches_the_formula(ctx, dtype, pad, shift):
    t = TYPES[dtype]
    for rows, cols in NORM_SHAPES:
        mk = Maker(cols, pad, shift)
        x = [mk.normal(r, cols, t, 1.5, 0.7) for r in rows]
        w, b = [mk.vec(cols, 0.3, 1.0) for _ in rows], [mk.vec(cols, 0.3) for _ in rows]
        y = [mk.view(r, cols, t) for r in rows]
        _, mean, rstd = ctx.layer_norm(x, w, b, 1e-5, y=y)
        ctx.synchronize()
        for q in range(len(rows)):
            ref, rm, rr, ty, tm, tr = norm_tolerance(x[q].double(), w[q].double(), b[q].double(), 1e-5, t)
            what = f"{dtype} {rows} x {cols} worker {q} "
            close(mean[q], rm, tm + tiny(torch.float32), what + "mean")
            close(rstd[q], rr, tr, what + "rstd")
            close(y[q], ref, ty, what + "y")
        mk.check_gaps()


def test_layer_norm_without_weight_or_bias_and_in_place(ctx):
    mk = Maker(5)
    x = [mk.normal(11, 300, torch.float32) for _ in range(2)]
    keep = [v.clone() for v in x]
    w = mk.vec(300, 0.2, 1.0)
    one, zero = torch.ones(300, device="cuda").double(), torch.zeros(300, device="cuda").double()
    y, _, _ = ctx.layer_norm(x, None, None)
    y2, _, _ = ctx.layer_norm(x, [w, None], None, y=x)                       # a worker without weight; y is x
    ctx.synchronize()
    for q in range(2):
        ref, _, _, tol, _, _ = norm_tolerance(keep[q].double(), one, zero, 1e-5, torch.float32)
        close(y[q], ref, tol, "plain")
        ref, _, _, tol, _, _ = norm_tolerance(keep[q].double(), w.double() if q == 0 else one, zero, 1e-5, torch.float32)
        close(x[q], ref, tol, "in place")


def test_layer_norm_of_far_means_constant_rows_and_values_that_are_not_finite(ctx):
    mk = Maker(6)
    x = mk.normal(8, 1000, torch.float32, 1.0, 4096.0)
    x[1] = 3.0                                                              # variance 0
    x[2, 17] = float("inf")
    x[3, 5] = float("nan")
    x[4] = 1e18                                                             # squares of distances overflow nowhere: they are 0
    y, mean, rstd = ctx.layer_norm([x], None, None)
    ctx.synchronize()
    ref, rm, rr, tol, _, tr = norm_tolerance(x.double(), torch.ones(1000, device="cuda").double(), torch.zeros(1000, device="cuda").double(),
                                             1e-5, torch.float32)
    for r in (0, 5, 6, 7):
        close(y[0][r], ref[r], tol[r], f"row {r}")
    assert bool((y[0][1] == 0).all()) and float(mean[0][1]) == 3.0
    close(rstd[0][1:2], torch.full((1,), 1e-5 ** -0.5, device="cuda"), 1e-5 ** -0.5 * 4 * F, "rstd of a constant row")
    assert bool(y[0][2].isnan().any()) and bool(y[0][3].isnan().all())
    assert bool(y[0][4].isfinite().all())


def norm_back_reference(dy, x, w, mean, rstd):
    n = x.shape[1]
    m, r = mean[:, None], rstd[:, None]
    xh = (x - m) * r
    a = dy * w
    s1, s2 = a.mean(1, keepdim=True), (a * xh).mean(1, keepdim=True)
    dx = r * (a - s1 - xh * s2)
    K = 96 * F + 4 * F * math.ceil(n / 4096)
    exh = 3 * F * r * (x.abs() + m.abs())                                   # error of xh
    axh = xh.abs() + exh
    es1 = K * a.abs().mean(1, keepdim=True)
    es2 = K * (a.abs() * axh).mean(1, keepdim=True) + (a.abs() * exh).mean(1, keepdim=True)
    e = r * (es1 + axh * es2 + exh * s2.abs() + 8 * F * (a.abs() + s1.abs() + axh * s2.abs()))
    return dx, e, xh, exh


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad,shift", [(0, 0), (5, 1)])
def test_layer_norm_backward_matches_the_formula(ctx, dtype, pad, shift):
    t = TYPES[dtype]
    for rows, cols in NORM_SHAPES:
        mk = Maker(cols + 1, pad, shift)
        x = [mk.normal(r, cols, t, 1.5, 0.7) for r in rows]
        dy = [mk.normal(r, cols, t, 0.3) for r in rows]
        w = [mk.vec(cols, 0.3, 1.0) for _ in rows]
        mean = [v.double().mean(1).float() for v in x]
        rstd = [((v.double() - v.double().mean(1, keepdim=True)).square().mean(1) + 1e-5).rsqrt().float() for v in x]
        dx = [mk.view(r, cols, t) for r in rows]
        old_w, old_b = [mk.vec(cols) for _ in rows], [mk.vec(cols) for _ in rows]
        dw, db = [v.clone() for v in old_w], [v.clone() for v in old_b]
        _, gw, gb = ctx.layer_norm_backward(dy, x, w, mean, rstd, dx=dx)
        ctx.layer_norm_backward(dy, x, w, mean, rstd, want_dx=False, dweight=dw, dbias=db, accumulate=True)
        ctx.synchronize()
        for q, r in enumerate(rows):
            what = f"{dtype} {rows} x {cols} worker {q} "
            dyd, xd = dy[q].double(), x[q].double()
            ref, e, xh, exh = norm_back_reference(dyd, xd, w[q].double(), mean[q].double(), rstd[q].double())
            close(dx[q], ref, u(t) * ref.abs() + 1.01 * e + tiny(t), what + "dx")
            n = (r + 8) * F
            tw = n * (dyd.abs() * (xh.abs() + exh)).sum(0) + (dyd.abs() * exh).sum(0) + 1e-30
            tb = n * dyd.abs().sum(0) + 1e-30
            rw, rb = (dyd * xh).sum(0), dyd.sum(0)
            close(gw[q], rw, tw, what + "dweight")
            close(gb[q], rb, tb, what + "dbias")
            close(dw[q], rw + old_w[q].double(), tw + F * (rw + old_w[q].double()).abs() + F * rw.abs(), what + "dweight added")
            close(db[q], rb + old_b[q].double(), tb + F * (rb + old_b[q].double()).abs() + F * rb.abs(), what + "dbias added")
        mk.check_gaps()


@pytest.mark.parametrize("alias", ["dy", "x"])
def test_layer_norm_backward_over_its_inputs(ctx, alias):
    mk = Maker(8)
    for cols in (48, 1500, 20000):
        x, dy, w = mk.normal(40, cols, torch.bfloat16), mk.normal(40, cols, torch.bfloat16), mk.vec(cols)
        mean, rstd = x.float().mean(1), (x.float().var(1, unbiased=False) + 1e-5).rsqrt()
        want = ctx.layer_norm_backward([dy], [x], [w], [mean], [rstd])
        x2, dy2 = x.clone(), dy.clone()
        got = ctx.layer_norm_backward([dy2], [x2], [w], [mean], [rstd], dx=[dy2 if alias == "dy" else x2])
        ctx.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a[0], b[0])


# ---------------------------------------------------------------------------------------------------------------
# matrix product
# ---------------------------------------------------------------------------------------------------------------
def act_value(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2.0))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def act_slope(z, act):
    z = z.detach().clone().requires_grad_(True)
    if act == "relu":
        return (z > 0).double()
    act_value(z, act).sum().backward()
    return z.grad.detach()


def steps(K, dtype):
    """Roundings that a sum of K products meets one after the other: inside an instruction's 32 (binary32: 4), then from instruction to
    instruction; pieces of a split sum shorten the chain, joining them adds as many as there are (64 at most)."""
    return (K / 32 + 32 + 64) if dtype != torch.float32 else (K / 4 + 4 + 64)


LINEAR_SHAPES = [
    ([1], 1, 1), ([1], 7, 3), ([2], 64, 64), ([3, 0, 1], 65, 130), ([1], 4096, 1024), ([4], 1000, 513), ([8], 512, 2048), ([5], 4099, 61),
    ([16], 256, 256), ([17], 130, 127), ([33, 64], 128, 128), ([127], 96, 129), ([128], 2048, 128), ([129], 72, 64), ([256], 256, 256),
    ([257, 31], 264, 520), ([300], 1, 300), ([300], 300, 1), ([40, 200, 0, 7], 321, 255), ([512], 192, 512), ([700], 1024, 640), ([64], 8192, 72),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1), (8, 8)])
def test_linear_matches_the_formula(ctx, dtype, pad, shift):
    t = TYPES[dtype]
    acts = ["none", "relu", "gelu", "gelu_tanh", "silu"]
    for j, (rows, cols, out) in enumerate(LINEAR_SHAPES):
        act = acts[j % 5]
        mk = Maker(j, pad, shift)
        x = [mk.normal(r, cols, t) for r in rows]
        w = [mk.normal(out, cols, t, cols ** -0.5) for _ in rows]
        b = [mk.vec(out, 0.3) for _ in rows]
        res = [mk.normal(r, out, t) for r in rows]
        y, z, y2 = [mk.view(r, out, t) for r in rows], [mk.view(r, out, t) for r in rows], [mk.view(r, out, t) for r in rows]
        ctx.linear(x, w, b, act, res, y=y, z=z)
        ctx.linear(x, w, None, y=y2)                                         # the product alone
        ctx.synchronize()
        for q in range(len(rows)):
            what = f"{dtype} {rows} x {cols} x {out} {act} worker {q} "
            xd, wd = x[q].double(), w[q].double()
            prod, mag = xd @ wd.t(), xd.abs() @ wd.abs().t()
            ez = steps(cols, t) * F * mag
            close(y2[q], prod, u(t) * prod.abs() + 1.01 * ez + tiny(t), what + "product")
            ref = prod + b[q].double()
            ez = ez + 2 * F * (ref.abs() + b[q].double().abs())
            close(z[q], ref, u(t) * ref.abs() + 1.01 * ez + tiny(t), what + "z")
            a = act_value(ref, act)
            # slopes are at most 1.13; the functions themselves are within 16 roundings of their argument's size
            ey = 1.13 * ez + (16 * F * (ref.abs() + 1) if act in ("gelu", "gelu_tanh", "silu") else 0.0)
            want = a + res[q].double()
            close(y[q], want, u(t) * want.abs() + 1.01 * ey + 2 * F * want.abs() + tiny(t), what + "y")
        mk.check_gaps()


def test_linear_over_its_residual_and_shared_weights(ctx):
    mk = Maker(3)
    x = [mk.normal(70, 200, torch.bfloat16) for _ in range(3)]
    w, b = mk.normal(96, 200, torch.bfloat16, 0.07), mk.vec(96)
    res = [mk.normal(70, 96, torch.bfloat16) for _ in range(3)]
    want, _ = ctx.linear(x, [w] * 3, [b, None, b], "silu", res)
    got, _ = ctx.linear(x, [w] * 3, [b, None, b], "silu", res, y=res)
    ctx.synchronize()
    for q in range(3):
        assert got[q] is res[q] and torch.equal(want[q], res[q])


@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
def test_activations_over_their_whole_range(ctx, act):
    """Value and slope by the definition, from the smallest to the largest arguments, and what infinities and NaN give."""
    e = torch.arange(-40, 12, 0.01, dtype=torch.float64)
    z = torch.cat([torch.exp2(e), -torch.exp2(e), torch.linspace(-12, 12, 9001, dtype=torch.float64), torch.zeros(1, dtype=torch.float64)]).float().cuda()
    z = torch.cat([z, torch.tensor([float("inf"), -float("inf"), float("nan"), 3e38, -3e38], device="cuda")])
    n = z.numel()
    one = torch.ones((1, 1), device="cuda")
    y, _ = ctx.linear([z[:, None].contiguous()], [one], None, act)
    dz, _ = ctx.linear_epilogue_backward([torch.ones((n, 1), device="cuda")], [z[:, None].contiguous()], act)
    ctx.synchronize()
    fin = n - 5
    zd = z[:fin].double()
    close(y[0][:fin, 0], act_value(zd, act), 16 * F * zd.abs().clamp(max=4096) + F * act_value(zd, act).abs(), act)
    # the slope's terms are of the size of 1 (z times a density at most 0.3, exponents up to 50 carry their own rounding)
    close(dz[0][:fin, 0], act_slope(zd, act), 64 * F, act + " slope")
    y, dz = y[0][fin:, 0].tolist(), dz[0][fin:, 0].tolist()
    assert y[0] == float("inf") and y[1] == 0.0 and math.isnan(y[2]) and y[3] == pytest.approx(3e38) and y[4] == 0.0
    assert dz[0] == 1.0 and dz[1] == 0.0 and dz[3] == 1.0 and dz[4] == 0.0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
def test_linear_epilogue_backward_matches_the_formula(ctx, dtype, pad, shift):
    t = TYPES[dtype]
    acts = ["none", "relu", "gelu", "gelu_tanh", "silu"]
    for j, (rows, out) in enumerate([([1], 1), ([5, 0, 3], 70), ([200], 257), ([64, 3000], 33), ([17], 4096), ([1000], 512), ([2], 9001)]):
        act = acts[j % 5]
        mk = Maker(j, pad, shift)
        dy, z = [mk.normal(r, out, t, 0.3) for r in rows], [mk.normal(r, out, t) for r in rows]
        dz = [mk.view(r, out, t) for r in rows]
        old = [mk.vec(out) for _ in rows]
        add = [v.clone() for v in old]
        _, db = ctx.linear_epilogue_backward(dy, z, act, dz=dz)
        ctx.linear_epilogue_backward(dy, z, act, dbias=add, accumulate=True)
        ctx.synchronize()
        for q, r in enumerate(rows):
            what = f"{dtype} {rows} x {out} {act} worker {q} "
            dyd = dy[q].double()
            ref = dyd * act_slope(z[q].double(), act)
            e = dyd.abs() * 64 * F
            close(dz[q], ref, u(t) * ref.abs() + e + tiny(t), what + "dz")
            tb = (r + 8) * F * (ref.abs() + e).sum(0) + e.sum(0) + 1e-30
            close(db[q], ref.sum(0), tb, what + "dbias")
            both = ref.sum(0) + old[q].double()
            close(add[q], both, tb + F * (both.abs() + ref.sum(0).abs()), what + "dbias added")
        mk.check_gaps()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1), (8, 8)])
def test_linear_backward_matches_the_formula(ctx, dtype, pad, shift):
    t = TYPES[dtype]
    for j, (rows, cols, out) in enumerate(LINEAR_SHAPES):
        mk = Maker(j + 50, pad, shift)
        dz, x = [mk.normal(r, out, t, 0.3) for r in rows], [mk.normal(r, cols, t) for r in rows]
        w = [mk.normal(out, cols, t, cols ** -0.5) for _ in rows]
        dx = [mk.view(r, cols, t) for r in rows]
        old = [mk.vec(out * cols).view(out, cols) for _ in rows]              # pieces of a flat gradient, at odd places with a shift
        add = [mk.vec(out * cols).view(out, cols).copy_(v) for v in old]
        _, dw = ctx.linear_backward(dz, x, w, dx=dx)
        ctx.linear_backward(dz, x, None, dweight=add, accumulate=True, want_dx=False)
        ctx.synchronize()
        for q, r in enumerate(rows):
            what = f"{dtype} {rows} x {cols} x {out} worker {q} "
            dzd, xd, wd = dz[q].double(), x[q].double(), w[q].double()
            ref, e = dzd @ wd, steps(out, t) * F * (dzd.abs() @ wd.abs())
            close(dx[q], ref, u(t) * ref.abs() + 1.01 * e + tiny(t), what + "dx")
            ref, e = dzd.t().contiguous() @ xd, steps(r, t) * F * (dzd.abs().t().contiguous() @ xd.abs()) + 1e-30
            close(dw[q], ref, F * ref.abs() + 1.01 * e, what + "dweight")
            both = ref + old[q].double()
            close(add[q], both, 1.01 * e + F * (ref.abs() + both.abs()), what + "dweight added")
        mk.check_gaps()


@pytest.mark.parametrize("R,K,N,pad,shift", [(2100, 1032, 2312, 0, 0), (4104, 1032, 4360, 8, 8), (2101, 1033, 2311, 0, 0), (4097, 1027, 4355, 1, 1),
                                             (4099, 60, 4102, 0, 0), (64, 4352, 4104, 0, 0), (4100, 4101, 190, 2, 0), (700, 9000, 130, 0, 0)])
def test_products_larger_than_a_wave_of_tiles(ctx, R, K, N, pad, shift):
    """Every tile size, both ways into the LDS, the whole chip busy and the sum in pieces; every element against 64 bits."""
    for t in (torch.bfloat16, torch.float16):
        mk = Maker(9, pad, shift)
        x, w, dz = mk.normal(R, K, t), mk.normal(N, K, t, 0.03), mk.normal(R, N, t, 0.1)
        y, _ = ctx.linear([x], [w])
        dx, dw = ctx.linear_backward([dz], [x], [w])
        ctx.synchronize()
        for ref, mag, got, n, ut in ((x.double() @ w.double().t(), x.double().abs() @ w.double().abs().t(), y[0], K, u(t)),
                                     (dz.double() @ w.double(), dz.double().abs() @ w.double().abs(), dx[0], N, u(t)),
                                     (dz.double().t() @ x.double(), dz.double().abs().t() @ x.double().abs(), dw[0], R, F)):
            close(got, ref, ut * ref.abs() + 1.01 * steps(n, t) * F * mag + tiny(t), str(t))


def test_rows_behind_infinite_and_nan_neighbours_stay_clean(ctx):
    """What lies behind a row's end or in other rows never enters: it is full of NaN here."""
    t = torch.bfloat16
    big = torch.full((200, 256), float("nan"), dtype=t, device="cuda")
    x, w = big[:77, :100], torch.full((130, 256), float("nan"), dtype=t, device="cuda")[:, :100]
    x.copy_(torch.randn(77, 100, generator=torch.Generator().manual_seed(1)))
    w.copy_(torch.randn(130, 100, generator=torch.Generator().manual_seed(2)))
    dz = torch.full((77, 256), float("nan"), dtype=t, device="cuda")[:, :130]
    dz.copy_(torch.randn(77, 130, generator=torch.Generator().manual_seed(3)))
    y, _ = ctx.linear([x], [w])
    dx, dw = ctx.linear_backward([dz], [x], [w])
    _, db = ctx.linear_epilogue_backward([dz])
    ctx.synchronize()
    for v in (y, dx, dw, db):
        assert bool(v[0].isfinite().all())
    # and one that belongs to a row stays in that row
    x[5, 3] = float("inf")
    y, _ = ctx.linear([x], [w])
    ctx.synchronize()
    assert not bool(y[0][5].isfinite().any()) and bool(torch.cat([y[0][:5], y[0][6:]]).isfinite().all())


def test_epilogue_backward_writes_no_sums_that_are_not_asked_for(ctx):
    """Without the bias's gradient a workspace is not touched, however small; workers that want none beside ones that do."""
    import ctypes as C
    mk = Maker(12)
    dy, z, out = [mk.normal(4000, 48, torch.float32) for _ in range(2)], [mk.normal(4000, 48, torch.float32) for _ in range(2)], mk.vec(48)
    want = ctx.linear_epilogue_backward(dy, z, "silu")
    need = ctx._L.slimdp_linear_workspace_bytes(2, (C.c_uint64 * 2)(4000, 4000), 1, 48, 0, 1)
    assert need > 0
    ws = torch.full((1024,), 7.0, device="cuda")
    dz = [torch.empty_like(v) for v in dy]
    rc = ctx._L.slimdp_linear_epilogue_backward(ctx._h, 2, (C.c_uint64 * 2)(4000, 4000), 48, 0, binding._table(dy), 48, binding._table(z), 48, 4,
                                                binding._table(dz), 48, None, 0, ws.data_ptr(), 64)
    assert rc == binding.OK
    _, db = ctx.linear_epilogue_backward(dy, z, "silu", dbias=[None, out])
    _, dw, dbn = ctx.layer_norm_backward(dy, z, None, [v[:, 0].contiguous() for v in z], [v[:, 1].abs().contiguous() for v in z], dweight=[None, out.clone()], dbias=[None, None])
    ctx.synchronize()
    assert bool((ws == 7.0).all())
    assert all(torch.equal(a, b) for a, b in zip(want[0], dz))
    assert torch.equal(out, want[1][1]) and bool(dw[1].isfinite().all())


# ---------------------------------------------------------------------------------------------------------------
# distillation
# ---------------------------------------------------------------------------------------------------------------
def distill_reference(logits, index, value, tau, weight, dtype):
    V = logits.shape[1]
    s = logits.double() / tau
    lse = torch.logsumexp(s, 1)
    valid = (index >= 0) & (index < V) & (value > -math.inf)
    v = torch.where(valid, value.double() / tau, torch.full_like(value, -math.inf, dtype=torch.float64))
    some = valid.any(1) & (weight != 0)
    v = torch.where(some[:, None], v, torch.zeros_like(v))
    logp = torch.log_softmax(v, 1)
    p = torch.where(valid & some[:, None], logp.exp(), torch.zeros_like(v))
    at = torch.where(valid, index, torch.zeros_like(index)).long()
    # from the row's largest logit, not from lse: where all logits are the type's lowest value, lse in 64 bits loses log V beside them
    logq_all = torch.log_softmax(s, 1)
    logq = logq_all.gather(1, at)
    diff = torch.where(p > 0, logp - logq, torch.zeros_like(p))
    w = torch.where(some, weight.double(), torch.zeros_like(weight, dtype=torch.float64))
    loss = w * tau * tau * torch.where(p > 0, p * diff, torch.zeros_like(p)).sum(1)
    q = torch.where(some[:, None], logq_all.exp(), torch.zeros_like(s))
    dense = torch.zeros_like(s).scatter_add_(1, at, p)
    # errors: a scaled logit is off by two roundings of its size, an exponential by that and a few more; sums of positive terms by their depth
    fin = lambda a: torch.where(a.isfinite(), a.abs(), torch.zeros_like(a)).amax(1)
    E = F * (8 * fin(s) + 4 * lse.abs().nan_to_num(posinf=0) + V / 256 + 64)
    Ep = F * (8 * (fin(v) if v.shape[1] else 0 * E) + v.shape[1] / 64 + 64)
    tl = w.abs() * tau * tau * (E + Ep + (2 * Ep + 8 * F) * (p * diff.abs().nan_to_num(posinf=0)).sum(1) + 8 * F)
    dref = (w * tau)[:, None] * (q - dense)
    td = u(dtype) * dref.abs() + (w.abs() * tau)[:, None] * (q * 2 * E[:, None] + dense * 2 * (Ep[:, None] + 4 * F)) + tiny(dtype)
    return loss, lse, dref, tl + 1e-30, E + F, td


DISTILL_SHAPES = [
    ([1], 1, 1), ([3], 2, 2), ([4, 0, 2], 7, 3), ([2], 64, 64), ([5], 1000, 20), ([3], 4097, 1), ([2], 10007, 255), ([2], 8192, 1024),
    ([3], 32768, 64), ([2], 50001, 100), ([2], 65536, 7), ([2], 131072, 64), ([1, 1], 131073, 33), ([2], 200000, 513), ([400], 300, 8), ([1], 600001, 50),
]


def teacher(mk, rows, V, top, short=True):
    idx = np.stack([mk.g.choice(V, top, replace=False) if V >= top else mk.g.integers(0, V, top) for _ in range(rows)]) if rows else np.zeros((0, top))
    if short:
        for r in range(0, rows, 2):
            idx[r, mk.g.integers(0, top + 1):] = -1
    return mk.view(rows, top, torch.int32, idx.astype(np.float64)), mk.view(rows, top, torch.float32, mk.g.normal(5, 2, (rows, top)))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad,shift,tau", [(0, 0, 1.0), (5, 1, 2.5), (8, 8, 0.5)])
def test_distill_loss_matches_the_formula(ctx, dtype, pad, shift, tau):
    t = TYPES[dtype]
    for rows, V, top in DISTILL_SHAPES:
        mk = Maker(V + top, pad, shift)
        logits = [mk.normal(r, V, t, 2.0) for r in rows]
        idx, val = zip(*[teacher(mk, r, V, top) for r in rows])
        wt = [mk.vec(r, 0.2, 1.0) for r in rows]
        for w in wt:
            if w.numel() > 2:
                w[2] = 0.0
        d = [mk.view(r, V, t) for r in rows]
        loss, lse, _ = ctx.distill_loss(logits, idx, val, tau, row_weight=wt, dlogits=d)
        only, _, none = ctx.distill_loss(logits, idx, val, tau, row_weight=wt, want_grad=False)
        ctx.synchronize()
        assert none is None
        for q, r in enumerate(rows):
            what = f"{dtype} {rows} x {V} top {top} worker {q} "
            if r == 0:
                continue
            rl, re, rd, tl, te, td = distill_reference(logits[q], idx[q], val[q], tau, wt[q], t)
            close(lse[q], re, te, what + "lse")
            close(loss[q], rl, tl, what + "loss")
            close(only[q], rl, tl, what + "loss alone")
            close(d[q], rd, td, what + "dlogits")
        mk.check_gaps()


def test_distill_loss_over_its_logits_gives_the_same(ctx):
    for V in (100, 5000, 40000, 140000):
        for t in (torch.float32, torch.bfloat16):
            mk = Maker(V)
            logits = mk.normal(5, V, t, 2.0)
            idx, val = teacher(mk, 5, V, 40)
            want = ctx.distill_loss([logits], [idx], [val], 2.0)
            x = logits.clone()
            got = ctx.distill_loss([x], [idx], [val], 2.0, dlogits=[x])
            ctx.synchronize()
            for a, b in zip(want, got):
                assert torch.equal(a[0], b[0])


def test_distill_rows_that_masks_leave_empty(ctx):
    V, t = 3000, torch.float32
    mk = Maker(4)
    logits = mk.normal(10, V, t, 2.0)
    idx, val = teacher(mk, 10, V, 16, short=False)
    wt = torch.ones(10, device="cuda")
    idx[0] = -1                                        # no entries
    val[1] = -float("inf")                             # entries without probability
    wt[2] = 0.0                                        # padding: whatever it holds
    logits[2] = float("nan")
    logits[0, 7] = float("nan")
    logits[3, 100:] = -float("inf")                    # a masked vocabulary, the teacher inside it
    idx[3] = torch.arange(16, dtype=torch.int32, device="cuda")
    logits[4, int(idx[4, 0])] = -float("inf")          # the student rules out what the teacher has
    logits[5] = torch.finfo(t).min                     # a mask of the lowest value over everything
    idx[6, 3:] = -1
    idx[7, ::2] = -1
    val[8, 5] = -float("inf")
    idx[9, 1] = idx[9, 0]                              # an entry twice
    idx[9, 9] = idx[9, 0]
    d = [torch.full((10, V), 9.0, device="cuda")]
    loss, lse, _ = ctx.distill_loss([logits], [idx], [val], 1.5, row_weight=[wt], dlogits=d)
    ctx.synchronize()
    for r in (0, 1, 2):
        assert float(loss[0][r]) == 0.0 and bool((d[0][r] == 0).all()), r
    assert float(loss[0][4]) == float("inf")
    rl, re, rd, tl, te, td = distill_reference(logits, idx, val, 1.5, wt, t)
    for r in (3, 6, 7, 8, 9):
        close(loss[0][r], rl[r], tl[r], f"loss {r}")
        close(lse[0][r], re[r], te[r], f"lse {r}")
    for r in (3, 4, 6, 7, 8, 9):
        close(d[0][r], rd[r], td[r], f"dlogits {r}")
    assert bool((d[0][3, 100:] == 0).all())
    close(d[0][5], rd[5], 1e-6, "dlogits of equal logits")      # q = 1 / V: a rounding of 1e38 would show in lse, not in q's size


@pytest.mark.parametrize("V,top", [(300, 4), (300, 400), (140000, 4)])
def test_distill_teacher_values_far_from_zero(ctx, V, top):
    """p depends on the differences of the values alone: far values whose quotients by the temperature overflow, or lose the difference."""
    tau, mk = 0.7, Maker(16)
    logits = mk.normal(6, V, torch.float32)
    idx = torch.full((6, top), -1, dtype=torch.int32, device="cuda")
    val = torch.zeros((6, top), device="cuda")
    idx[:, :4] = torch.tensor([7, 100, 299, 1], dtype=torch.int32)
    val[0, :4] = torch.tensor([3e38, 2e38, -3e38, 1.0])
    val[1, :4] = torch.finfo(torch.float32).min                             # all equal: a quarter each
    val[2, :4] = torch.finfo(torch.float32).max
    val[3, :4] = 1e7 + torch.tensor([0.0, 1.0, 2.0, 3.0])                    # every value and difference exact
    val[4, :4] = -1e7 + torch.tensor([3.0, 1.0, 0.0, 2.0])
    val[5, :4] = torch.tensor([-float("inf"), -3e38, -3e38, -float("inf")])
    loss, _, d = ctx.distill_loss([logits], [idx], [val], tau)
    ctx.synchronize()
    v = val[:, :4].double()
    p = torch.softmax((v - v.amax(1, keepdim=True)) / tau, 1)
    logq = torch.log_softmax(logits.double() / tau, 1)
    q = logq.exp()
    # p: a quotient of at most 5 off by half a step of 8, an exponential and its sum a few steps; q: a product of at most 12 off by three
    # half steps of 16, an exponential and a sum of V terms in chains of V / 1024 and joined in twelve steps
    ep, eq = 32 * F, F * (64 + V / 256)
    dense = torch.zeros_like(q).scatter_add_(1, idx[:, :4].long(), p)
    want = tau * (q - dense)
    close(d[0], want, F * want.abs() + tau * (q * eq + dense * ep) + tiny(torch.float32), "dlogits")
    terms = torch.where(p > 0, p * (p.clamp(min=1e-300).log() - logq.gather(1, idx[:, :4].long())), torch.zeros_like(p))
    close(loss[0], tau * tau * terms.sum(1), tau * tau * (terms.abs().sum(1) * ep + eq + ep + 32 * F), "loss")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [7, 301, 9001, 140001])
def test_distill_logits_of_plus_infinity(ctx, dtype, V):
    """lse is infinite; q is 0 beside such a logit and undefined at it; a NaN in the row still goes through.  The last element lies behind
    the whole vectors."""
    mk, t = Maker(17), TYPES[dtype]
    logits = mk.normal(6, V, t)
    idx = torch.tensor([[1, 2]] * 6, dtype=torch.int32, device="cuda")
    val = torch.tensor([[0.5, 0.25]] * 6, device="cuda")
    inf, places = float("inf"), [[V // 2], [V - 1], [0, V - 1], [1], [V // 2], []]
    for r, at in enumerate(places):
        for i in at:
            logits[r, i] = inf
    logits[4, V - 2] = float("nan")
    if dtype != "f16":
        logits[2, 3] = torch.finfo(t).max
    p = torch.softmax(val.double(), 1)[0]
    loss, lse, d = ctx.distill_loss([logits], [idx], [val])
    only, lse2, _ = ctx.distill_loss([logits], [idx], [val], want_grad=False)
    ctx.synchronize()
    for e in (lse[0], lse2[0]):
        assert e[:4].tolist() == [inf] * 4 and bool(e[4].isnan()) and bool(e[5].isfinite())
    for l in (loss[0], only[0]):
        assert l[:3].tolist() == [inf] * 3 and bool(l[3:5].isnan().all()) and bool(l[5].isfinite())
    for r in range(4):
        own = torch.zeros(V, dtype=torch.bool, device="cuda")
        own[places[r]] = True
        want = torch.zeros(V, dtype=torch.float64, device="cuda")
        want[1], want[2] = -p[0], -p[1]
        assert bool(d[0][r][own].isnan().all())
        close(d[0][r][~own], want[~own], 2 * u(t) * want[~own].abs(), f"dlogits {r}")
    assert bool(d[0][5].isfinite().all())


def test_distill_nan_goes_through(ctx):
    mk = Maker(14)
    for V in (300, 140000):
        logits = mk.normal(4, V, torch.float32)
        idx, val = teacher(mk, 4, V, 5, short=False)
        val[0, 2] = float("nan")
        val[1] = float("nan")                          # every entry
        logits[2, 11] = float("nan")
        loss, lse, d = ctx.distill_loss([logits], [idx], [val])
        ctx.synchronize()
        assert bool(loss[0][:3].isnan().all()) and bool(loss[0][3].isfinite())
        assert bool(d[0][:3].isnan().any(1).all()) and bool(d[0][3].isfinite().all())
        assert bool(lse[0][[0, 1, 3]].isfinite().all()) and bool(lse[0][2].isnan())


def test_distill_all_logits_masked_and_no_teacher_at_all(ctx):
    logits = torch.full((2, 100), -float("inf"), device="cuda")
    idx = torch.full((2, 4), -1, dtype=torch.int32, device="cuda")
    val = torch.zeros((2, 4), device="cuda")
    loss, lse, d = ctx.distill_loss([logits], [idx], [val])
    l0, _, d0 = ctx.distill_loss([torch.randn(2, 100, device="cuda")], [idx[:, :0]], [val[:, :0]])
    ctx.synchronize()
    assert bool((loss[0] == 0).all()) and bool((d[0] == 0).all()) and bool((lse[0] == -float("inf")).all())
    assert bool((l0[0] == 0).all()) and bool((d0[0] == 0).all())


def test_distill_index_outside_the_vocabulary_is_reported_and_taken_as_none():
    sd = binding.SlimDP(1000, 1)
    mk = Maker(2)
    logits = mk.normal(3, 500, torch.float32)
    idx, val = teacher(mk, 3, 500, 8, short=False)
    good = idx.clone()
    good[1, 2] = -1
    want = sd.distill_loss([logits], [good], [val])
    sd.synchronize()
    for outside in (500, 2 ** 31 - 1, -2):
        idx[1, 2] = outside
        got = sd.distill_loss([logits], [idx], [val])
        with pytest.raises(binding.SlimDPError) as e:
            sd.synchronize()
        assert e.value.code == binding.ERR_DEVICE_STATUS and "vocabulary" in str(e.value)
        for a, b in zip(want, got):
            assert torch.equal(a[0], b[0])
        sd.synchronize()                               # reported once
    sd.close()


def test_rows_that_lie_further_apart_than_32_bits_reach(ctx):
    """Inputs and outputs whose last rows begin behind 2^32 bytes and 2^31 elements: the same bits as of the rows side by side."""
    R, ld, t = 40_000, 60_000, torch.bfloat16
    mk = Maker(15)
    big = [torch.empty((R, ld), dtype=t, device="cuda") for _ in range(2)]
    x = mk.normal(R, 200, t)
    far, out = big[0][:, 24:224], big[1][:, 7:207]
    far.copy_(x)
    w, b = mk.vec(200), mk.vec(200)
    y, mean, rstd = ctx.layer_norm([x], [w], [b])
    _, m2, r2 = ctx.layer_norm([far], [w], [b], y=[out])
    ctx.synchronize()
    assert torch.equal(out, y[0]) and torch.equal(m2[0], mean[0]) and torch.equal(r2[0], rstd[0])
    dx, dw, _ = ctx.layer_norm_backward([x], y, [w], mean, rstd)
    _, dw2, _ = ctx.layer_norm_backward([far], y, [w], mean, rstd, dx=[out])
    ctx.synchronize()
    assert torch.equal(out, dx[0]) and torch.equal(dw[0], dw2[0])
    W = mk.normal(200, 200, t, 0.07)
    z, _ = ctx.linear([x], [W], [b], "silu", residual=y)
    ctx.linear([far], [W], [b], "silu", residual=y, y=[out])
    ctx.synchronize()
    assert torch.equal(out, z[0])
    dx, dw = ctx.linear_backward([x], y, [W])
    _, dw2 = ctx.linear_backward([far], y, [W], dx=[out])
    ctx.synchronize()
    assert torch.equal(out, dx[0]) and torch.equal(dw[0], dw2[0])
    dz, db = ctx.linear_epilogue_backward([x], y, "gelu")
    _, db2 = ctx.linear_epilogue_backward([far], y, "gelu", dz=[out])
    ctx.synchronize()
    assert torch.equal(out, dz[0]) and torch.equal(db[0], db2[0])
    idx, val = teacher(mk, R, 200, 3)
    l1, e1, d1 = ctx.distill_loss([x], [idx], [val])
    l2, e2, _ = ctx.distill_loss([far], [idx], [val], dlogits=[out])
    ctx.synchronize()
    assert torch.equal(l1[0], l2[0]) and torch.equal(e1[0], e2[0]) and torch.equal(out, d1[0])
    del big, far, out
    torch.cuda.empty_cache()


# ---------------------------------------------------------------------------------------------------------------
# all of them
# ---------------------------------------------------------------------------------------------------------------
def everything(sd, mk, W, rows, D, H, V, t):
    """One call of each on small inputs; a list of all outputs."""
    x, w, b = [mk.normal(rows, D, t) for _ in range(W)], [mk.vec(D) for _ in range(W)], [mk.vec(D) for _ in range(W)]
    W1, b1 = [mk.normal(H, D, t, 0.1) for _ in range(W)], [mk.vec(H) for _ in range(W)]
    lg = [mk.normal(rows, V, t) for _ in range(W)]
    idx, val = zip(*[teacher(mk, rows, V, 12) for _ in range(W)])
    dh = [mk.normal(rows, H, t) for _ in range(W)]

    def run():
        y, mean, rstd = sd.layer_norm(x, w, b)
        h, z = sd.linear(y, W1, b1, "gelu", keep=True)
        dz, db1 = sd.linear_epilogue_backward(dh, z, "gelu")
        dy, dw1 = sd.linear_backward(dz, y, W1)
        dx, dw, db = sd.layer_norm_backward(dy, x, w, mean, rstd)
        loss, lse, dl = sd.distill_loss(lg, idx, val, 2.0)
        return [v for part in (y, mean, rstd, h, z, dz, db1, dy, dw1, dx, dw, db, loss, lse, dl) for v in part]
    return run, x


@pytest.mark.parametrize("dtype", DTYPES)
def test_operators_on_another_stream_and_twice_at_once(dtype):
    """Two contexts on streams of their own, neither the current one, at the same time: same bits as alone."""
    t = TYPES[dtype]
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    a, b = binding.SlimDP(100, 3, stream=s1), binding.SlimDP(100, 3, stream=s2)
    run_a, _ = everything(a, Maker(1), 3, 150, 200, 264, 1000, t)
    run_b, _ = everything(b, Maker(2), 2, 90, 520, 72, 3001, t)
    torch.cuda.synchronize()
    want_a = run_a()
    a.synchronize()
    want_b = run_b()
    b.synchronize()
    for _ in range(5):
        got_a, got_b = run_a(), run_b()
        junk = torch.full((1 << 20,), float("nan"), device="cuda")          # the current stream's own allocations meanwhile
        a.synchronize(), b.synchronize()
        del junk
        assert all(torch.equal(p, q) for p, q in zip(want_a, got_a))
        assert all(torch.equal(p, q) for p, q in zip(want_b, got_b))
    a.close(), b.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_operators_recorded_and_replayed(dtype):
    t = TYPES[dtype]
    stream = torch.cuda.Stream()
    sd = binding.SlimDP(100, 2, stream=stream)
    run, x = everything(sd, Maker(3), 2, 70, 328, 200, 2000, t)
    torch.cuda.synchronize()
    run()
    sd.synchronize()
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1, stream=stream):
        out1 = run()
    with torch.cuda.graph(g2, stream=stream):
        out2 = run()
    for turn in range(4):
        for v in x:
            v.mul_(0.9).add_(0.01 * turn)
        torch.cuda.synchronize()
        want = [v.clone() for v in run()]
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            g1.replay()
            g2.replay()
        sd.synchronize()
        for w, p, q in zip(want, out1, out2):
            assert torch.equal(w, p) and torch.equal(w, q)
    sd.close()


def test_operators_of_32_workers_each_get_their_own(ctx):
    W = 32
    run, _ = everything(ctx, Maker(5), W, 21, 72, 40, 130, torch.float32)
    all_out = run()
    ctx.synchronize()
    run1, _ = everything(ctx, Maker(5), W, 21, 72, 40, 130, torch.float32)
    again = run1()
    ctx.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(all_out, again))
    for part in range(15):
        vals = all_out[part * W:(part + 1) * W]
        assert not any(torch.equal(vals[0], v) for v in vals[1:])


class Net:
    """Two workers' local models of one block: norm -> linear, gelu -> linear + residual -> norm -> vocabulary, flat in one vector each."""

    def __init__(self, D, H, V):
        shapes = [("g1", (D,)), ("c1", (D,)), ("w1", (H, D)), ("b1", (H,)), ("w2", (D, H)), ("b2", (D,)), ("g2", (D,)), ("c2", (D,)), ("wv", (V, D))]
        self.shapes, self.off, at = shapes, {}, 0
        for name, s in shapes:
            self.off[name] = at
            at += int(np.prod(s))
        self.n = at

    def part(self, flat, name):
        s = dict(self.shapes)[name]
        return flat[self.off[name]:self.off[name] + int(np.prod(s))].view(*s)

    def parts(self, flats, name):
        return [self.part(f, name) for f in flats]


def net_loss64(net, flat, x, idx, val, tau, weight):
    """The same in 64 bits with torch's own differentiation."""
    p = lambda name: net.part(flat, name)
    ln = lambda v, g, c: (v - v.mean(1, keepdim=True)) / (v.var(1, unbiased=False, keepdim=True) + 1e-5).sqrt() * g + c
    h = ln(x, p("g1"), p("c1")) @ p("w1").t() + p("b1")
    r = act_value(h, "gelu") @ p("w2").t() + p("b2") + x
    s = ln(r, p("g2"), p("c2")) @ p("wv").t() / tau
    lt = torch.log_softmax(torch.where(idx >= 0, val / tau, torch.full_like(val, -math.inf)), 1)
    pt = torch.where(idx >= 0, lt.exp(), torch.zeros_like(lt))
    lq = torch.log_softmax(s, 1).gather(1, idx.clamp(min=0).long())
    return (weight * tau * tau * torch.where(pt > 0, pt * (lt - lq), torch.zeros_like(pt)).sum(1)).sum()


def test_a_workers_mini_batch_from_the_local_model_to_the_push(ctx):
    """Forward and backward pass of two workers' mini-batches with parameters and gradients in the flat vectors of the path, in two
    parts of a mini-batch each, then the local step fused with the extraction, merge and pull: gradients against 64 bits and against
    differences, the rest to the bit against the oracle."""
    import oracle
    D, H, V, tau, eta, W = 40, 104, 301, 2.0, 0.05, 2
    rows = [[9, 14], [7, 0]]                                   # per part and worker
    net = Net(D, H, V)
    mk = Maker(77)
    w0 = (mk.g.normal(0, 0.15, net.n)).astype(np.float32)
    for name in ("g1", "g2"):
        w0[net.off[name]:net.off[name] + D] += 1.0
    sd = binding.SlimDP(net.n, W, seed=3)
    w = torch.from_numpy(w0).cuda()
    local = [w.clone() for _ in range(W)]
    grad, delta = [torch.full_like(w, float("nan")) for _ in range(W)], [torch.zeros_like(w) for _ in range(W)]
    x = [[mk.normal(r, D, torch.float32) for r in part] for part in rows]
    teach = [[teacher(mk, r, V, 6, short=False) for r in part] for part in rows]
    wt = [[torch.full((r,), 1.0 / 23, device="cuda") for r in part] for part in rows]
    total = np.zeros(W)
    for part in range(2):
        add = part > 0
        P, G = (lambda name: net.parts(local, name)), (lambda name: net.parts(grad, name))
        n1, m1, r1 = sd.layer_norm(x[part], P("g1"), P("c1"))
        h, z = sd.linear(n1, P("w1"), P("b1"), "gelu", keep=True)
        r, _ = sd.linear(h, P("w2"), P("b2"), residual=x[part])
        n2, m2, r2 = sd.layer_norm(r, P("g2"), P("c2"))
        logits, _ = sd.linear(n2, P("wv"))
        loss, _, dl = sd.distill_loss(logits, [t[0] for t in teach[part]], [t[1] for t in teach[part]], tau, row_weight=wt[part], dlogits=logits)
        dn2, _ = sd.linear_backward(dl, n2, P("wv"), dweight=G("wv"), accumulate=add)
        dr, _, _ = sd.layer_norm_backward(dn2, r, P("g2"), m2, r2, dweight=G("g2"), dbias=G("c2"), accumulate=add)
        sd.linear_epilogue_backward(dr, dbias=G("b2"), accumulate=add)
        dh, _ = sd.linear_backward(dr, h, P("w2"), dweight=G("w2"), accumulate=add)
        dz, _ = sd.linear_epilogue_backward(dh, z, "gelu", dbias=G("b1"), accumulate=add)
        dn1, _ = sd.linear_backward(dz, n1, P("w1"), dweight=G("w1"), accumulate=add)
        dx, _, _ = sd.layer_norm_backward(dn1, x[part], P("g1"), m1, r1, dweight=G("g1"), dbias=G("c1"), accumulate=add)
        sd.synchronize()
        total += [float(v.double().sum()) for v in loss]
    worst = 0.0
    for q in range(W):
        flat = local[q].double().requires_grad_(True)
        want = sum(net_loss64(net, flat, x[p][q].double(), teach[p][q][0], teach[p][q][1].double(), tau, wt[p][q].double())
                   for p in range(2) if rows[p][q])
        want.backward()
        # the whole chain in binary32: some two hundred roundings along the longest way from a parameter to the loss and back, on values
        # whose size (not the sum's, which may cancel) is bounded by the gradient's largest entry times the block's width
        tol = 256 * F * float(flat.grad.abs().max()) * 16 + 1e-9
        close(grad[q], flat.grad, tol, f"gradient of worker {q}")
        assert abs(total[q] - float(want.detach())) <= 256 * F * 16 * max(1.0, abs(float(want.detach())))
        # differences of the 64-bit loss along a few coordinates of every parameter
        for name, shape in net.shapes:
            for i in mk.g.integers(0, int(np.prod(shape)), 2):
                j = net.off[name] + int(i)
                e = 1e-4
                both = []
                for sign in (1, -1):
                    f = local[q].double()
                    f[j] += sign * e
                    both.append(float(sum(net_loss64(net, f, x[p][q].double(), teach[p][q][0], teach[p][q][1].double(), tau, wt[p][q].double())
                                          for p in range(2) if rows[p][q])))
                diff = (both[0] - both[1]) / (2 * e)
                assert abs(diff - float(grad[q][j])) <= 1e-5 * max(1.0, float(flat.grad.abs().max())), (name, int(i))
    # and into the path
    g_h, k, m = [g.cpu().numpy() for g in grad], net.n // 10, net.n // 50
    S = sd.score(w, grad, 1.0)
    core_idx, core_bits, core_off, epoch = sd.select_core(S, [k], reuse_histogram=True)
    ei, eo = sd.sample_explore(core_bits, [k], 0, [m], 0, W)
    cv, ev = sd.local_step_pack(local, grad, delta, eta, True, core_idx, core_off, ei, eo, epoch)
    sd.merge(w, eta, epoch, core_idx, core_off, cv, ei, eo, ev)
    sd.synchronize()
    core_o = oracle.select_core(oracle.score(w0, g_h, 1.0), k)
    assert np.array_equal(core_idx.cpu().numpy().view(np.uint32), core_o)
    ei_o = [oracle.sample_explore(net.n, core_o, 3, 0, q, m) for q in range(W)]
    packs = [oracle.pack(g_h[q], core_o, ei_o[q]) for q in range(W)]
    w_o = oracle.merge(w0, eta, core_o, [p[0] for p in packs], ei_o, [p[1] for p in packs])
    assert np.array_equal(w.cpu().numpy().view(np.uint32), w_o.view(np.uint32))
    sd.close()


# ---------------------------------------------------------------------------------------------------------------
# refusals
# ---------------------------------------------------------------------------------------------------------------
def test_refusals_of_the_c_entries(ctx):
    """Every wrong argument is refused before anything is enqueued: the outputs keep what they held."""
    import ctypes as C
    L, h = ctx._L, ctx._h
    n = (C.c_uint64 * 1)(4)
    keep = torch.full((4096,), 5.0, device="cuda")
    buf = torch.zeros(4096, device="cuda")
    tab = lambda p: (C.c_void_p * 1)(p)
    a, o, vec, odd = tab(buf.data_ptr()), tab(keep.data_ptr()), tab(buf.data_ptr() + 8192), tab(buf.data_ptr() + 2)
    OKAY, INV, RANGE, WS = binding.OK, binding.ERR_INVALID_ARG, binding.ERR_OUT_OF_RANGE, binding.ERR_WORKSPACE
    big = (C.c_uint64 * 1)(binding.MAX_ROWS + 1)

    def norm(W=1, rows=n, cols=16, dt=0, x=a, ldx=16, w=vec, b=vec, eps=1e-5, y=o, ldy=16, mean=None, rstd=None):
        return L.slimdp_layer_norm(h, W, rows, cols, dt, x, ldx, w, b, eps, y, ldy, mean, rstd)
    for want, kw in [(INV, dict(W=0)), (INV, dict(W=33)), (INV, dict(rows=None)), (INV, dict(dt=3)), (INV, dict(cols=0)), (RANGE, dict(cols=65537, ldx=70000, ldy=70000)),
                     (INV, dict(x=None)), (INV, dict(x=tab(None))), (INV, dict(ldx=15)), (INV, dict(ldy=3)), (INV, dict(y=None)), (INV, dict(eps=0.0)),
                     (INV, dict(eps=float("nan"))), (INV, dict(eps=float("inf"))), (INV, dict(eps=-1.0)), (RANGE, dict(rows=big)), (INV, dict(x=odd)),
                     (INV, dict(w=odd)), (INV, dict(y=a, ldy=20)), (INV, dict(mean=tab(None)))]:
        assert norm(**kw) == want, kw
        assert L.slimdp_last_error(h), kw
    assert L.slimdp_layer_norm(None, 1, n, 16, 0, a, 16, vec, vec, 1e-5, o, 16, None, None) == INV

    def back(dy=a, x=vec, mean=vec, rstd=vec, dx=o, lddx=16, dw=None, db=None, flags=0, ws=None, nb=0, rows=n):
        return L.slimdp_layer_norm_backward(h, 1, rows, 16, 0, dy, 16, x, 16, vec, mean, rstd, dx, lddx, dw, db, flags, ws, nb)
    many = (C.c_uint64 * 1)(4000)
    need = L.slimdp_layer_norm_workspace_bytes(1, many, 16, 0)
    assert need > 0 and L.slimdp_layer_norm_workspace_bytes(1, n, 16, 0) == 0
    for want, kw in [(INV, dict(flags=2)), (INV, dict(dy=None)), (INV, dict(mean=None)), (INV, dict(rstd=tab(None))), (INV, dict(dx=a, lddx=17)),
                     (WS, dict(rows=many, dw=o)), (WS, dict(rows=many, dw=o, ws=buf.data_ptr(), nb=need - 1)),
                     (INV, dict(rows=many, dw=o, ws=buf.data_ptr() + 4, nb=need))]:
        assert back(**kw) == want, kw

    def lin(rows=n, cin=8, cout=8, dt=0, x=a, ldx=8, w=vec, ldw=8, b=None, act=0, r=None, ldr=8, y=o, ldy=8, z=None, ldz=8, ws=None, nb=0):
        return L.slimdp_linear(h, 1, rows, cin, cout, dt, x, ldx, w, ldw, b, act, r, ldr, y, ldy, z, ldz, ws, nb)
    for want, kw in [(INV, dict(act=5)), (INV, dict(cin=0)), (INV, dict(cout=0)), (RANGE, dict(cin=binding.MAX_FEATURES + 1)), (INV, dict(w=None)), (INV, dict(w=tab(None))),
                     (INV, dict(ldw=7)), (INV, dict(y=a)), (INV, dict(y=vec)), (INV, dict(z=o)), (INV, dict(r=a, y=a)), (INV, dict(r=o, ldr=9)), (INV, dict(r=o, z=o)),
                     (INV, dict(x=odd)), (INV, dict(dt=9)), (INV, dict(b=odd)), (WS, dict(cin=4096, ldx=4096, ldw=4096))]:
        assert lin(**kw) == want, kw

    def epi(act=1, z=a, dz=o, lddz=8, flags=0, dy=vec, db=None):
        return L.slimdp_linear_epilogue_backward(h, 1, n, 8, 0, dy, 8, z, 8, act, dz, lddz, db, flags, None, 0)
    for want, kw in [(INV, dict(act=7)), (INV, dict(z=None)), (INV, dict(dy=None)), (INV, dict(flags=4)), (INV, dict(dz=vec, lddz=9)), (INV, dict(db=odd))]:
        assert epi(**kw) == want, kw

    def lback(dz=a, x=vec, w=vec, dx=o, dw=None, flags=0):
        return L.slimdp_linear_backward(h, 1, n, 8, 8, 0, dz, 8, x, 8, w, 8, dx, 8, dw, flags, None, 0)
    for want, kw in [(INV, dict(dz=None)), (INV, dict(w=None)), (INV, dict(x=None, dw=o, dx=None)), (INV, dict(dx=a)), (INV, dict(flags=2)), (INV, dict(dw=tab(None)))]:
        assert lback(**kw) == want, kw

    def dist(V=100, dt=0, x=a, ldl=100, top=4, i=vec, v=vec, ldt=4, tau=1.0, w=None, loss=None, lse=None, d=o, ldd=100):
        return L.slimdp_distill_loss(h, 1, n, V, dt, x, ldl, top, i, v, ldt, tau, w, loss, lse, d, ldd)
    for want, kw in [(INV, dict(V=0)), (RANGE, dict(V=binding.MAX_VOCAB + 1, ldl=1 << 25, ldd=1 << 25)), (RANGE, dict(top=1025, ldt=1025)), (INV, dict(i=None)), (INV, dict(v=None)),
                     (INV, dict(ldt=3)), (INV, dict(ldl=99)), (INV, dict(tau=0.0)), (INV, dict(tau=-1.0)), (INV, dict(tau=float("nan"))), (INV, dict(tau=float("inf"))),
                     (INV, dict(tau=1e-45)), (INV, dict(tau=3e-39)), (INV, dict(d=a, ldd=101)), (INV, dict(x=None)), (INV, dict(w=odd))]:
        assert dist(**kw) == want, kw
    assert norm(mean=o, rstd=o) == INV and back(rows=n, dw=vec, db=vec) == INV and dist(loss=vec, lse=vec) == INV
    two = (C.c_uint64 * 2)(4, 4)
    # one worker's output over another's input: also where a worker's own would be allowed
    cross, here = (C.c_void_p * 2)(buf.data_ptr(), keep.data_ptr()), (C.c_void_p * 2)(keep.data_ptr(), buf.data_ptr() + 4096)
    assert L.slimdp_layer_norm(h, 2, two, 16, 0, cross, 16, None, None, 1e-5, here, 16, None, None) == INV
    assert L.slimdp_linear_epilogue_backward(h, 2, two, 8, 0, cross, 8, cross, 8, 1, here, 8, None, 0, None, 0) == INV
    xs, ys = (C.c_void_p * 2)(buf.data_ptr(), buf.data_ptr()), (C.c_void_p * 2)(keep.data_ptr(), keep.data_ptr())
    assert L.slimdp_layer_norm(h, 2, two, 16, 0, xs, 16, None, None, 1e-5, ys, 16, None, None) == INV      # one output for two workers
    ctx.synchronize()
    assert bool((keep == 5.0).all())
    zero = (C.c_uint64 * 1)(0)
    assert norm(rows=zero, x=tab(None), y=tab(None)) == OKAY and norm() == OKAY
    ctx.synchronize()


def test_results_of_more_tiles_than_a_grid_numbers_are_refused_before_anything_runs(ctx):
    """Also where the second of a call's two products is the one that is too large: the first is not launched either."""
    import ctypes as C
    L, h, most = ctx._L, ctx._h, binding.MAX_FEATURES
    keep, ws = torch.full((4096,), 5.0, device="cuda"), torch.zeros(1 << 20, device="cuda")
    o, a = (C.c_void_p * 1)(keep.data_ptr()), (C.c_void_p * 1)(ws.data_ptr())
    b = (C.c_void_p * 1)(ws.data_ptr() + 4096)
    n = (C.c_uint64 * 1)(4)
    assert (most // 64) ** 2 > binding.MAX_TILES >= most // 64
    rc = L.slimdp_linear_backward(h, 1, n, most, most, 0, a, most, b, most, b, most, o, most, (C.c_void_p * 1)(ws.data_ptr() + 8192), 0, ws.data_ptr(), 1 << 62)
    assert rc == binding.ERR_OUT_OF_RANGE and b"tiles" in L.slimdp_last_error(h)
    n = (C.c_uint64 * 1)(binding.MAX_ROWS)
    assert L.slimdp_linear(h, 1, n, 8, 2049, 0, a, 8, b, 8, None, 0, None, 0, o, 2049, None, 0, ws.data_ptr(), 1 << 62) == binding.ERR_OUT_OF_RANGE
    assert b"tiles" in L.slimdp_last_error(h)
    assert L.slimdp_linear_backward(h, 1, n, 2049, 8, 0, a, 8, None, 0, b, 2049, o, 2049, None, 0, ws.data_ptr(), 1 << 62) == binding.ERR_OUT_OF_RANGE
    ctx.synchronize()
    assert bool((keep == 5.0).all())


def check_products(ctx, mk, R, K, N, t, what):
    x, w, dz, res = mk.normal(R, K, t), mk.normal(N, K, t, 0.03), mk.normal(R, N, t, 0.1), mk.normal(R, N, t)
    b, old = mk.vec(N), mk.vec(N * K).view(N, K)
    y, _ = ctx.linear([x], [w], [b], "none", [res])
    dx, dw = ctx.linear_backward([dz], [x], [w])
    add = [old.clone()]
    ctx.linear_backward([dz], [x], None, dweight=add, want_dx=False, accumulate=True)
    ctx.synchronize()
    xd, wd, zd = x.double(), w.double(), dz.double()
    # two additions behind the sum, of bias and residual, each rounded once to binary32; one behind the weight's gradient
    ref, e = xd @ wd.t(), 1.01 * steps(K, t) * F * (xd.abs() @ wd.abs().t())
    one, two = ref + b.double(), ref + b.double() + res.double()
    close(y[0], two, u(t) * two.abs() + 1.01 * (e + F * (one.abs() + two.abs())) + tiny(t), what + " y")
    ref = zd @ wd
    close(dx[0], ref, u(t) * ref.abs() + 1.01 * steps(N, t) * F * (zd.abs() @ wd.abs()) + tiny(t), what + " dx")
    ref, e = zd.t() @ xd, 1.01 * steps(R, t) * F * (zd.abs().t() @ xd.abs()) + 1e-30
    close(dw[0], ref, F * ref.abs() + e, what + " dweight")
    both = ref + old.double()
    close(add[0], both, 1.01 * e + F * (ref.abs() + both.abs()), what + " dweight added")
    mk.check_gaps()


@pytest.mark.parametrize("R,K,N,pad,shift", [(2100, 1032, 2312, 0, 0), (2101, 1033, 2311, 3, 1), (1, 2001, 3005, 0, 0), (3, 2050, 4001, 1, 3), (2, 5, 4, 0, 0),
                                             (640, 3, 2000, 0, 0), (5000, 2000, 3, 0, 1), (70, 4, 4100, 0, 0), (65, 6000, 66, 0, 0)])
def test_products_in_binary32_of_every_tile(ctx, R, K, N, pad, shift):
    """Large tiles and small ones, sums in pieces and whole, one to three rows, rows shorter than four elements; every element."""
    check_products(ctx, Maker(31, pad, shift), R, K, N, torch.float32, f"{R} {K} {N}")


def test_products_with_rows_far_apart(ctx):
    """Distances between rows that no 32-bit offset of a tile holds."""
    for t in (torch.bfloat16, torch.float16):
        check_products(ctx, Maker(32, (1 << 21) + 5, 1), 67, 75, 70, t, str(t))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R", [1, 17, 40, 64])
def test_few_rows_with_every_share_of_a_wave(ctx, dtype, R):
    """Rows shorter than a vector, waves without a share, with one to several turns of steps, and ends inside a vector."""
    for pad, shift, K in ((0, 0, 3), (1, 1, 9), (0, 0, 33), (3, 1, 130), (0, 0, 999), (8, 8, 1280), (5, 3, 1290), (0, 0, 2049), (0, 0, 2600), (1, 0, 4111)):
        check_products(ctx, Maker(33, pad, shift), R, K, 1040, TYPES[dtype], f"{dtype} {R} {K}")


def check_workers(ctx, rows, K, N, t, pad=0, shift=0):
    """The three products of several workers, element by element; gradients added up as well."""
    mk = Maker(34, pad, shift)
    W, what = len(rows), f"{rows} x {K} x {N} "
    x, dz, w = [mk.normal(r, K, t) for r in rows], [mk.normal(r, N, t, 0.1) for r in rows], [mk.normal(N, K, t, 0.03) for _ in rows]
    y, dx, old = [mk.view(r, N, t) for r in rows], [mk.view(r, K, t) for r in rows], [mk.vec(N * K).view(N, K) for _ in rows]
    add = [v.clone() for v in old]
    ctx.linear(x, w, y=y)
    _, dw = ctx.linear_backward(dz, x, w, dx=dx)
    ctx.linear_backward(dz, x, None, dweight=add, want_dx=False, accumulate=True)
    ctx.synchronize()
    for q in range(W):
        xd, wd, zd = x[q].double(), w[q].double(), dz[q].double()
        ref = xd @ wd.t()
        close(y[q], ref, u(t) * ref.abs() + 1.01 * steps(K, t) * F * (xd.abs() @ wd.abs().t()) + tiny(t), what + f"y {q}")
        ref = zd @ wd
        close(dx[q], ref, u(t) * ref.abs() + 1.01 * steps(N, t) * F * (zd.abs() @ wd.abs()) + tiny(t), what + f"dx {q}")
        zt = zd.t().contiguous()
        ref, e = zt @ xd, 1.01 * steps(rows[q], t) * F * (zt.abs() @ xd.abs()) + 1e-30
        close(dw[q], ref, F * ref.abs() + e, what + f"dweight {q}")
        both = ref + old[q].double()
        close(add[q], both, 1.01 * e + F * (ref.abs() + both.abs()), what + f"dweight added {q}")
    mk.check_gaps()


@pytest.mark.parametrize("rows,K,N", [([1529], 832, 1119), ([24], 3592, 1608), ([58, 3], 1592, 608), ([2500], 1000, 16), ([1300], 24, 700), ([1100], 700, 40),
                                      ([2300, 0, 1, 33], 130, 97), ([0, 0, 5, 0, 900], 33, 260), ([700, 31, 32, 33, 0, 1, 64, 65], 100, 72), ([5], 4, 4),
                                      ([31] * 32, 36, 68), ([4000, 20], 17, 19), ([333], 4097, 5), ([9], 5, 4097)])
def test_products_in_binary32_of_uneven_workers_and_thin_results(ctx, rows, K, N):
    """Sums in one and in many pieces (fewer of them for workers with few rows), tiles of every width, and edges inside a vector."""
    for pad, shift in ((0, 0), (3, 1)):
        check_workers(ctx, rows, K, N, torch.float32, pad, shift)


def test_products_in_binary32_of_more_blocks_than_one_dimension_numbers(ctx):
    rows, K, N = 1 << 20, 4, 4160
    x, w = torch.randn(rows, K, device="cuda"), torch.randn(N, K, device="cuda")
    y = torch.full((rows, N), float("nan"), device="cuda")
    assert -(-rows // 64) * -(-N // 64) > 1 << 20
    ctx.linear([x], [w], y=[y])
    ctx.synchronize()
    wt, mag = w.double().t().contiguous(), w.double().abs().t().contiguous()
    for a in range(0, rows, 1 << 16):
        xd = x[a:a + (1 << 16)].double()
        close(y[a:a + (1 << 16)], xd @ wt, 5 * F * (xd.abs() @ mag), f"rows {a}")           # four products in one instruction's chain
    del y
    torch.cuda.empty_cache()


@pytest.mark.parametrize("R,K,N,what", [(58, 3592, 4608, "forward"), (13286, 6638, 16, "forward"), (2048, 2048, 2048, "forward"), (1772, 4388, 264, "dx"),
                                        (8608, 2496, 16, "dweight"), (1, 960, 6776, "dx")])
def test_products_in_binary32_keep_up_with_the_elementary_form(R, K, N, what):
    """Not slower than half again what torch's product takes (58 x 3592 x 4608 and 13,286 x 6638 x 16 once took two and three times it)."""
    import time
    sd = binding.SlimDP(100, 1)
    x, w, dz = (torch.randn(a, b, device="cuda") for a, b in ((R, K), (N, K), (R, N)))
    y, dx, dw = torch.empty_like(dz), torch.empty_like(x), torch.empty_like(w)
    own = {"forward": lambda: sd.linear([x], [w], y=[y]), "dx": lambda: sd.linear_backward([dz], None, [w], dx=[dx], want_dweight=False),
           "dweight": lambda: sd.linear_backward([dz], [x], None, dweight=[dw], want_dx=False)}[what]
    plain = {"forward": lambda: x @ w.t(), "dx": lambda: dz @ w, "dweight": lambda: dz.t() @ x}[what]
    torch.cuda.synchronize()

    def once(f):
        t = time.perf_counter()
        for _ in range(20):
            f()
        torch.cuda.synchronize()
        return time.perf_counter() - t
    once(own), once(plain)
    pairs = [(once(own), once(plain)) for _ in range(9)]
    a, b = (sorted(p[i] for p in pairs)[4] for i in (0, 1))
    assert a < 1.5 * b + 20 * 5e-6, (a / 20 * 1e6, b / 20 * 1e6)                            # 5 us: a second launch from the host
    sd.close()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows,K,N", [([2300, 0, 1, 33], 136, 104), ([0, 0, 5, 0, 900], 40, 264), ([700, 31, 32, 33, 0, 1, 64, 65], 104, 72), ([4100, 0, 40, 1030], 1032, 2312),
                                      ([0, 2500, 129], 2056, 520), ([70] * 32, 64, 48), ([1, 9000], 264, 264)])
def test_products_of_uneven_workers(ctx, dtype, rows, K, N):
    """Every tile, copied into the LDS and through registers, whole and in pieces, for workers of few rows beside others of many, or of none."""
    for pad, shift in ((0, 0), (8, 8), (3, 1)):
        check_workers(ctx, rows, K, N, TYPES[dtype], pad, shift)


@pytest.mark.parametrize("what", ["forward", "dx", "dweight"])
@pytest.mark.parametrize("rows", [[8192, 0, 0, 0, 0, 0, 0, 0], [0, 300, 7000, 892], [1, 4000, 4000, 63, 64, 64]])
def test_products_take_the_time_of_their_rows_however_the_workers_share_them(rows, what):
    """One worker with all the rows once took five to six times the time of eight with as many."""
    import time
    K, N, t = 2048, 2048, torch.bfloat16

    def call(rows):
        sd = binding.SlimDP(100, len(rows))
        x, dz = [torch.randn(r, K, device="cuda").to(t) for r in rows], [torch.randn(r, N, device="cuda").to(t) for r in rows]
        w = [torch.randn(N, K, device="cuda").to(t) for _ in rows]
        y, dx, dw = [torch.empty_like(v) for v in dz], [torch.empty_like(v) for v in x], [torch.empty((N, K), device="cuda") for _ in rows]
        return sd, {"forward": lambda: sd.linear(x, w, y=y), "dx": lambda: sd.linear_backward(dz, None, w, dx=dx, want_dweight=False),
                    "dweight": lambda: sd.linear_backward(dz, x, None, dweight=dw, want_dx=False)}[what]
    a, uneven = call(rows)
    b, equal = call([1024] * 8 if len(rows) == 8 else [8192 // len(rows)] * len(rows))

    def once(f):
        t0 = time.perf_counter()
        for _ in range(10):
            f()
        torch.cuda.synchronize()
        return time.perf_counter() - t0
    torch.cuda.synchronize()
    once(uneven), once(equal)
    pairs = [(once(uneven), once(equal)) for _ in range(9)]
    got, want = (sorted(p[i] for p in pairs)[4] for i in (0, 1))
    assert got < 1.6 * want, (got / 10 * 1e6, want / 10 * 1e6)
    a.close(), b.close()


def device_normal(seed, rows, cols, t, sigma=1.0, mean=0.0):
    """Large matrices are drawn where they are used."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.empty((rows, cols), device="cuda").normal_(mean, sigma, generator=g).to(t)


def check_norm(ctx, rows, cols, t):
    """Layer norm and its backward pass of several workers against 64 bits, with and without each other's outputs."""
    x = [device_normal(q, r, cols, t, 1.5, 0.7) for q, r in enumerate(rows)]
    dy = [device_normal(q + 100, r, cols, t, 0.3) for q, r in enumerate(rows)]
    mk = Maker(cols)
    w, b = [mk.vec(cols, 0.3, 1.0) for _ in rows], [mk.vec(cols, 0.3) for _ in rows]
    y, mean, rstd = ctx.layer_norm(x, w, b)
    dx, gw, gb = ctx.layer_norm_backward(dy, x, w, mean, rstd)
    _, gw2, gb2 = ctx.layer_norm_backward(dy, x, w, mean, rstd, want_dx=False)
    ctx.synchronize()
    for q, r in enumerate(rows):
        what, sw, sb, tw, tb = f"{t} {rows} x {cols} worker {q} ", 0.0, 0.0, 1e-30, 1e-30
        for a in range(0, r, 4096):
            part = slice(a, min(r, a + 4096))
            xd, dyd = x[q][part].double(), dy[q][part].double()
            ref, rm, rr, ty, tm, tr = norm_tolerance(xd, w[q].double(), b[q].double(), 1e-5, t)
            close(mean[q][part], rm, tm + tiny(torch.float32), what + "mean")
            close(rstd[q][part], rr, tr, what + "rstd")
            close(y[q][part], ref, ty, what + "y")
            ref, e, xh, exh = norm_back_reference(dyd, xd, w[q].double(), mean[q][part].double(), rstd[q][part].double())
            close(dx[q][part], ref, u(t) * ref.abs() + 1.01 * e + tiny(t), what + "dx")
            n = (r + 8) * F
            sw, sb = sw + (dyd * xh).sum(0), sb + dyd.sum(0)
            tw, tb = tw + n * (dyd.abs() * (xh.abs() + exh)).sum(0) + (dyd.abs() * exh).sum(0), tb + n * dyd.abs().sum(0)
        for got_w, got_b in ((gw[q], gb[q]), (gw2[q], gb2[q])):
            close(got_w, sw if r else torch.zeros_like(got_w), tw, what + "dweight")
            close(got_b, sb if r else torch.zeros_like(got_b), tb, what + "dbias")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [([3000, 0, 1, 17, 0, 0, 0, 0], 96), ([0, 2500], 2048), ([1, 900, 2], 4099), ([0, 0, 400, 1], 20000), ([700, 3], 33000),
                                       ([40] * 32, 130), ([9000, 9], 24)])
def test_layer_norm_of_uneven_workers(ctx, dtype, rows, cols):
    """Rows of one pass and of two, blocks without rows, sums of workers that have a block or two beside others that have hundreds."""
    check_norm(ctx, rows, cols, TYPES[dtype])


@pytest.mark.parametrize("what", ["norm", "norm_back", "act_back"])
@pytest.mark.parametrize("rows", [[16384, 0, 0, 0, 0, 0, 0, 0], [0, 0, 16000, 100, 100, 100, 84, 0]])
def test_sums_over_rows_take_the_time_of_their_rows_however_the_workers_share_them(rows, what):
    """One worker with all the rows once had an eighth of the chip for layer norm's backward pass, and took five times the time."""
    import time
    D, t = 4096, torch.bfloat16

    def call(rows):
        sd = binding.SlimDP(100, len(rows))
        x, dy = [device_normal(q, r, D, t) for q, r in enumerate(rows)], [device_normal(q + 9, r, D, t) for q, r in enumerate(rows)]
        w, y = [torch.ones(D, device="cuda") for _ in rows], [torch.empty_like(v) for v in x]
        mean, rstd = [torch.zeros(r, device="cuda") for r in rows], [torch.ones(r, device="cuda") for r in rows]
        a, b = [torch.empty(D, device="cuda") for _ in rows], [torch.empty(D, device="cuda") for _ in rows]
        return sd, {"norm": lambda: sd.layer_norm(x, w, w, y=y, mean=mean, rstd=rstd),
                    "norm_back": lambda: sd.layer_norm_backward(dy, x, w, mean, rstd, dx=y, dweight=a, dbias=b),
                    "act_back": lambda: sd.linear_epilogue_backward(dy, x, "gelu", dz=y, dbias=a)}[what]
    (a, uneven), (b, equal) = call(rows), call([2048] * 8)

    def once(f):
        t0 = time.perf_counter()
        for _ in range(10):
            f()
        torch.cuda.synchronize()
        return time.perf_counter() - t0
    torch.cuda.synchronize()
    once(uneven), once(equal)
    pairs = [(once(uneven), once(equal)) for _ in range(9)]
    got, want = (sorted(p[i] for p in pairs)[4] for i in (0, 1))
    assert got < 1.8 * want, (got / 10 * 1e6, want / 10 * 1e6)
    a.close(), b.close()


@pytest.mark.parametrize("rows,cols", [([30000], 40), ([140000, 3], 48), ([20000], 200), ([9000], 500), ([5000, 2600], 1000), ([6000], 1024), ([2100], 2100), ([2200, 2200], 4000),
                                       ([700], 9000), ([1200], 16000), ([300], 30000), ([600], 65536)])
def test_layer_norm_of_more_rows_than_blocks(ctx, rows, cols):
    """Blocks that take a second and a third row, the next one under way, for every number of threads to a row; more than 128 and 512 blocks'
    sums for the joining pass."""
    for t in (torch.float32, torch.bfloat16):
        check_norm(ctx, rows, cols, t)


@pytest.mark.parametrize("dtype,rows,cols", [("bf16", [30000, 10000], 2048), ("f16", [20000], 4101), ("f32", [40000], 1000), ("f32", [2500], 20000), ("bf16", [4300], 33000),
                                             ("bf16", [900000], 100)])
def test_layer_norm_of_streams_that_no_cache_holds(ctx, dtype, rows, cols):
    """More than 256 MB: the variants that pass the caches by."""
    assert sum(rows) * cols * 2 * (4 if dtype == "f32" else 2) > 256 << 20
    check_norm(ctx, rows, cols, TYPES[dtype])


def check_epilogue_backward(ctx, rows, out, t, act):
    dy = [device_normal(q, r, out, t, 0.3) for q, r in enumerate(rows)]
    z = [device_normal(q + 50, r, out, t) for q, r in enumerate(rows)]
    dz, db = ctx.linear_epilogue_backward(dy, z, act, dz=[torch.empty_like(v) for v in dy])
    ctx.synchronize()
    for q, r in enumerate(rows):
        what, total, tb = f"{t} {rows} x {out} {act} worker {q} ", torch.zeros(out, dtype=torch.float64, device="cuda"), 1e-30
        for a in range(0, r, 1 << 16):
            part = slice(a, min(r, a + (1 << 16)))
            dyd = dy[q][part].double()
            ref = dyd * act_slope(z[q][part].double(), act)
            e = dyd.abs() * 64 * F
            close(dz[q][part], ref, u(t) * ref.abs() + e + tiny(t), what + "dz")
            total, tb = total + ref.sum(0), tb + (r + 8) * F * (ref.abs() + e).sum(0) + e.sum(0)
        close(db[q], total, tb, what + "dbias")


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("dtype,rows,out", [("bf16", [200000], 48), ("f32", [70000, 5, 0], 33), ("f16", [9000, 0, 1], 300), ("f32", [0, 3000], 1001), ("bf16", [45000], 1111),
                                            ("f32", [30000], 1000), ("bf16", [1500000], 33)])
def test_epilogue_backward_of_many_and_uneven_rows(ctx, act, dtype, rows, out):
    """More than 128 and 512 slabs, slabs of one worker alone, and streams of more than 256 MB."""
    check_epilogue_backward(ctx, rows, out, TYPES[dtype], act)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V,top", [([70000, 5], 100, 7), ([66000], 130, 300)])
def test_distill_of_more_rows_than_blocks(ctx, dtype, rows, V, top):
    """A block's second row: its lists, counts and sums begin anew."""
    t, mk = TYPES[dtype], Maker(18)
    logits = [device_normal(q, r, V, t, 2.0) for q, r in enumerate(rows)]
    idx = [torch.from_numpy(mk.g.integers(0, V, (r, top)).astype(np.int32)).cuda() for r in rows]          # entries that appear twice among them
    for i, r in zip(idx, rows):
        keep = torch.from_numpy(mk.g.integers(0, top + 1, r)).cuda()
        i[torch.arange(top, device="cuda")[None] >= keep[:, None]] = -1
    val = [device_normal(q + 9, r, top, torch.float32, 2.0, 5.0) for q, r in enumerate(rows)]
    wt = [torch.from_numpy(mk.g.random(r).astype(np.float32)).cuda() for r in rows]
    wt[0][3::7] = 0.0
    loss, lse, d = ctx.distill_loss(logits, idx, val, 1.5, row_weight=wt)
    only, lse2, _ = ctx.distill_loss(logits, idx, val, 1.5, row_weight=wt, want_grad=False)
    ctx.synchronize()
    for q in range(len(rows)):
        rl, re, rd, tl, te, td = distill_reference(logits[q], idx[q], val[q], 1.5, wt[q], t)
        close(loss[q], rl, tl, f"loss {q}")
        close(only[q], rl, tl, f"loss alone {q}")
        close(lse[q], re, te, f"lse {q}")
        close(lse2[q], re, te, f"lse alone {q}")
        close(d[q], rd, td, f"dlogits {q}")


@pytest.mark.parametrize("dtype,rows,V", [("f32", 70000, 500), ("bf16", 20000, 4000), ("f16", 9000, 8000), ("f32", 4500, 8000), ("bf16", 3000, 30000), ("bf16", 1100, 65000),
                                          ("f32", 600, 65536), ("bf16", 700, 131072), ("f32", 500, 100001), ("bf16", 500, 152064)])
def test_distill_of_streams_that_no_cache_holds(ctx, dtype, rows, V):
    """More than 256 MB of logits and gradients, every number of threads to a row."""
    t, mk, top = TYPES[dtype], Maker(19), 12
    assert rows * V * 2 * (4 if dtype == "f32" else 2) > 256 << 20
    logits = device_normal(3, rows, V, t, 2.0)
    idx, val = torch.from_numpy(mk.g.integers(0, V, (rows, top)).astype(np.int32)).cuda(), device_normal(4, rows, top, torch.float32, 2.0, 5.0)
    wt = torch.ones(rows, device="cuda")
    loss, lse, d = ctx.distill_loss([logits], [idx], [val], 2.0)
    only, _, _ = ctx.distill_loss([logits], [idx], [val], 2.0, want_grad=False)
    ctx.synchronize()
    step = max(1, (1 << 26) // V)
    for a in range(0, rows, step):
        part = slice(a, min(rows, a + step))
        rl, re, rd, tl, te, td = distill_reference(logits[part], idx[part], val[part], 2.0, wt[part], t)
        close(loss[0][part], rl, tl, f"loss {a}")
        close(only[0][part], rl, tl, f"loss alone {a}")
        close(lse[0][part], re, te, f"lse {a}")
        close(d[0][part], rd, td, f"dlogits {a}")


@pytest.mark.parametrize("act,lowest", [("gelu", -12.5), ("gelu_tanh", -8.0), ("silu", -80.0)])
def test_activations_of_negative_arguments_relative_to_their_value(ctx, act, lowest):
    """Where the value is far smaller than its argument.  An exponential of an argument w that was made with n roundings is off by n F |w| of
    itself: gelu 3 of z^2 / 2, gelu_tanh 7 of u, silu 2 of z; the factor beside gelu's is off by 4e-7, and six more steps are a few
    roundings each.  Slopes are sums of two terms of different sign: the same of their sizes."""
    z = torch.linspace(lowest, -1e-3, 40001, dtype=torch.float64).float().cuda()
    zd = z.double()
    y, _ = ctx.linear([z[:, None].contiguous()], [torch.ones((1, 1), device="cuda")], None, act)
    dz, _ = ctx.linear_epilogue_backward([torch.ones_like(z)[:, None]], [z[:, None].contiguous()], act)
    ctx.synchronize()
    u_ = 2 * math.sqrt(2 / math.pi) * (zd + 0.044715 * zd ** 3)
    if act == "gelu":
        value, e = zd * 0.5 * torch.erfc(-zd / math.sqrt(2.0)), 4e-7 + F * (1.5 * zd ** 2 + 12)
        parts = (value / zd).abs() + (zd * torch.exp(-zd ** 2 / 2) / math.sqrt(2 * math.pi)).abs()
        slope = value / zd + zd * torch.exp(-zd ** 2 / 2) / math.sqrt(2 * math.pi)
    else:
        u_, factor = (u_, 2 * math.sqrt(2 / math.pi) * (1 + 0.134145 * zd ** 2)) if act == "gelu_tanh" else (zd, 1.0)
        s = torch.exp(u_) / (1 + torch.exp(u_))
        value, e = zd * s, F * ((7 if act == "gelu_tanh" else 2) * u_.abs() + 16)
        slope = s + zd * s * (1 - s) * factor
        parts = s + (zd * s * (1 - s) * factor).abs()
    close(y[0][:, 0], value, e * value.abs(), act)
    close(dz[0][:, 0], slope, (e + 16 * F) * parts, act + " slope")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,K,N", [([300, 0, 17], 264, 136), ([2100], 1032, 2312), ([40], 520, 1040), ([5, 700], 1000, 96)])
def test_bits_do_not_depend_on_addresses(ctx, dtype, rows, K, N):
    """The same values at every alignment and distance of rows: copied into the LDS or through registers, vectors whole or broken, the same order of
    every sum."""
    t, first = TYPES[dtype], None
    for pad, shift in ((0, 0), (8, 8), (3, 1), (0, 5)):
        mk = Maker(35, pad, shift)
        x, dz, w = [mk.normal(r, K, t) for r in rows], [mk.normal(r, N, t, 0.1) for r in rows], [mk.normal(N, K, t, 0.05) for _ in rows]
        b, g = [mk.vec(N) for _ in rows], [mk.vec(K) for _ in rows]
        idx, val = zip(*[teacher(mk, r, K, 9) for r in rows])
        y, z = ctx.linear(x, w, b, "gelu", keep=True)
        dx, dw = ctx.linear_backward(dz, x, w)
        da, db = ctx.linear_epilogue_backward(dz, z, "silu")
        n, mean, rstd = ctx.layer_norm(x, g, g)
        dn, dg, dc = ctx.layer_norm_backward(x, x, g, mean, rstd)
        loss, lse, dl = ctx.distill_loss(x, idx, val, 2.0)
        ctx.synchronize()
        out = [v.clone() for part in (y, z, dx, dw, da, db, n, mean, rstd, dn, dg, dc, loss, lse, dl) for v in part]
        first = first or out
        for i, (a, c) in enumerate(zip(first, out)):
            assert torch.equal(a, c), (pad, shift, i)


@pytest.mark.parametrize("K", [96, 777, 4096, 8192])
@pytest.mark.parametrize("R,N", [(64, 64), (33, 1001), (2048, 512), (4000, 16)])
def test_products_in_binary32_are_as_exact_as_short_chains(ctx, R, K, N):
    """Root mean square error of products of random signs.  A rounding's square is (half a step)^2 / 3 on average, F^2 / 3 of the value's at
    most; the k-th partial sum of a chain of n has the mean square k / n of the whole's, so a chain is off by F sqrt(n / 6) of its result.
    Chains here hold 13 steps of 32 at most; K / 256 of them and up to 48 pieces are joined by chains likewise, and one more rounding."""
    x, w = device_normal(1, R, K, torch.float32), device_normal(2, N, K, torch.float32)
    y, _ = ctx.linear([x], [w])
    dx, _ = ctx.linear_backward([x], None, [w.t().contiguous()], want_dweight=False)
    _, dw = ctx.linear_backward([x.t().contiguous()], [w.t().contiguous()], None, want_dx=False)
    ctx.synchronize()
    ref = x.double() @ w.double().t()
    size = float(ref.square().mean().sqrt())
    bound = F * math.sqrt(min(K, 416) / 6 + (K / 256 + 48) / 6 + 1)
    for what, got in (("forward", y[0]), ("dx", dx[0]), ("dweight", dw[0])):
        err = float((got.double() - ref).square().mean().sqrt()) / size
        assert err <= bound, (what, err, bound)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [[64, 65], [128, 192], [128, 129], [256, 512], [16, 17], [1, 700], [64, 64, 200], [300, 300, 300, 1000], [0, 64], [64, 0], [64, 64, 0], [0, 0, 64, 128]])
def test_workers_whose_numbers_of_tiles_begin_alike(ctx, dtype, rows):
    """The last worker has a tile more, or none: blocks are not shared out as if all had the first one's number."""
    for K, N in ((64, 48), (1024, 72)):
        check_workers(ctx, rows, K, N, TYPES[dtype])

"""dvdq_group_norm and dvdq_group_norm_backward against the formulas in 64 bits.

Tolerances.  With n = S C / G values per group, sums of d = x - pivot are fp32 over at most S / 32 + 32 steps per thread, then
trees, then fp64: relative error of mean - pivot and of the second moment below e = 2^-24 * 64, taken of the sums' magnitudes
(mean |d|, mean d^2 about the pivot).  h = (x - mean) rstd in fp32: 2^-22 |h| more.  One rounding u |y| of the output."""
import math

import pytest
import torch

from paper_2505_18663_b200 import binding as B

gpu = pytest.mark.gpu
DEV = "cuda"
DTYPES = [torch.bfloat16, torch.float16, torch.float32]
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
EPS = 1e-5
E = 64 * 2.0 ** -24

# (N, S, C, G): one place; one channel per group; groups inside a 16-byte access and across several; channel counts that
# 16 bytes do not divide; wide rows (channel blocks); one group of many channels (cut into pieces); long samples;
# sample counts that share the SMs evenly (one launch), leave SMs idle and exceed them (three launches);
# large samples whose channels go in pieces of 8, 4 and 2 bytes
SHAPES = [(1, 1, 32, 2), (2, 1, 24, 1), (1, 70, 8, 8), (3, 77, 180, 12), (2, 50, 64, 32), (1, 333, 30, 3), (2, 64, 7, 7), (1, 40, 2304, 32),
          (1, 9, 4160, 1), (2, 17, 600, 2), (1, 33, 5000, 8), (1, 20000, 128, 32), (4, 1000, 96, 4), (1, 3000, 5, 1),
          (40, 1500, 64, 4), (100, 1200, 64, 4), (200, 40, 64, 8), (1, 70, 9000, 9),
          (1, 9000, 36, 4), (2, 7000, 34, 2), (1, 5000, 35, 5), (3, 7, 2048, 1)]


def act64(z, act):
    if act == B.ACT_SILU:
        return z * torch.sigmoid(z)
    if act == B.ACT_GELU_TANH:
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def norm64(x, G, gamma, beta, act, eps=EPS):
    N, S, C = x.shape
    v = x.view(N, S, G, C // G)
    mean = v.mean((1, 3), keepdim=True)
    rstd = ((v - mean).square().mean((1, 3), keepdim=True) + eps).rsqrt()
    h = ((v - mean) * rstd).reshape(N, S, C)
    z = h * (gamma if gamma is not None else 1.0) + (beta if beta is not None else 0.0)
    return act64(z, act), mean.reshape(N, G), rstd.reshape(N, G), h, z


def make(shape, dt, seed, offset=0.5):
    N, S, C, G = shape
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = (torch.randn(N, S, C, generator=g, device=DEV) + offset * torch.randn(N, 1, C, generator=g, device=DEV) + offset).to(dt)
    gamma, beta = (1 + 0.3 * torch.randn(C, generator=g, device=DEV)), 0.3 * torch.randn(C, generator=g, device=DEV)
    return x, gamma, beta, g


def workspace(N, S, C, G):
    return torch.full((max(1, B.dvdq_group_norm_workspace_bytes(N, S, C, G)),), 255, dtype=torch.uint8, device=DEV)


def spreads(x, G):
    """mean |d| and mean d^2 about each group's pivot, the first place's first channel"""
    N, S, C = x.shape
    v = x.view(N, S, G, C // G)
    d = v - v[:, :1, :, :1]
    return d.abs().mean((1, 3)), d.square().mean((1, 3))


@gpu
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("act,params", [(0, None), (1, "own"), (2, "fp32")])
def test_forward(dt, shape, act, params):
    N, S, C, G = shape
    x, gamma, beta, _ = make(shape, dt, S + C)
    if params is None:
        gamma = beta = None
    elif params == "own":
        gamma, beta = gamma.to(dt), beta.to(dt)
    y = torch.full_like(x, float("nan"))
    mean, rstd = (torch.full((N, G), float("nan"), device=DEV) for _ in range(2))
    B.dvdq_group_norm(x, G, gamma, beta, EPS, act, y, mean, rstd, workspace(*shape))
    x6 = x.double()
    ga, be = (None if t is None else t.double() for t in (gamma, beta))
    y6, m6, r6, h6, z6 = norm64(x6, G, ga, be, act)
    a1, a2 = spreads(x6, G)
    em = E * a1 + 2.0 ** -23 * m6.abs()                          # of the mean
    ev = E * (a2 + a1 * a1) * 2                                   # of the variance
    er = 0.5 * ev * r6 ** 3 * 1.5 + 2.0 ** -23 * r6               # of rstd
    assert ((mean - m6).abs() <= em).all()
    assert ((rstd - r6).abs() <= er).all()
    wide = lambda t: t[:, None, :, None].expand(N, S, G, C // G).reshape(N, S, C)  # noqa: E731
    eh = wide(em * r6) + h6.abs() * wide(er / r6) + 2.0 ** -21 * (h6.abs() + wide(m6.abs() * r6))
    g_abs = ga.abs() if ga is not None else 1.0
    inner = 1.13 * (eh * g_abs + 2.0 ** -22 * z6.abs()) + (2.0 ** -18 * z6.abs() if act else 0.0)
    bound = inner + U[dt] * (y6.abs() + inner) + (2.0 ** -25 if dt == torch.float16 else 0)
    assert ((y.double() - y6).abs() <= bound).all(), float(((y.double() - y6).abs() - bound).max())
    y2 = x.clone()                                                # in place, without statistics: the same bits
    B.dvdq_group_norm(y2, G, gamma, beta, EPS, act, y2, None, None, workspace(*shape))
    assert torch.equal(y2, y)


@gpu
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("shape", [s for s in SHAPES if s[1] * s[2] // s[3] >= 16])
@pytest.mark.parametrize("act,params", [(0, None), (1, "own"), (2, "fp32")])
def test_backward(dt, shape, act, params):
    N, S, C, G = shape
    x, gamma, beta, g = make(shape, dt, 2 * S + C)
    if params is None:
        gamma = beta = None
    elif params == "own":
        gamma, beta = gamma.to(dt), beta.to(dt)
    dy = torch.randn(N, S, C, generator=g, device=DEV).to(dt)
    x6, dy6 = x.double(), dy.double()
    ga = gamma.double() if gamma is not None else torch.ones(C, dtype=torch.float64, device=DEV)
    be = beta.double() if beta is not None else torch.zeros(C, dtype=torch.float64, device=DEV)
    _, m6, r6, _, _ = norm64(x6, G, ga, be, act)
    mean, rstd = m6.float(), r6.float()
    dx = torch.full_like(x, float("nan"))
    dgamma, dbeta = (torch.full((C,), float("nan"), device=DEV) for _ in range(2))
    ws = workspace(*shape)
    B.dvdq_group_norm_backward(dy, x, mean, rstd, G, gamma, beta, act, dx, dgamma, dbeta, ws)
    wide = lambda t: t[:, None, :, None].expand(N, S, G, C // G).reshape(N, S, C)  # noqa: E731
    r = wide(rstd.double())
    h = (x6 - wide(mean.double())) * r                             # the statistics that were given
    eh = 2.0 ** -22 * (h.abs() + wide(mean.double().abs()) * r)
    z = (h * ga + be).requires_grad_(True)
    act64(z, act).sum().backward()
    slope, z = z.grad, z.detach()
    dz = dy6 * slope
    # the slope's own slope is at most 1.2; ex2 / rcp: 2^-18 (1 + |z|)
    ez = dy6.abs() * ((1.2 * (eh * ga.abs() + 2.0 ** -22 * z.abs()) + 2.0 ** -18 * (1 + z.abs())) if act else 0.0) + 2.0 ** -23 * dz.abs()
    assert (dbeta - dz.sum((0, 1))).abs().le(ez.sum((0, 1)) + E * dz.abs().sum((0, 1))).all()
    ezh = ez * h.abs() + dz.abs() * eh
    assert (dgamma - (dz * h).sum((0, 1))).abs().le(ezh.sum((0, 1)) + E * (dz * h).abs().sum((0, 1))).all()
    group = lambda t: wide(t.view(N, S, G, C // G).mean((1, 3)))   # noqa: E731
    dh, edh = dz * ga, (ez + 2.0 ** -23 * dz.abs()) * ga.abs()
    m1, m2 = group(dh), group(dh * h)
    e1 = group(edh) + 2 * E * group(dh.abs())
    e2 = group(ezh * ga.abs()) + 2 * E * group((dh * h).abs())
    want = r * (dh - m1 - h * m2)
    inner = r * (edh + e1 + h.abs() * e2 + eh * m2.abs() + 2.0 ** -22 * (dh.abs() + m1.abs() + (h * m2).abs()))
    bound = inner + U[dt] * (want.abs() + inner) + (2.0 ** -25 if dt == torch.float16 else 0)
    assert ((dx.double() - want).abs() <= bound).all(), float(((dx.double() - want).abs() - bound).max())
    # each alone, and dx over dy: the same bits
    d2 = dy.clone()
    B.dvdq_group_norm_backward(d2, x, mean, rstd, G, gamma, beta, act, d2, None, None, ws)
    g2, b2 = torch.empty_like(dgamma), torch.empty_like(dbeta)
    B.dvdq_group_norm_backward(dy, x, mean, rstd, G, gamma, beta, act, None, g2, None, ws)
    B.dvdq_group_norm_backward(dy, x, mean, rstd, G, gamma, beta, act, None, None, b2, ws)
    assert torch.equal(d2, dx) and torch.equal(g2, dgamma) and torch.equal(b2, dbeta)


@gpu
def test_gradient_against_differences():
    """fp32; f = sum(c y).  Central differences along sign(dx) with step 1/64: the third-order term is below 1 % of the
    first for h of order one and steps of 2^-6 (relative (2^-6)^2 times a third derivative of order 10)."""
    shape = N, S, C, G = 2, 19, 24, 3
    x, gamma, beta, g = make(shape, torch.float32, 9)
    c = torch.randn(N, S, C, generator=g, device=DEV)
    y, mean, rstd, ws = torch.empty_like(x), torch.empty(N, G, device=DEV), torch.empty(N, G, device=DEV), workspace(*shape)

    def f(xx, ga):
        B.dvdq_group_norm(xx, G, ga, beta, EPS, B.ACT_SILU, y, mean, rstd, ws)
        return float((y.double() * c.double()).sum())

    f(x, gamma)
    dx, dgamma = torch.empty_like(x), torch.empty(C, device=DEV)
    B.dvdq_group_norm_backward(c, x, mean.clone(), rstd.clone(), G, gamma, beta, B.ACT_SILU, dx, dgamma, None, ws)
    for t, grad in ((x, dx), (gamma, dgamma)):
        d = torch.sign(grad) * 2.0 ** -6
        diff = f(x + d, gamma) - f(x - d, gamma) if t is x else f(x, gamma + d) - f(x, gamma - d)
        want = 2 * float((grad.double() * d.double()).sum())
        assert abs(diff - want) <= 0.02 * abs(want), (diff, want)


@gpu
@pytest.mark.parametrize("C,pad", [(64, 8), (64, 3), (30, 0)])
def test_pitches(C, pad):
    """Places further apart than their channels, samples further apart than their places; nothing between is written."""
    N, S, G, dt = 2, 37, 2, torch.bfloat16
    x, gamma, beta, _ = make((N, S, C, G), dt, 10)
    big = torch.full((N, S + 2, C + pad), float("nan"), dtype=dt, device=DEV)
    xv = big[:, :S, :C]
    xv.copy_(x)
    out = torch.full_like(big, float("nan"))
    yv, y = out[:, 1:S + 1, pad:], torch.empty_like(x)
    B.dvdq_group_norm(xv, G, gamma, beta, EPS, 2, yv, None, None, workspace(N, S, C, G))
    B.dvdq_group_norm(x, G, gamma, beta, EPS, 2, y, None, None, workspace(N, S, C, G))
    # other accesses, other order of the sums: equal up to one rounding of the output
    assert ((yv.double() - y.double()).abs() <= 2.0 ** -7 * y.double().abs() + 1e-5).all()
    assert out[:, 0].isnan().all() and out[:, S + 1].isnan().all() and (pad == 0 or out[:, :, :pad].isnan().all())


@gpu
def test_a_mean_far_from_zero_costs_no_digits():
    x = (1000.0 + torch.randn(1, 5000, 16, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1)))
    y, ws = torch.empty_like(x), workspace(1, 5000, 16, 2)
    B.dvdq_group_norm(x, 2, None, None, 0.0, 0, y, None, None, ws)
    want, _, _, _, _ = norm64(x.double(), 2, None, None, 0, eps=0.0)
    # the mean itself is an fp32 number: 2^-24 * 1000 = 6e-5 of a value's size
    assert (y.double() - want).abs().max() <= 1.2e-4


@gpu
def test_a_constant_group_gives_beta():
    x = torch.full((1, 50, 8), 3.0, device=DEV)
    beta, y, ws = torch.arange(8.0, device=DEV), torch.empty_like(x), workspace(1, 50, 8, 2)
    B.dvdq_group_norm(x, 2, None, beta, EPS, 0, y, None, None, ws)
    assert torch.equal(y, beta.expand_as(x))


@gpu
def test_nan_and_infinity_stay_in_their_group():
    x = torch.randn(2, 40, 16, device=DEV)
    x[0, 3, 1], x[1, 7, 9] = float("nan"), float("inf")
    y = torch.empty_like(x)
    B.dvdq_group_norm(x, 4, None, None, EPS, 0, y, None, None, workspace(2, 40, 16, 4))
    bad = torch.zeros(2, 40, 16, dtype=torch.bool, device=DEV)
    bad[0, :, 0:4] = True
    bad[1, :, 8:12] = True
    assert y[~bad].isfinite().all() and y[0, :, 0:4].isnan().all() and not y[1, :, 8:12].isfinite().all()


@gpu
def test_empty_samples():
    e = torch.empty(2, 0, 8, device=DEV)
    mean, rstd = torch.ones(2, 2, device=DEV), torch.ones(2, 2, device=DEV)
    B.dvdq_group_norm(e, 2, None, None, 4.0, 0, e, mean, rstd, None)
    assert (mean == 0).all() and (rstd == 0.5).all()
    dg, db = torch.ones(8, device=DEV), torch.ones(8, device=DEV)
    B.dvdq_group_norm_backward(e, e, mean, rstd, 2, None, None, 0, None, dg, db, None)
    assert (dg == 0).all() and (db == 0).all()
    z = torch.empty(0, 5, 8, device=DEV)
    B.dvdq_group_norm(z, 2, None, None, EPS, 0, z, None, None, None)


# ------------------------------------------------------------------ refusals (no GPU needed)

P = 4096


def forward(**k):
    a = dict(X=P, xn=320, xs=32, N=2, S=10, C=32, G=4, gamma=P, beta=P, pt=2, eps=1e-5, act=2, Y=P, yn=320, ys=32, mean=None, rstd=None, dtype=0,
             ws=P, n=1 << 20, stream=None)
    a.update(k)
    return B.load().dvdq_group_norm(*a.values())


def backward(**k):
    a = dict(dY=P, dn=320, ds=32, X=P, xn=320, xs=32, mean=P, rstd=P, N=2, S=10, C=32, G=4, gamma=P, beta=P, pt=2, act=2, dX=P, en=320, es=32,
             dg=P, db=P, dtype=0, ws=P, n=1 << 20, stream=None)
    a.update(k)
    return B.load().dvdq_group_norm_backward(*a.values())


@pytest.mark.parametrize("change,status", [
    (dict(N=-1), B.ERR_SHAPE), (dict(N=65536), B.ERR_SHAPE), (dict(S=-1), B.ERR_SHAPE), (dict(C=0), B.ERR_SHAPE), (dict(G=0), B.ERR_SHAPE),
    (dict(G=5), B.ERR_SHAPE), (dict(eps=-1.0), B.ERR_SHAPE), (dict(eps=float("nan")), B.ERR_SHAPE), (dict(act=3), B.ERR_UNSUPPORTED),
    (dict(dtype=3), B.ERR_UNSUPPORTED), (dict(pt=1), B.ERR_UNSUPPORTED), (dict(dtype=2, pt=0), B.ERR_UNSUPPORTED), (dict(X=None), B.ERR_NULL),
    (dict(Y=None), B.ERR_NULL), (dict(ws=None), B.ERR_NULL), (dict(n=10), B.ERR_WORKSPACE), (dict(ws=P + 8), B.ERR_ALIGN),
    (dict(X=P + 1), B.ERR_ALIGN), (dict(gamma=P + 2), B.ERR_ALIGN), (dict(mean=P + 2), B.ERR_ALIGN), (dict(ys=31), B.ERR_SHAPE),
    (dict(xs=-32), B.ERR_SHAPE), (dict(yn=0), B.ERR_SHAPE), (dict(xs=40, xn=400), B.ERR_SHAPE), (dict(xn=640), B.ERR_SHAPE), (dict(N=0), B.OK), (dict(S=0), B.OK)])
def test_forward_refuses(change, status):
    assert forward(**change) == status


@pytest.mark.parametrize("change,status", [
    (dict(G=3), B.ERR_SHAPE), (dict(act=-1), B.ERR_UNSUPPORTED), (dict(dY=None), B.ERR_NULL), (dict(X=None), B.ERR_NULL),
    (dict(mean=None), B.ERR_NULL), (dict(rstd=None), B.ERR_NULL), (dict(ws=None), B.ERR_NULL), (dict(n=10), B.ERR_WORKSPACE),
    (dict(es=16), B.ERR_SHAPE), (dict(en=640), B.ERR_SHAPE), (dict(dY=2 * P, es=40, en=400), B.ERR_SHAPE), (dict(dX=P + 1), B.ERR_ALIGN), (dict(dg=P + 2), B.ERR_ALIGN), (dict(N=0, dg=None, db=None), B.OK)])
def test_backward_refuses(change, status):
    assert backward(**change) == status


def test_workspace_sizes():
    assert B.dvdq_group_norm_workspace_bytes(0, 10, 8, 2) == 0 and B.dvdq_group_norm_workspace_bytes(1, 10, 8, 3) == 0
    assert B.dvdq_group_norm_workspace_bytes(1, 10, 8, 2) > 0
    assert B.dvdq_group_norm_workspace_bytes(1, 499200, 128, 32) < 8 << 20


@gpu
@pytest.mark.parametrize("shape", [(1, 162285, 8, 4), (2, 60000, 12, 4), (1, 3000, 8, 1), (1, 40000, 3, 1)])
def test_small_squares_are_not_lost_in_long_sums(shape):
    """bf16 values near the mean have squares below half a unit of a sum of some hundred terms, and they are the many: a
    plain running fp32 sum of 1000 squares is 7e-6 low.  Sums of at most 16 terms, then pairwise, stay within 16 + 10
    roundings of 2^-24 that partly cancel: 1e-6 for the variance, half of that for rstd."""
    N, S, C, G = shape
    x = (0.4 + torch.randn(N, S, C, device=DEV, generator=torch.Generator(device=DEV).manual_seed(7))).bfloat16()
    y, mean, rstd = torch.empty_like(x), torch.empty(N, G, device=DEV), torch.empty(N, G, device=DEV)
    B.dvdq_group_norm(x, G, None, None, EPS, 0, y, mean, rstd, workspace(*shape))
    _, m6, r6, _, _ = norm64(x.double(), G, None, None, 0)
    assert ((rstd - r6) / r6).abs().max() <= 5e-7
    assert (mean - m6).abs().max() <= 2.0 ** -23


# ------------------------------------------------------------------ values that are far out

# one launch in shared memory; gradients in one launch over all SMs (forward three: the tensor is small); three launches (80 samples leave SMs idle)
PATHS = {"small": (2, 40), "one": (1, 20000), "three": (80, 3000)}


def run_forward(x, G, gamma, beta, act, eps=EPS):
    N, S, C = x.shape
    y, mean, rstd = torch.full_like(x, float("nan")), torch.empty(N, G, device=DEV), torch.empty(N, G, device=DEV)
    B.dvdq_group_norm(x, G, gamma, beta, eps, act, y, mean, rstd, workspace(N, S, C, G))
    return y, mean, rstd


def run_backward(dy, x, mean, rstd, G, gamma, beta, act):
    N, S, C = x.shape
    dx, dg, db = torch.full_like(x, float("nan")), torch.empty(C, device=DEV), torch.empty(C, device=DEV)
    B.dvdq_group_norm_backward(dy, x, mean, rstd, G, gamma, beta, act, dx, dg, db, workspace(N, S, C, G))
    return dx, dg, db


@gpu
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("shape", [(1, 162285, 8, 4), (1, 20000, 128, 32), (4, 1000, 96, 4), (80, 3000, 64, 4), (1, 40000, 35, 5), (2, 64, 64, 4),
                                   (1, 30000, 36, 4), (1, 9000, 34, 2), (1, 70, 9000, 9), (1, 30000, 1, 1)])
@pytest.mark.parametrize("first", [-50.0, -1000.0, -10000.0, 0.0])
def test_an_outlying_first_value_costs_no_digits(dt, shape, first):
    """Whatever the first value of each group is (far from the rest, or 0 where the rest is near 300), the variance keeps the accuracy
    of its own size, not of the spread about that value.  Per thread: short sums of 16 squares, 8 channels brought to one centre,
    each of at most twice the squares about the mean, 2^-24 a rounding: 2 (16 + 8) 2^-24 = 2.9e-6 if none cancelled, half of
    that for rstd; most do: 1e-6.  The mean: the same roundings of at most the deviations' sizes."""
    N, S, C, G = shape
    g = torch.Generator(device=DEV).manual_seed(S)
    x = (0.3 + torch.randn(N, S, C, generator=g, device=DEV)).to(dt)
    if first == 0.0:
        x = (x.float() + 300.0).to(dt)
    x[:, 0, ::C // G] = first
    _, mean, rstd = run_forward(x, G, None, None, 0)
    _, m6, r6, _, _ = norm64(x.double(), G, None, None, 0)
    assert ((rstd - r6) / r6).abs().max() <= 1e-6
    assert (((mean - m6).abs() - 2.0 ** -24 * m6.abs()) * r6).max() <= 1e-6   # 2^-24: its own rounding


@gpu
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("C,G", [(24, 8), (16, 16), (40, 8), (64, 16)])
@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_not_finite_stays_in_its_group(dt, path, C, G, act, bad):
    (N, S), per = PATHS[path], C // G
    g = torch.Generator(device=DEV).manual_seed(C)
    x, dy = torch.randn(N, S, C, generator=g, device=DEV).to(dt), torch.randn(N, S, C, generator=g, device=DEV).to(dt)
    gamma, beta = 1 + 0.3 * torch.randn(C, generator=g, device=DEV), 0.3 * torch.randn(C, generator=g, device=DEV)
    clean = run_forward(x, G, gamma, beta, act)
    clean_back = run_backward(dy, x, clean[1], clean[2], G, gamma, beta, act)
    xb = x.clone()
    xb[:, S // 2, 2 * per - 1] = bad
    y, mean, rstd = run_forward(xb, G, gamma, beta, act)
    dx, dg, db = run_backward(dy, xb, mean, rstd, G, gamma, beta, act)
    rest = [c for c in range(C) if c // per != 1]
    inside = [c for c in range(C) if c // per == 1]
    assert y[..., inside].isnan().all() and dx[..., inside].isnan().all()
    # what shares an access with a value that is not a number has its logistic function formed in another way: both runs are
    # within 2^-18 (1 + |z|) of the slope (1.2 at most times as much), of 2^-18 |z| of the value
    groups = lambda t: t.view(N, S, G, per).mean((1, 3), keepdim=True).expand(N, S, G, per).reshape(N, S, C)  # noqa: E731
    r = clean[2].double().repeat_interleave(per, 1)[:, None]
    h = (x.double() - clean[1].double().repeat_interleave(per, 1)[:, None]) * r
    z, g6 = h * gamma.double() + beta.double(), gamma.double().abs()
    ez = 2 * 2.0 ** -18 * 1.2 * dy.double().abs() * (1 + z.abs()) if act else torch.zeros_like(z)
    dz, h = 1.2 * dy.double().abs(), h.abs()
    rx = r * (ez * g6 + groups(ez * g6) + h * groups(ez * g6 * h) + 2.0 ** -20 * (dz * g6 + groups(dz * g6) + h * groups(dz * g6 * h)))
    for got, want, rough, u in ((y, clean[0], 2 * 2.0 ** -18 * z.abs(), U[dt]), (dx, clean_back[0], rx, U[dt]),
                                (dg, clean_back[1], (ez * h + E * dz * h).sum((0, 1)), 0.0), (db, clean_back[2], (ez + E * dz).sum((0, 1)), 0.0)):
        got, want, rough = got[..., rest].double(), want[..., rest].double(), rough[..., rest]
        assert ((got - want).abs() <= rough + 2 * u * (want.abs() + rough) + (2.0 ** -24 if dt == torch.float16 else 0.0)).all()


@gpu
@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("act", [1, 2])
def test_a_parameter_that_is_not_a_number_stays_in_its_channel(path, act):
    (N, S), C, G, dt = PATHS[path], 32, 4, torch.bfloat16
    g = torch.Generator(device=DEV).manual_seed(C)
    x = torch.randn(N, S, C, generator=g, device=DEV).to(dt)
    gamma, beta = 1 + 0.3 * torch.randn(C, generator=g, device=DEV), 0.3 * torch.randn(C, generator=g, device=DEV)
    clean, _, _ = run_forward(x, G, gamma, beta, act)
    gamma[9], beta[20] = float("nan"), float("nan")
    y, _, _ = run_forward(x, G, gamma, beta, act)
    rest = [c for c in range(C) if c not in (9, 20)]
    got, want = y[..., rest].double(), clean[..., rest].double()
    assert y[..., [9, 20]].isnan().all() and ((got - want).abs() <= 2 * U[dt] * want.abs() + 2.0 ** -18).all()


@gpu
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("act", [1, 2])
def test_activations_of_the_lowest_values(dt, path, act):
    """A channel whose beta is the lowest value (a mask) is 0 after the activation, and its slope is 0; z = -inf gives NaN, as
    z / (1 + exp(-z)) does.  2e-5: 2^-18 of |z| < 5, twice for the statistics' roundings in z."""
    (N, S), C, G = PATHS[path], 32, 2
    x = torch.randn(N, S, C, device=DEV, generator=torch.Generator(device=DEV).manual_seed(3)).to(dt)
    lowest = torch.finfo(torch.float32).min
    beta = torch.zeros(C, device=DEV)
    special = torch.tensor([-45.0, -60.0, -100.0, -1e4, -1e20, lowest, 1e20 if dt != torch.float16 else 6e4, float("-inf")], device=DEV)
    beta[5:13] = special
    beta[20] = -1e20
    y, mean, rstd = run_forward(x, G, None, beta, act)
    y6, _, _, _, _ = norm64(x.double(), G, None, beta.double(), act)
    assert torch.equal(y.isnan(), y6.isnan())
    ok = ~y6.isnan()
    assert ((y.double() - y6)[ok].abs() <= (U[dt] + 2.0 ** -18) * 2 * y6[ok].abs() + 2e-5).all()
    beta[12] = 0.0
    dy = torch.randn(N, S, C, device=DEV).to(dt)
    dx, dg, db = run_backward(dy, x, mean, rstd, G, None, beta, act)
    assert dx.isfinite().all()
    far = [6, 7, 8, 9, 10, 20]    # slopes below 1e-24: nothing reaches the parameters' gradients
    assert (dg[far].abs() <= 1e-15).all() and (db[far].abs() <= 1e-15).all()


@gpu
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("C,G", [(32, 4), (35, 5)])
def test_a_constant_group_far_from_zero_gives_beta(dt, path, C, G):
    """x - mean is 0, whatever 1000 / sqrt(eps) rounds to: y is beta itself, and h is 0 in the gradients."""
    N, S = PATHS[path]
    x = torch.full((N, S, C), 1000.0, device=DEV).to(dt)
    beta = (torch.arange(C, device=DEV) / 8.0).to(dt)
    y, mean, rstd = run_forward(x, G, None, beta, 0, eps=EPS)
    assert torch.equal(y, beta.expand_as(x))
    dy = torch.ones_like(x)
    _, dg, db = run_backward(dy, x, mean, rstd, G, None, beta, 0)
    assert (dg == 0).all() and (db == N * S).all()


@gpu
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("shape", [(1, 30000, 1, 1), (1, 16000, 2, 1), (1, 100, 128, 16), (1, 700, 1024, 4), (80, 3000, 64, 4)])
def test_an_outlier_in_few_pieces(dt, shape):
    """-60000 at the first place, where a thread has a piece or two, or one channel's sums are long: no channel's square counts for its
    neighbours too, and the mean is as good as the variance.  Bounds as above."""
    N, S, C, G = shape
    x = (0.3 + torch.randn(N, S, C, generator=torch.Generator(device=DEV).manual_seed(S), device=DEV)).to(dt)
    x[:, 0, ::C // G] = -60000.0
    _, mean, rstd = run_forward(x, G, None, None, 0)
    _, m6, r6, _, _ = norm64(x.double(), G, None, None, 0)
    assert ((rstd - r6) / r6).abs().max() <= 1e-6
    assert (((mean - m6).abs() - 2.0 ** -24 * m6.abs()) * r6).max() <= 1e-6


@gpu
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("C,G", [(128, 32), (56, 8), (64, 64)])
@pytest.mark.parametrize("act", [1, 2])
def test_large_tensors_in_one_launch(dt, C, G, act):
    """70 MB of whole 16-byte pieces, groups of 4, 7 and 1 channels (an odd number goes through the sums in two rounds), each of the far
    values in a group of its own: an outlier first, a masked channel, equal values, NaN.
    h is off by the statistics' 1e-6 and its own roundings, 2^-22 (|h| + |mean| rstd); the activation by 2^-18 |z|."""
    S, per = 70_000_000 // (C * torch.empty(0, dtype=dt).element_size()), C // G
    g = torch.Generator(device=DEV).manual_seed(C)
    x = (0.3 + torch.randn(1, S, C, generator=g, device=DEV)).to(dt)
    gamma, beta = 1 + 0.3 * torch.randn(C, generator=g, device=DEV), 0.3 * torch.randn(C, generator=g, device=DEV)
    x[:, 0, 0] = -10000.0
    beta[per] = -1e20
    x[..., 2 * per:3 * per] = 1000.0
    x[:, S // 2, 4 * per - 1] = float("nan")
    y, mean, rstd = run_forward(x, G, gamma, beta, act)
    y6, m6, r6, h6, z6 = norm64(x.double(), G, gamma.double(), beta.double(), act)
    assert y[..., 3 * per:4 * per].isnan().all() and mean[:, 3].isnan().all() and rstd[:, 3].isnan().all()
    keep, groups = [c for c in range(C) if c // per != 3], [k for k in range(G) if k != 3]
    assert ((rstd - r6) / r6)[:, groups].abs().max() <= 1e-6
    assert (((mean - m6).abs() - 2.0 ** -24 * m6.abs()) * r6)[:, groups].max() <= 1e-6
    h6, z6, y6, y = h6[..., keep].abs(), z6[..., keep].abs(), y6[..., keep], y[..., keep].double()
    far = (m6.abs() * r6).repeat_interleave(per, 1)[0, keep] * (h6.amax((0, 1)) > 0)   # equal values leave no rounding
    inner = 1.2 * gamma.double().abs()[keep] * ((1e-6 + 2.0 ** -22) * (1 + h6) + 2.0 ** -22 * far) + 2.0 ** -18 * z6 * (z6 < 1e10)
    assert ((y - y6).abs() <= inner + U[dt] * (y6.abs() + inner) + 2.0 ** -24).all()

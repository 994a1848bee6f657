"""dvdq_rms_norm, its gradients and dvdq_quantize_rows against the formulas in 64 bits.

Tolerances, element by element, with u the unit roundoff of the type (2^-8 bf16, 2^-11 fp16, 2^-24 fp32) and e = 2^-24:
  a sum over a row passes through at most ADDS additions (a thread's own, the shuffles, the warps): ADDS e of the sum of magnitudes
  y: half of that from the mean square, a square root, a division and three products: (ADDS / 2 + 6) e |y|, and u |y| for the output
  scales: the same as y's, and a division; codes: within half a step of y / s, and 127 times the relative error of both
  dx: ADDS e of |q hh| mean |dh hh|, 8 e of each term's magnitude, u |dx|
  dgamma: a CTA adds up its rows one after another: (rows / 100 + 40) e of the sum of magnitudes
"""
import math

import pytest
import torch

from paper_2505_18663_b200 import binding as B

gpu = pytest.mark.gpu
DEV = "cuda"
DTYPES = [torch.bfloat16, torch.float16, torch.float32]
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}   # half the smallest number
E = 2.0 ** -24


def adds(C):
    return 80 if C <= 8192 else 80 + C // 1024


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def check(got, want, bound, what):
    got = got.double()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = ((got - want).abs() - bound).max()
    assert float(over) <= 0, f"{what}: {float((got - want).abs().max()):.3e} off, {float(over):.3e} over the bound"


def status_ok():
    assert B.dvdq_last_device_status()[0] == B.OK


def place(shape, dt, layout, fill=None):
    """An [N, S, C] tensor whose surroundings are NaN (int8: 99): dense, rows padded to 16 bytes, heads of a fused projection, an odd
    start, samples behind one another along the rows."""
    N, S, C = shape
    bad = 99 if dt == torch.int8 else float("nan")
    if layout == "dense":
        t = torch.full(shape, bad, dtype=dt, device=DEV)
    elif layout == "padded":
        t = torch.full((N, S, -(-C // 16) * 16 + 16), bad, dtype=dt, device=DEV)[..., :C]
    elif layout == "heads":
        t = torch.full((N, 3 * S, C), bad, dtype=dt, device=DEV)[:, S:2 * S]
    elif layout == "odd":
        t = torch.full((N * S * C + 1,), bad, dtype=dt, device=DEV)[1:].view(shape)
    else:
        t = torch.full((S, N, C), bad, dtype=dt, device=DEV).transpose(0, 1)
    if fill is not None:
        t.copy_(fill)
    return t


# rows that share a warp (one channel up), a warp's rows, a CTA's; few and many rows; sizes that no piece divides; rows read twice
SHAPES = [(1, 1, 1), (1, 3, 5), (3, 7, 8), (2, 50, 64), (37, 12, 128), (1, 7, 1536), (5, 3, 1541), (1, 1400, 1536), (1, 1300, 2049), (1, 20, 4100),
          (1, 700, 5120), (2, 9, 9001), (1, 400, 16384), (1, 4, 40000)]


def reference(x, r, gamma, eps):
    h = x.double() if r is None else x.double() + r.double()
    q = (h.square().mean(-1, keepdim=True) + eps).rsqrt()
    y = h * q if gamma is None else h * q * gamma.double()
    return h, q, y


@gpu
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("shape", SHAPES + [(700, 5, 96), (1, 700, 768), (3, 411, 1200), (1, 1300, 2048), (2, 300, 2560), (1, 300, 8960), (1, 200, 12288)])
@pytest.mark.parametrize("layout,residual,params,outs", [("dense", True, "own", "hycr"), ("heads", False, "fp32", "y"), ("padded", True, "own", "hc"),
                                                         ("odd", False, None, "yc"), ("turned", True, "fp32", "hyr")])
def test_forward(dt, shape, layout, residual, params, outs):
    N, S, C = shape
    g = gen(N * 7 + S * 3 + C)
    x = place(shape, dt, layout, torch.randn(shape, device=DEV, generator=g) * 3)
    r = place(shape, dt, "dense" if layout == "turned" else layout, torch.randn(shape, device=DEV, generator=g)) if residual else None
    gamma = None if params is None else (1 + torch.randn(C, device=DEV, generator=g)).to(dt if params == "own" else torch.float32)
    h = place(shape, dt, layout) if "h" in outs else None
    y = place(shape, dt, layout) if "y" in outs else None
    c = place(shape, torch.int8, "padded" if layout == "dense" else layout) if "c" in outs else None
    s = torch.full((N, S), float("nan"), device=DEV) if "c" in outs else None
    rstd = torch.full((N, S), float("nan"), device=DEV) if "r" in outs else None
    B.dvdq_rms_norm(x, r, gamma, 1e-5, h, y, c, s, rstd)
    status_ok()
    h6, q6, y6 = reference(x, r, gamma, 1e-5)
    rel = (adds(C) / 2 + 6) * E
    if h is not None:
        check(h, h6, (U[dt] + 2 * E) * h6.abs() + TINY[dt], "h")
    if y is not None:
        check(y, y6, (U[dt] + rel * 1.01) * y6.abs() + TINY[dt], "y")
    if rstd is not None:
        check(rstd, q6[..., 0], rel * q6[..., 0], "rstd")
    if c is not None:
        check_codes(c, s, y6, rel)
    for t in (h, y, c):  # what lies between the rows stays as it was
        if t is not None and layout == "heads":
            around = torch.as_strided(t, (N, 3 * S, C), (3 * S * C, C, 1), t.storage_offset() - S * C)
            assert (around[:, :S].isnan() if t.dtype != torch.int8 else around[:, :S] == 99).all()
            assert (around[:, 2 * S:].isnan() if t.dtype != torch.int8 else around[:, 2 * S:] == 99).all()


def check_codes(c, s, y6, rel):
    top = y6.abs().amax(-1, keepdim=True)
    check(s, (top / 127)[..., 0], (rel + 4 * E) * (top / 127)[..., 0] + 2.0 ** -149, "scales")
    steps = torch.where(top > 0, y6 * 127 / torch.where(top > 0, top, 1.0), 0.0)
    assert (c.double() - steps).abs().max() <= 0.5 + 127 * (2 * rel + 8 * E)
    assert (c.abs().amax(-1)[top[..., 0] > 0] == 127).all()   # the row's largest value


@gpu
@pytest.mark.parametrize("dt", DTYPES)
def test_in_place(dt):
    g = gen(2)
    shape = (2, 33, 520)
    x0, r0 = (torch.randn(shape, device=DEV, generator=g).to(dt) for _ in range(2))
    want_h, want_y = torch.empty_like(x0), torch.empty_like(x0)
    B.dvdq_rms_norm(x0, r0, None, 1e-6, want_h, want_y)
    for swap in (False, True):
        x, r = x0.clone(), r0.clone()
        h, y = (r, x) if swap else (x, r)
        B.dvdq_rms_norm(x, r, None, 1e-6, h, y)
        assert torch.equal(h, want_h) and torch.equal(y, want_y)
    x = x0.clone()
    B.dvdq_rms_norm(x, None, None, 1e-6, None, x)
    B.dvdq_rms_norm(x0, None, None, 1e-6, None, want_y)
    assert torch.equal(x, want_y)
    # long rows, which are read again
    x0 = torch.randn(2, 50000, device=DEV, generator=g).to(dt)
    want = torch.empty_like(x0)
    B.dvdq_rms_norm(x0, None, None, 1e-6, None, want)
    B.dvdq_rms_norm(x0, None, None, 1e-6, None, x0)
    assert torch.equal(x0, want)


@gpu
@pytest.mark.parametrize("C", [40000, 40008, 33333])
@pytest.mark.parametrize("over", ["x", "r"])
def test_long_rows_whose_sum_is_kept_in_place(C, over):
    """Rows that are read again for y and codes, after h has gone over x or r."""
    g = gen(8)
    x, r = (torch.randn(3, C, device=DEV, generator=g).bfloat16() for _ in range(2))
    want = [torch.empty_like(x), torch.empty_like(x), torch.empty(3, C, dtype=torch.int8, device=DEV), torch.empty(3, device=DEV)]
    B.dvdq_rms_norm(x, r, None, 1e-6, *want)
    got = [x if over == "x" else r, torch.empty_like(x), torch.empty(3, C, dtype=torch.int8, device=DEV), torch.empty(3, device=DEV)]
    B.dvdq_rms_norm(x, r, None, 1e-6, *got)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@gpu
@pytest.mark.parametrize("C", [12, 300, 4100, 50000])
@pytest.mark.parametrize("dt,scale,eps", [(torch.float32, 1e25, 1e-6), (torch.float32, 3e38, 0.0), (torch.float32, 1e-30, 0.0), (torch.float32, 1e-30, 1e-6),
                                          (torch.float32, 1e-41, 0.0), (torch.bfloat16, 1e30, 1e-6), (torch.bfloat16, 1e-30, 0.0),
                                          (torch.float16, 6e4, 1e-6), (torch.float32, 1e-20, 1e-38), (torch.float32, 1e-24, 1e-35)])
def test_far_from_one(dt, scale, eps, C):
    """Rows whose squares leave fp32, among rows that stay: y has the size of gamma whatever the row's.  (Values below 2^-126 hold fewer digits: their spacing is
    2^-149, and no more is asked of y than that of the inputs.)"""
    g = gen(3)
    x = torch.rand(9, C, device=DEV, generator=g) * 2 - 1
    x[::2] *= scale
    x = x.to(dt)
    y, c, s, q = torch.empty_like(x), torch.empty(x.shape, dtype=torch.int8, device=DEV), torch.empty(9, device=DEV), torch.empty(9, device=DEV)
    eps = float(torch.tensor(eps, dtype=torch.float32))
    B.dvdq_rms_norm(x, None, None, eps, None, y, c, s, q)
    h6, q6, y6 = reference(x, None, None, eps)
    rel = (adds(C) / 2 + 8) * E
    check(y, y6, (U[dt] + rel) * y6.abs() + TINY[dt], "y")
    check_codes(c, s, y6, rel)
    fine = q6[:, 0] < 3e38
    check(q[fine], q6[fine, 0], rel * q6[fine, 0] + 2.0 ** -149, "rstd")


@gpu
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("C", [40, 1536, 50000])
def test_what_is_not_finite_stays_in_its_row(dt, C):
    g = gen(4)
    x = torch.randn(7, C, device=DEV, generator=g).to(dt)
    x[1, C // 2], x[3, 0], x[5] = float("nan"), float("inf"), 0.0
    y, c, s = torch.full_like(x, 5.0), torch.full(x.shape, 7, dtype=torch.int8, device=DEV), torch.zeros(7, device=DEV)
    B.dvdq_rms_norm(x, None, None, 1e-6, None, y, c, s)
    assert y[1].isnan().all() and s[1].isnan() and s[3].isnan() and (c[[1, 3, 5]] == 0).all()
    assert y[3, 0].isnan() and (y[3, 1:] == 0).all()          # infinity over itself, and the rest over infinity
    assert (y[5] == 0).all() and s[5] == 0
    rest = [0, 2, 4, 6]
    _, _, y6 = reference(x[rest], None, None, 1e-6)
    check(y[rest], y6, (U[dt] + (adds(C) / 2 + 6) * E) * y6.abs() + TINY[dt], "y")
    # a parameter that is not finite reaches its channel, and every row's scale
    gamma = torch.ones(C, device=DEV)
    gamma[3] = float("nan")
    B.dvdq_rms_norm(x[rest], None, gamma, 1e-6, None, z := torch.empty_like(x[rest]), d := torch.empty(4, C, dtype=torch.int8, device=DEV), t := torch.empty(4, device=DEV))
    assert z[:, 3].isnan().all() and z.isnan().sum() == 4 and t.isnan().all() and (d == 0).all()
    # no epsilon, nothing to divide by
    B.dvdq_rms_norm(x, None, None, 0.0, None, y)
    assert y[5].isnan().all() and y[rest].isfinite().all()


@gpu
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("M,K,layout", [(1, 1, "dense"), (5, 13, "dense"), (3, 1030, "padded"), (1500, 96, "padded"), (300, 1541, "odd"), (2000, 1536, "padded"),
                                        (40, 8960, "padded"), (2, 70000, "padded")])
def test_quantize_rows(dt, M, K, layout):
    g = gen(M + K)
    x = place((1, M, K), dt, layout, torch.randn(1, M, K, device=DEV, generator=g) * torch.rand(1, M, 1, device=DEV, generator=g))[0]
    x[M // 2] = 0
    c, s = place((1, M, K), torch.int8, layout)[0], torch.full((M,), float("nan"), device=DEV)
    B.dvdq_quantize_rows(x, c, s)
    check_codes(c, s, x.double(), 2 * E)
    assert (c[M // 2] == 0).all() and s[M // 2] == 0
    # the scale is the row's largest value over 127 to the last bit
    assert torch.equal(s, x.float().abs().amax(1) / torch.full((M,), 127.0, device=DEV))
    # values that whole multiples of the scale stand for come back
    back = torch.empty_like(c)
    B.dvdq_quantize_rows((c.float() * 0.5), back, s)
    assert torch.equal(back, c)


@gpu
def test_ties_go_to_even_and_tiny_rows_keep_their_codes():
    x = torch.tensor([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 126.5]], device=DEV)
    for f in (1.0, 2.0 ** 100, 2.0 ** -120):   # the last: scales near the smallest normal number
        c, s = torch.empty(1, 8, dtype=torch.int8, device=DEV), torch.empty(1, device=DEV)
        B.dvdq_quantize_rows(x * f, c, s)
        assert c[0].tolist() == [127, 0, 2, 2, 0, -2, -2, 126] and float(s[0]) == f
    x = torch.tensor([[2.0 ** -140, -2.0 ** -141, 0.0]], device=DEV)
    c, s = torch.empty(1, 3, dtype=torch.int8, device=DEV), torch.empty(1, device=DEV)
    B.dvdq_quantize_rows(x, c, s)
    assert c[0].tolist() == [127, -64, 0]


# ------------------------------------------------------------------ gradients

def gradient64(dy, h, rstd, gamma, dh):
    q = rstd.double()[..., None]
    hh, d = h.double() * q, dy.double() if gamma is None else dy.double() * gamma.double()
    along = (d * hh).mean(-1, keepdim=True)
    dx = q * (d - hh * along)
    return dx if dh is None else dx + dh.double(), q * d, q * hh, (d * hh).abs().mean(-1, keepdim=True), dy.double() * hh


@gpu
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("shape", SHAPES + [(1, 5000, 320), (3000, 12, 128), (700, 5, 96), (1, 700, 768), (3, 211, 1200), (1, 1000, 1544), (2, 300, 2560), (1, 650, 8008),
                                            (1, 620, 8960)])
@pytest.mark.parametrize("layout,residual,params,outs", [("dense", True, "own", "xg"), ("heads", False, "fp32", "xg"), ("padded", True, None, "x"),
                                                         ("odd", False, "own", "g"), ("turned", True, "fp32", "xg")])
def test_backward(dt, shape, layout, residual, params, outs):
    N, S, C = shape
    g = gen(N * 7 + S * 3 + C)
    dy, h = (place(shape, dt, l, torch.randn(shape, device=DEV, generator=g)) for l in ("dense" if layout == "turned" else layout, layout))
    dh = place(shape, dt, layout, torch.randn(shape, device=DEV, generator=g)) if residual else None
    gamma = None if params is None else (1 + torch.randn(C, device=DEV, generator=g)).to(dt if params == "own" else torch.float32)
    rstd = (h.double().square().mean(-1) + 1e-6).rsqrt().float()
    dx = place(shape, dt, layout) if "x" in outs else None
    dgamma = torch.full((C,), float("nan"), device=DEV) if "g" in outs else None
    ws = torch.full((B.dvdq_rms_norm_backward_workspace_bytes(N, S, C),), 255, dtype=torch.uint8, device=DEV) if "g" in outs else None
    B.dvdq_rms_norm_backward(dy, h, rstd, gamma, dh, dx, dgamma, ws)
    status_ok()
    want, d6, hh6, along, t6 = gradient64(dy, h, rstd, gamma, dh)
    if dx is not None:
        inner = adds(C) * E * hh6.abs() * along + 8 * E * (d6.abs() + hh6.abs() * along) + 2 * E * want.abs()
        check(dx, want, inner + U[dt] * (want.abs() + inner) + TINY[dt], "dx")
    if dgamma is not None:
        check(dgamma, t6.sum((0, 1)), (N * S / 100 + 40) * E * t6.abs().sum((0, 1)) + 1e-30, "dgamma")


@gpu
@pytest.mark.parametrize("dt", DTYPES)
def test_backward_in_place_and_again_the_same_bits(dt):
    g = gen(6)
    shape = (1, 3001, 776)
    dy, h, dh = (torch.randn(shape, device=DEV, generator=g).to(dt) for _ in range(3))
    rstd = (h.double().square().mean(-1) + 1e-6).rsqrt().float()
    gamma = torch.randn(776, device=DEV, generator=g)
    ws = torch.empty(B.dvdq_rms_norm_backward_workspace_bytes(*shape), dtype=torch.uint8, device=DEV)
    dx, dg = torch.empty_like(h), torch.empty(776, device=DEV)
    B.dvdq_rms_norm_backward(dy, h, rstd, gamma, dh, dx, dg, ws)
    for i in range(3):
        t = [dy.clone(), h.clone(), dh.clone()]
        dg2 = torch.empty(776, device=DEV)
        B.dvdq_rms_norm_backward(t[0], t[1], rstd, gamma, t[2], t[i], dg2, ws.fill_(255))
        assert torch.equal(t[i], dx) and torch.equal(dg2, dg)


# dgamma by columns: whole and partial groups of columns and of rows, single elements and pieces, every number of lanes to a row; and where sums of CTAs
# take over (rows, rows a lane, bytes)
FEW_ROWS = [(1, 2, 64), (1, 96, 33), (1, 512, 1536), (1, 591, 2560), (1, 592, 2560), (1, 577, 128), (49, 12, 72), (1, 590, 40), (1, 300, 5120), (1, 100, 16384), (1, 590, 1541),
            (3, 130, 1542), (2, 256, 8192), (1, 591, 14336), (1, 60, 12001)]


@gpu
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("shape", FEW_ROWS)
@pytest.mark.parametrize("layout,residual,params,outs", [("dense", True, "own", "xg"), ("heads", False, "fp32", "xg"), ("odd", True, "own", "xg"), ("padded", False, None, "g")])
def test_gradients_of_few_rows(dt, shape, layout, residual, params, outs):
    """A lane adds 24 products at most in fp32, and doubles join the lanes: 26 E of the bound's 40."""
    test_backward(dt, shape, layout, residual, params, outs)


@gpu
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("shape", [(1, 509, 1536), (1, 70, 131), (30, 12, 64), (1, 128, 5120)])
def test_few_rows_in_place_have_the_same_bits(dt, shape):
    g, C = gen(8), shape[-1]
    dy, h, dh = (torch.randn(shape, device=DEV, generator=g).to(dt) for _ in range(3))
    rstd = (h.double().square().mean(-1) + 1e-6).rsqrt().float()
    gamma = torch.randn(C, device=DEV, generator=g)
    ws = torch.empty(B.dvdq_rms_norm_backward_workspace_bytes(*shape), dtype=torch.uint8, device=DEV)
    dx, dg = torch.empty_like(h), torch.empty(C, device=DEV)
    B.dvdq_rms_norm_backward(dy, h, rstd, gamma, dh, dx, dg, ws)
    for i in range(3):
        for _ in range(3):
            t = [dy.clone(), h.clone(), dh.clone()]
            dg2 = torch.empty(C, device=DEV)
            B.dvdq_rms_norm_backward(t[0], t[1], rstd, gamma, t[2], t[i], dg2, ws.fill_(255))
            assert torch.equal(t[i], dx) and torch.equal(dg2, dg)
    status_ok()


@gpu
def test_a_row_that_is_not_finite_leaves_the_other_columns_of_dgamma():
    g = gen(9)
    for C in (1536, 131):
        dy, h = (torch.randn(1, 200, C, device=DEV, generator=g) for _ in range(2))
        rstd, ws = torch.ones(1, 200, device=DEV), torch.empty(B.dvdq_rms_norm_backward_workspace_bytes(1, 200, C), dtype=torch.uint8, device=DEV)
        clean, dg, dx = torch.empty(C, device=DEV), torch.empty(C, device=DEV), torch.empty_like(h)
        B.dvdq_rms_norm_backward(dy, h, rstd, None, None, dx, clean, ws)
        h[0, 199, 7], dy[0, 3, 100] = float("inf"), float("nan")
        B.dvdq_rms_norm_backward(dy, h, rstd, None, None, dx, dg, ws)
        assert dg[7].isinf() and dg[100].isnan()
        keep = torch.ones(C, dtype=torch.bool, device=DEV)
        keep[[7, 100]] = False
        assert torch.equal(dg[keep], clean[keep])


@gpu
def test_gradients_are_those_of_the_forward_pass_by_differences():
    g = gen(7)
    C, eps, step = 37, 1e-3, 1e-2
    x, r, w = (torch.randn(4, C, device=DEV, generator=g) for _ in range(3))
    gamma = torch.randn(C, device=DEV, generator=g)

    def loss(x, r, gamma):   # sum w y + sum h^2 / 2, whose gradient along the residual stream is h
        h, y = torch.empty_like(x), torch.empty_like(x)
        B.dvdq_rms_norm(x, r, gamma, eps, h, y)
        return float((w.double() * y.double()).sum() + h.double().square().sum() / 2)

    h, rstd, dx, dg = torch.empty_like(x), torch.empty(4, device=DEV), torch.empty_like(x), torch.empty(C, device=DEV)
    B.dvdq_rms_norm(x, r, gamma, eps, h, None, None, None, rstd)
    ws = torch.empty(B.dvdq_rms_norm_backward_workspace_bytes(1, 4, C), dtype=torch.uint8, device=DEV)
    B.dvdq_rms_norm_backward(w, h, rstd, gamma, h, dx, dg, ws)
    for t, grad in ((x, dx), (r, dx), (gamma, dg)):
        for i in (0, 5, t.numel() - 1):
            sides = []
            for sign in (1, -1):
                moved = t.clone()
                moved.view(-1)[i] += sign * step
                sides.append(loss(*(moved if a is t else a for a in (x, r, gamma))))
            # a third derivative of order one times step^2, and the loss's own rounding over the step
            assert abs((sides[0] - sides[1]) / (2 * step) - float(grad.view(-1)[i])) < 20 * step ** 2 + 1e-3


@gpu
def test_no_rows():
    for dt in DTYPES:
        e = torch.empty(0, 40, dtype=dt, device=DEV)
        B.dvdq_rms_norm(e, None, None, 1e-6, None, torch.empty_like(e))
        B.dvdq_quantize_rows(e, torch.empty(0, 40, dtype=torch.int8, device=DEV), torch.empty(0, device=DEV))
        dg = torch.ones(40, device=DEV)
        B.dvdq_rms_norm_backward(e, e, torch.empty(0, device=DEV), None, None, None, dg)
        assert (dg == 0).all()
    assert B.dvdq_rms_norm_backward_workspace_bytes(0, 5, 40) == 0


@gpu
def test_binding_refuses():
    x = torch.randn(4, 6, 8, device=DEV)
    y, c, s = torch.empty_like(x), torch.empty(x.shape, dtype=torch.int8, device=DEV), torch.empty(4, 6, device=DEV)
    for bad in (lambda: B.dvdq_rms_norm(x, None, None, 1e-6, None, y.half()), lambda: B.dvdq_rms_norm(x, x[:2], None, 1e-6, None, y),
                lambda: B.dvdq_rms_norm(x, None, torch.ones(7, device=DEV), 1e-6, None, y), lambda: B.dvdq_rms_norm(x.double(), None, None, 1e-6, None, y),
                lambda: B.dvdq_rms_norm(x, None, torch.ones(8, device=DEV).half(), 1e-6, None, y), lambda: B.dvdq_rms_norm(x.transpose(1, 2), None, None, 1e-6, None, y),
                lambda: B.dvdq_rms_norm(x, None, None, 1e-6, None, None, c, s[:3]), lambda: B.dvdq_rms_norm(x[0, 0], None, None, 1e-6, None, y[0, 0]),
                lambda: B.dvdq_rms_norm(x, None, None, 1e-6, None, None, c.float(), s), lambda: B.dvdq_rms_norm(x.cpu(), None, None, 1e-6, None, y),
                lambda: B.dvdq_quantize_rows(x, c, s), lambda: B.dvdq_quantize_rows(x[0], c[0], s[0, :5])):
        with pytest.raises((TypeError, ValueError)):
            bad()
    with pytest.raises(ValueError):   # memory of the host beside memory of the device
        B.dvdq_rms_norm(x, None, None, 1e-6, None, y.cpu())
    for call, status in ((lambda: B.dvdq_rms_norm(x, None, None, -1.0, None, y), B.ERR_SHAPE), (lambda: B.dvdq_rms_norm(x, None, None, 1e-6), B.ERR_NULL),
                         (lambda: B.dvdq_rms_norm(x, None, None, 1e-6, None, None, c), B.ERR_NULL),
                         (lambda: B.dvdq_rms_norm(x, None, None, 1e-6, y, y), B.ERR_SHAPE),
                         (lambda: B.dvdq_rms_norm_backward(x, x, s, None, None, None, torch.empty(8, device=DEV), None), B.ERR_NULL),
                         (lambda: B.dvdq_rms_norm_backward(x, x, s, None, None, None, torch.empty(8, device=DEV), torch.empty(256, dtype=torch.uint8, device=DEV)), B.ERR_WORKSPACE)):
        with pytest.raises(B.DvdqError) as e:
            call()
        assert e.value.status == status


def test_argument_structs_are_packed_as_the_header_lays_them_out():
    import ctypes as C
    p, i64 = C.c_void_p, C.c_int64

    def size(counts, tail):
        fields = [(f"f{i}", i64) for i in range(counts)] + [(f"t{i}", t) for i, t in enumerate(tail)]
        return C.sizeof(type("S", (C.Structure,), {"_fields_": fields}))

    assert B.RMS_NORM_ARGS.size == size(21, [C.c_int32, C.c_int32, C.c_float])
    assert B.RMS_NORM_BACKWARD_ARGS.size == size(20, [C.c_int32, C.c_int32])
    assert B.LINEAR_INT8_ARGS.size == size(16, [C.c_int32, C.c_int32])


def test_refusals_before_any_cuda_call():
    import ctypes as C
    lib = B.load()
    one, two = 256, 512   # never dereferenced: validation fails first

    def norm(N=2, S=3, Ch=8, x=one, r=0, gamma=0, pt=B.F32, eps=1e-6, h=0, y=two, yo=24, yr=8, c=0, s=0, q=0, dt=B.F32, xo=24, xr=8):
        return lib.dvdq_rms_norm(B.RMS_NORM_ARGS.pack(x or 0, xo, xr, r, 24, 8, h, yo, yr, y or 0, yo, yr, c, 24, 8, N, S, Ch, gamma, s, q, pt, dt, eps), None)

    assert lib.dvdq_rms_norm(None, None) == lib.dvdq_rms_norm_backward(None, None) == B.ERR_NULL
    assert norm(Ch=0) == norm(Ch=(1 << 20) + 1, xo=1 << 24, yo=1 << 24) == norm(N=-1) == norm(N=1 << 20, S=1 << 20) == B.ERR_SHAPE
    assert norm(eps=-1e-6) == norm(eps=float("nan")) == norm(eps=float("inf")) == B.ERR_SHAPE
    assert norm(dt=3) == norm(pt=B.F16) == norm(pt=7) == B.ERR_UNSUPPORTED
    assert norm(x=None) == norm(y=None) == norm(c=one) == norm(s=one) == B.ERR_NULL
    assert norm(yr=7) == norm(yo=4) == norm(xr=-8) == B.ERR_SHAPE                      # outputs that overlap, a negative pitch
    assert norm(y=one, yo=48) == norm(r=two, yo=48) == norm(h=two) == B.ERR_SHAPE       # in place with other pitches; two outputs in one place
    assert norm(y=514) == norm(gamma=258) == norm(q=514) == norm(c=one, s=514) == B.ERR_ALIGN
    assert norm(N=0) == norm(S=0, x=None) == B.OK

    def back(N=2, S=3, Ch=8, dy=one, h=one, q=one, dh=0, gamma=0, pt=B.F32, dx=two, xr=8, dg=0, dt=B.F32, ws=0, room=0):
        return lib.dvdq_rms_norm_backward(B.RMS_NORM_BACKWARD_ARGS.pack(dy or 0, 24, 8, h or 0, 24, 8, dh, 24, 8, dx or 0, 24, xr, N, S, Ch, gamma, q or 0, dg, ws, room,
                                                                        pt, dt), None)

    assert back(dx=None) == back(dy=None) == back(h=None) == back(q=None) == B.ERR_NULL
    assert back(dg=one) == B.ERR_NULL and back(dg=one, ws=128, room=1 << 20) == B.ERR_ALIGN and back(dg=one, ws=one, room=100) == B.ERR_WORKSPACE
    assert back(xr=4) == back(dx=one, xr=9) == back(Ch=0) == B.ERR_SHAPE
    assert back(dt=5) == back(pt=B.BF16) == B.ERR_UNSUPPORTED and back(q=6) == back(dx=6) == B.ERR_ALIGN
    assert back(N=0) == B.OK

    p = C.c_void_p

    def rows(M=4, K=8, x=one, ldx=8, c=two, ldc=8, s=one, dt=B.F32):
        return lib.dvdq_quantize_rows(x, M, K, ldx, c, ldc, s, dt, None)

    assert rows(M=-1) == rows(K=0) == rows(M=1 << 31) == rows(ldc=7) == rows(ldx=-1) == B.ERR_SHAPE
    assert rows(x=None) == rows(c=None) == rows(s=None) == B.ERR_NULL and rows(dt=9) == B.ERR_UNSUPPORTED
    assert rows(x=p(258)) == rows(s=p(258)) == B.ERR_ALIGN and rows(M=0, x=None) == B.OK
    assert B.dvdq_rms_norm_backward_workspace_bytes(1, 10, 0) == 0 and B.dvdq_rms_norm_backward_workspace_bytes(1, 10, 64) == 10 * 64 * 4
    assert B.dvdq_rms_norm_backward_workspace_bytes(1, 1 << 30, 1 << 20) <= 256 << 20

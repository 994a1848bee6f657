"""dvdq_rms_norm where h, gamma or their products leave the middle of fp32's range, against the formula in 64 bits.

Tolerances as in test_rms_norm.py, with two halves of the smallest number more for y (2^-150 from each of the two products behind h q: y is (h q) gamma, rounded twice) and for scales
(y's, and their own).  Codes: what they stand for, c s, is within half a step of y; s is off by 2^-150 at most, which 127 steps multiply.
"""
import pytest
import torch

from paper_2505_18663_b200 import binding as B

gpu = pytest.mark.gpu
DEV = "cuda"
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}
E = 2.0 ** -24
# lanes of a row, a warp's row, rows of a CTA, rows that are read twice; pieces of 16 bytes and single elements
WIDTHS = [4, 12, 37, 300, 1541, 4096, 50000]


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def check_row_outputs(y, c, s, y6, C, dt):
    rel = ((80 if C <= 8192 else 80 + C // 1024) / 2 + 8) * E
    over = (y.double() - y6).abs() - ((U[dt] + rel) * y6.abs() + TINY[dt] + 2.0 ** -149)
    assert y.isfinite().all() and float(over.max()) <= 0
    top = y6.abs().amax(-1)
    assert float(((s.double() - top / 127).abs() - (rel + 4 * E) * top / 127 - 2.0 ** -148).max()) <= 0
    stands = c.double() * s.double()[..., None]
    half = s.double()[..., None] / 2
    assert float(((stands - y6).abs() - half * (1 + 2.0 ** -14) - rel * y6.abs() - 127 * 2.0 ** -149).max()) <= 0


# h and gamma of these sizes: products below 2^-126 and below 2^-149, of rows with and without eps, with squares that are zero in fp32
SMALL = [(1e-15, 1e-30, 0.0), (2e-22, 1e-23, 1e-6), (1e-36, 1e-8, 1e-6), (1e-30, 1e-16, 1e-6), (1e-10, 1e-35, 1e-6), (1e-3, 1e-41, 1e-6), (1e-20, 1e-20, 1e-38)]


@gpu
@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scale,size,eps", SMALL)
def test_codes_where_h_gamma_is_subnormal(scale, size, eps, dt, C):
    """Among rows of ordinary size and rows of zeros."""
    g = gen(C)
    x = (torch.rand(11, C, device=DEV, generator=g) * 2 - 1) * scale
    x[3], x[7] = x[3] / scale, 0.0
    x = x.to(dt)
    gamma = (torch.rand(C, device=DEV, generator=g) + 0.5) * size
    y, c, s = torch.empty_like(x), torch.full(x.shape, 99, dtype=torch.int8, device=DEV), torch.empty(11, device=DEV)
    eps = float(torch.tensor(eps, dtype=torch.float32))
    B.dvdq_rms_norm(x, None, gamma, eps, None, y, c, s)
    rows = [i for i in range(11) if eps > 0 or i != 7]   # zeros without eps have no y
    x6 = x[rows].double()
    y6 = x6 * (x6.square().mean(-1, keepdim=True) + eps).rsqrt() * gamma.double()
    check_row_outputs(y[rows], c[rows], s[rows], y6, C, dt)
    assert (c[7] == 0).all() and (s[7].isnan() if eps == 0 else s[7] == 0)


@gpu
@pytest.mark.parametrize("a,size,eps", [(1e-15, 1e-30, 0.0), (1e-15, 1e-30, 1e-37), (1e-22, 1e-23, 0.0)])
def test_an_example_by_hand(a, size, eps):
    """h = (2, -1.5, 1, 0.5) a: whatever q and gamma, y is (127, -95.25, 63.5, 31.75) steps."""
    x = torch.tensor([[2.0, -1.5, 1.0, 0.5]], device=DEV) * a
    c, s = torch.empty(1, 4, dtype=torch.int8, device=DEV), torch.empty(1, device=DEV)
    B.dvdq_rms_norm(x, None, torch.full((4,), size, device=DEV), eps, None, None, c, s)
    got = c[0].tolist()
    assert got[:2] == [127, -95] and got[2] in (63, 64) and got[3] == 32


# sizes of h and gamma: squares beyond fp32 either way, h gamma beyond it while the squares are not, both at once
FAR = [(1e25, 1.0, 1e-6), (1e30, 1e-3, 1e-6), (1e-30, 1.0, 0.0), (1e-30, 1e4, 0.0), (3e10, 1e29, 1e-6), (1e14, 3e25, 0.0), (3e37, 50.0, 1e-6), (1e-24, 1e-3, 1e-37)]


@gpu
@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("dt,params", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("scale,size,eps", FAR)
@pytest.mark.parametrize("over", [None, "x", "r", "alone"])
def test_gamma_and_residual_of_rows_far_from_one(scale, size, eps, dt, params, C, over):
    """Among ordinary rows that share a warp or a CTA with them.  h goes beside x and r, over x or over r; alone: no residual.  Y is of the size of gamma.
    With |x| and |r| below `scale`, h is rounded in fp32 by 2^-24 of itself, which q and y pass on."""
    g = gen(C + 1)
    x, r = (torch.rand(9, C, device=DEV, generator=g) * 2 - 1 for _ in range(2))
    for t in (x, r):
        t[::2] *= scale
        t[5] = 0
    x, r = x.to(dt), None if over == "alone" else r.to(dt)
    gamma = ((torch.rand(C, device=DEV, generator=g) + 0.5) * size).to(params)
    eps = float(torch.tensor(eps, dtype=torch.float32))
    h6 = x.double() + (0 if r is None else r.double())
    h = {None: torch.empty_like(x), "x": x, "r": r, "alone": None}[over]
    y, c = torch.empty_like(x), torch.full(x.shape, 99, dtype=torch.int8, device=DEV)
    s, q = torch.empty(9, device=DEV), torch.empty(9, device=DEV)
    B.dvdq_rms_norm(x, r, gamma, eps, h, y, c, s, q)
    q6 = (h6.square().mean(-1, keepdim=True) + eps).rsqrt()
    rows = [i for i in range(9) if eps > 0 or i != 5]
    check_row_outputs(y[rows], c[rows], s[rows], (h6 * q6 * gamma.double())[rows], C, dt)
    rel = ((80 if C <= 8192 else 80 + C // 1024) / 2 + 8) * E
    fine = [i for i in rows if q6[i, 0] < 3e38]
    assert float(((q[fine].double() - q6[fine, 0]).abs() - rel * q6[fine, 0] - 2.0 ** -149).max()) <= 0
    if h is not None:
        assert float(((h.double() - h6).abs() - (U[dt] + 2 * E) * h6.abs() - TINY[dt]).max()) <= 0


@gpu
@pytest.mark.parametrize("C", [40, 1536, 50000])
def test_far_rows_give_the_same_bits_in_place(C):
    g = gen(C + 2)
    x, r = ((torch.rand(6, C, device=DEV, generator=g) * 2 - 1) * torch.tensor([1.0, 1e30, 1e-30, 1e25, 1.0, 1e-35], device=DEV)[:, None] for _ in range(2))
    gamma = torch.rand(C, device=DEV, generator=g) + 0.5

    def outputs(x, r, h, y):
        c, s, q = torch.empty(x.shape, dtype=torch.int8, device=DEV), torch.empty(6, device=DEV), torch.empty(6, device=DEV)
        B.dvdq_rms_norm(x, r, gamma, 1e-12, h, y, c, s, q)
        return [t.clone() for t in (h, y, c, s, q)]

    want = outputs(x, r, torch.empty_like(x), torch.empty_like(x))
    for swap in (False, True):
        a, b = x.clone(), r.clone()
        got = outputs(a, b, *((b, a) if swap else (a, b)))
        assert all(torch.equal(t, w) for t, w in zip(got, want))

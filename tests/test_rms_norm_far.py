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

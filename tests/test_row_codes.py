"""Codes of dvdq_quantize_rows and dvdq_rms_norm next to their borders: c = round_half_even(127 y / max |y|).

Rows in 16 bits: to the bit.  Values in 32 bits (a norm's y among them): the same wherever the quotient is half of an odd number; else it may be off by 2^-22 of itself
(the factor 127 / max |y|, rounded up, or the divisor max |y| / 127, rounded down, by 2^-23, and a quotient's own rounding by 2^-24), and next to a border the code is one of
the two beside it.  With gamma max |y| is taken as q max |h gamma|, y as (h q) gamma: four roundings, 2^-22, more.
"""
import pytest
import torch

from paper_2505_18663_b200 import binding as B

gpu = pytest.mark.gpu
DEV = "cuda"
DTYPES = [torch.bfloat16, torch.float16, torch.float32]
BITS = {torch.bfloat16: 7, torch.float16: 10}


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def quotient(y, s):
    """In fp32, on the host; 0 where there is no scale."""
    y, s = y.float().cpu(), s.cpu()[..., None]
    return torch.where(s > 0, y / s, torch.zeros(()))


def tie(y, top):
    """Where y is half of an odd number of steps: products of a number below 256 and a mantissa are exact in fp64."""
    n = torch.round(y.abs() * 254 / top)   # twice the number of steps
    return (n % 2 == 1) & (n * top == y.abs() * 254)


def check_codes(c, y, gamma=False):
    c, v = c.cpu().double(), y.double().cpu()
    top = v.abs().amax(-1, keepdim=True)
    q = torch.where(top > 0, v * 127 / torch.where(top > 0, top, 1.0), 0.0)
    ties = tie(v, top)
    off = c != torch.where(ties, 2 * torch.round(q / 2), torch.round(q))   # a half to even; fp64 may have put it beside the border
    if y.dtype is torch.float32:
        border = (torch.floor(q.abs()) + 0.5 - q.abs()).abs()
        off &= (ties & (not gamma)) | (border > q.abs() * 2.0 ** (-21 if gamma else -22)) | ((c - q).abs() > 0.501)
    assert not off.any()
    return int(ties.sum())


def tops(dt):
    """Largest values of rows: every mantissa in 16 bits, in 32 odd multiples of 127 and others; small and large ones among them."""
    if dt is torch.float32:
        g = torch.Generator().manual_seed(1)
        m = torch.cat([torch.randint(1 << 23, 1 << 24, (1500,), generator=g), 127 * torch.randint((1 << 23) // 127 + 1, (1 << 24) // 127, (500,), generator=g)])
        m = m.double() * 2.0 ** -23
    else:
        m = 1 + torch.arange(1 << BITS[dt]).double() * 2.0 ** -BITS[dt]
    exponents = (0, -8, 5) if dt is torch.float16 else (0, -80, -95, -118, 100)
    return torch.cat([m * 2.0 ** e for e in exponents]).to(dt)


@gpu
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("layout", ["whole", "tail", "odd"])
def test_values_at_and_next_to_a_border(dt, layout):
    """Halves of steps as near as the type has them, with the two values on each side: among them the exact ties, and top / 2 = 63.5 steps."""
    top = tops(dt)
    half = ((torch.arange(127).double() + 0.5)[None, :] * top.double()[:, None] / 127).to(dt)
    bits = torch.int32 if dt is torch.float32 else torch.int16
    near = torch.cat([(half.view(bits) + d).view(dt) for d in range(-2, 3)], 1)
    near[:, 1::2] *= -1
    rows = torch.cat([top[:, None], near.minimum(top[:, None]).maximum(-top[:, None])], 1)   # 636 values
    M, K = rows.shape[0], 640 if layout == "whole" else 636
    x = torch.zeros(M * 648 + 1, dtype=dt, device=DEV)[1 if layout == "odd" else 0:][:M * 648].view(M, 648)[:, :K]
    x[:, :636] = rows.to(DEV)
    c, s = torch.full((M, 656), 99, dtype=torch.int8, device=DEV)[:, :K], torch.empty(M, device=DEV)
    B.dvdq_quantize_rows(x, c, s)
    assert torch.equal(s.cpu(), top.float() / torch.full((M,), 127.0))
    assert check_codes(c, x) >= M


@gpu
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
def test_every_value_of_16_bits_under_every_top(dt):
    n = 1 << BITS[dt]
    m = (1 + torch.arange(n).double() / n)
    y = torch.cat([m * 2.0 ** -e for e in range(9)])   # down to less than half a step
    x = torch.cat([m[:, None], y[None, :].minimum(m[:, None])], 1).to(dt).to(DEV)
    x = torch.nn.functional.pad(x, (0, -x.shape[1] % 16))
    c, s = torch.empty(x.shape, dtype=torch.int8, device=DEV), torch.empty(n, device=DEV)
    B.dvdq_quantize_rows(x, c, s)
    check_codes(c, x)


@gpu
@pytest.mark.parametrize("shape", [(300, 8, 40), (1, 900, 96), (40, 12, 128), (1, 500, 1541), (1, 700, 1536), (1, 200, 5120), (1, 8, 5120), (1, 40, 9001), (2, 3, 50000)])
@pytest.mark.parametrize("residual,gamma", [(False, False), (True, True)])
def test_codes_of_the_norm_are_those_of_its_output(shape, residual, gamma):
    """In fp32 the output is y itself.  Values of 8 bits with a largest one: without gamma, halves of it are ties here too."""
    g = gen(shape[1] + shape[2])
    x, r = (torch.randn(shape, device=DEV, generator=g).bfloat16().float() for _ in range(2))
    x[..., 1], x[..., 2], x[..., shape[2] - 1] = x.abs().amax(-1), x.abs().amax(-1) / 2, x.abs().amax(-1) / -2
    w = torch.randn(shape[2], device=DEV, generator=g) if gamma else None
    y, c, s = torch.empty_like(x), torch.empty(shape, dtype=torch.int8, device=DEV), torch.empty(shape[:2], device=DEV)
    B.dvdq_rms_norm(x, r if residual else None, w, 1e-6, None, y, c, s)
    assert check_codes(c, y, gamma) or gamma


@gpu
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("C", [5, 64, 1541])
def test_scales_among_the_smallest_numbers(dt, C):
    """A scale below 2^-126 is a multiple of 2^-149: codes count that scale, so that c s is within half of it of y, or, where y is more than 127 of it, as near as 127 steps come
    (s is at most 2^-150 below max |y| / 127).  No scale, no codes."""
    g = torch.Generator().manual_seed(C)
    units = torch.cat([torch.arange(1, 400), torch.randint(400, 1 << 14, (400,), generator=g), torch.randint(1 << 14, 1 << 28, (400,), generator=g)]).double()
    x = (torch.rand(units.numel(), C, generator=g, dtype=torch.float64) * 2 - 1) * units[:, None]
    x[:, C // 2] = units
    x = (torch.round(x) * 2.0 ** -149).to(dt).to(DEV)
    c, s = torch.full(x.shape, 99, dtype=torch.int8, device=DEV), torch.empty(x.shape[0], device=DEV)
    B.dvdq_quantize_rows(x, c, s)
    top = x.double().abs().amax(-1)
    assert torch.equal(s.cpu(), top.cpu().float() / torch.full_like(top, 127.0).cpu().float())
    assert (s == 0).any() or dt is torch.bfloat16
    want = quotient(x, s).clamp(-127, 127)
    small = s.cpu() < 2.0 ** -126
    assert small.any() and torch.equal(c.cpu()[small].float(), torch.round(want)[small])
    off = (c.double() * s.double()[:, None] - x.double()).abs() - s.double()[:, None] / 2 * (1 + 2.0 ** -14) - 127 * 2.0 ** -150
    assert float(off.max()) <= 0

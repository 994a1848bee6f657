"""The norm's forward pass on rows past 2^31 elements against the same rows in a small tensor of their own."""
import pytest
import torch

from paper_2505_18663_b200 import binding as B

gpu = pytest.mark.gpu
DEV = "cuda"
LAST = 2000   # rows; as many as the kernels need to lay them out as they do millions


@gpu
@pytest.mark.parametrize("rows,C", [(1_100_000, 2048), (450_000, 5120), (1_500_000, 1541)])
def test_the_last_rows_are_those_of_a_small_tensor(rows, C):
    g = torch.Generator(device=DEV).manual_seed(rows)
    dt = torch.bfloat16
    assert (rows - LAST) * C > 1 << 31
    x = torch.zeros(rows, C, dtype=dt, device=DEV)
    x[-LAST:] = (torch.randn(LAST, C, generator=g, device=DEV) * torch.rand(LAST, 1, generator=g, device=DEV)).to(dt)
    r = torch.randn(LAST, C, generator=g, device=DEV).to(dt)
    gamma = torch.randn(C, generator=g, device=DEV)
    small = x[-LAST:].clone()

    def outputs(n):
        return torch.empty(n, C, dtype=torch.int8, device=DEV), torch.empty(n, device=DEV), torch.empty(n, device=DEV)

    y, want = torch.empty_like(small), outputs(LAST)
    B.dvdq_rms_norm(small, None, gamma, 1e-6, None, y, *want)
    y6 = small.double() * (small.double().square().mean(-1, keepdim=True) + 1e-6).rsqrt() * gamma.double()
    assert (y.double() - y6).abs().le(2.0 ** -8 * (1 + 2.0 ** -12) * y6.abs() + 2.0 ** -134).all()   # (80 / 2 + 6) 2^-24 < 2^-18 before the rounding
    c, s, q = outputs(rows)
    B.dvdq_rms_norm(x, None, gamma, 1e-6, None, x, c, s, q)   # y over x
    for t, w in zip((x, c, s, q), (y, *want)):
        assert torch.equal(t[-LAST:], w)
    assert (s[:-LAST] == 0).all() and (c[:-LAST:977] == 0).all() and (x[:-LAST:977] == 0).all()
    # with a residual that is as far away, h over it
    x[-LAST:] = small
    far = torch.zeros_like(x)
    far[-LAST:] = r
    h, y = torch.empty_like(small), torch.empty_like(small)
    B.dvdq_rms_norm(small, r, gamma, 1e-6, h, y, *want)
    B.dvdq_rms_norm(x, far, gamma, 1e-6, far, x, c, s, q)
    for t, w in zip((far, x, c, s, q), (h, y, *want)):
        assert torch.equal(t[-LAST:], w)
    assert B.dvdq_last_device_status()[0] == B.OK

"""dvdq_rope_frequencies, dvdq_rope_table and dvdq_rope against the formulas in 64 bits.

Tolerances: a rotated channel is one product and one fused multiply-add in fp32 (2 roundings of at most
2^-24 (|a| + |b|) times the amplitude), then one rounding to the type (u |y|).  Table entries: fp64 angles and sines,
one rounding to fp32 (2^-24), plus 2^-50 |angle| of the fp64 product."""
import ctypes as C
import math

import pytest
import torch

from paper_2505_18663_b200 import binding as B

gpu = pytest.mark.gpu
DEV = "cuda"
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def make_table(n, pairs, theta=10000.0):
    i = torch.arange(pairs, dtype=torch.float64, device=DEV)
    a = torch.arange(n, dtype=torch.float64, device=DEV)[:, None] * theta ** (-i / pairs)
    return torch.stack([a.cos(), a.sin()], -1).float().contiguous()


def turn(x, table, rot, layout, inverse):
    """x [B, S, H, D] in 64 bits, table [B or 1, S, rot / 2, 2]"""
    c, s = table[..., 0].double()[:, :, None], table[..., 1].double()[:, :, None]
    s = -s if inverse else s
    y = x.clone()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if layout == B.ROPE_PAIRS else (x[..., :rot // 2], x[..., rot // 2:rot])
    ya, yb = a * c - b * s, b * c + a * s
    if layout == B.ROPE_PAIRS:
        y[..., 0:rot:2], y[..., 1:rot:2] = ya, yb
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = ya, yb
    return y


def check(got, x, want, dt):
    bound = U[dt] * want.abs() + 2.0 ** -21 * (x.abs() + x.abs().amax(-1, keepdim=True)) + (2.0 ** -25 if dt == torch.float16 else 0)
    bound = torch.where(want == x, U[dt] * want.abs() + 2.0 ** -21 * x.abs().amax(-1, keepdim=True) + 2.0 ** -25, bound)
    assert (got.double() - want).abs().le(bound).all(), float((got.double() - want).abs().max())


# (B, S, Hq, Hk, D, rot): whole heads and parts; widths that 16, 8, 4 and 2 byte accesses divide; one token; one head;
# many tokens (four heads per thread)
SHAPES = [(1, 1, 1, 1, 2, 2), (2, 3, 2, 1, 64, 64), (1, 5, 3, 3, 80, 40), (3, 1, 8, 2, 128, 64), (1, 7, 5, 1, 72, 34), (2, 4, 1, 1, 36, 36),
          (1, 33, 4, 2, 96, 96), (1, 9, 2, 2, 256, 62), (1, 2, 3, 1, 7, 6), (1, 3001, 12, 4, 128, 128), (2, 1500, 9, 9, 64, 32)]


@gpu
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("layout", [B.ROPE_PAIRS, B.ROPE_HALVES])
@pytest.mark.parametrize("inverse,gather", [(False, False), (True, True)])
def test_rotation(dt, shape, layout, inverse, gather):
    n, S, Hq, Hk, D, rot = shape
    g = torch.Generator(device=DEV).manual_seed(S + D)
    q, k = (torch.randn(n, S, h, D, generator=g, device=DEV).to(dt) for h in (Hq, Hk))
    T = S + 50
    table = make_table(T, rot // 2)
    rows = torch.randint(0, T, (n, S), generator=g, device=DEV, dtype=torch.int32) if gather else None
    qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    B.dvdq_rope(q, k, table, rows, layout, inverse, qo, ko)
    assert B.dvdq_last_device_status()[0] == B.OK
    picked = table[rows.long()] if gather else table[None, :S]
    for x, y in ((q, qo), (k, ko)):
        check(y, x.double(), turn(x.double(), picked, rot, layout, inverse), dt)
        assert torch.equal(y[..., rot:], x[..., rot:])
    # in place: the same bits
    B.dvdq_rope(q, k, table, rows, layout, inverse, q, k)
    assert torch.equal(q, qo) and torch.equal(k, ko)


@gpu
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", [B.ROPE_PAIRS, B.ROPE_HALVES])
@pytest.mark.parametrize("offset", [0, 1, 4])
def test_views_strides_and_alignments(dt, layout, offset):
    """q and k inside a fused projection's output that starts `offset` elements into its memory, heads before tokens in the
    output, rows shared by all sequences; nothing outside the views is written."""
    n, S, Hq, Hk, D = 2, 11, 4, 2, 32
    g = torch.Generator(device=DEV).manual_seed(3)
    flat = torch.randn(offset + n * S * (Hq + 2 * Hk) * D, generator=g, device=DEV).to(dt)
    fused = flat[offset:].view(n, S, Hq + 2 * Hk, D)
    q, k = fused[:, :, :Hq], fused[:, :, Hq:Hq + Hk]
    table = make_table(40, D // 2)
    rows = torch.randint(0, 40, (S,), generator=g, device=DEV, dtype=torch.int32)
    out = torch.full((n, Hq, S + 1, D), float("nan"), dtype=dt, device=DEV)
    qo, ko = out[:, :, :S].transpose(1, 2), torch.empty(n, S, Hk, D, dtype=dt, device=DEV)
    B.dvdq_rope(q, k, table, rows, layout, False, qo, ko)
    picked = table[rows.long()][None]
    check(qo, q.double(), turn(q.double(), picked, D, layout, False), dt)
    check(ko, k.double(), turn(k.double(), picked, D, layout, False), dt)
    assert out[:, :, S].isnan().all()
    before = flat.clone()
    B.dvdq_rope(q, k, table, rows, layout, False, q, k)
    assert torch.equal(q, qo) and torch.equal(k, ko)
    v = slice(Hq + Hk, None)
    assert torch.equal(fused[:, :, v], before[offset:].view_as(fused)[:, :, v]) and torch.equal(flat[:offset], before[:offset])


@gpu
def test_broadcast_input_and_query_alone():
    x = torch.randn(1, 6, 1, 64, device=DEV).expand(3, 6, 4, 64)
    y = torch.empty(3, 6, 4, 64, device=DEV)
    t = make_table(6, 32)
    B.dvdq_rope(x, None, t, None, B.ROPE_HALVES, False, y)
    check(y, x.double(), turn(x.double().clone(), t[None], 64, B.ROPE_HALVES, False), torch.float32)


@gpu
def test_the_inverse_is_the_gradient_and_undoes_the_rotation():
    """<y, dy> is bilinear: the gradient of sum(y dy) along any direction v is sum(rope(v) dy) = sum(v rope^-1(dy)), exactly in
    exact arithmetic; in fp32, sums of 2 * 5 * 3 * 64 products leave 1e-5 of the sum of magnitudes."""
    g = torch.Generator(device=DEV).manual_seed(4)
    v, dy = (torch.randn(2, 5, 3, 64, generator=g, device=DEV) for _ in range(2))
    t = make_table(5, 32)
    rv, back = torch.empty_like(v), torch.empty_like(v)
    for layout in (B.ROPE_PAIRS, B.ROPE_HALVES):
        B.dvdq_rope(v, None, t, None, layout, False, rv)
        B.dvdq_rope(dy, None, t, None, layout, True, back)
        left, right = (rv.double() * dy.double()).sum(), (v.double() * back.double()).sum()
        assert abs(float(left - right)) <= 1e-5 * float((rv * dy).abs().sum())
        B.dvdq_rope(rv, None, t, None, layout, True, back)
        assert (back - v).abs().max() <= 2.0 ** -20 * v.abs().max()


@gpu
def test_a_row_outside_the_table_is_reported():
    q = torch.randn(1, 4, 2, 16, device=DEV)
    t = make_table(8, 4)
    rows = torch.tensor([[0, 8, -1, 7]], dtype=torch.int32, device=DEV)
    y = torch.empty_like(q)
    B.dvdq_rope(q, None, t, rows, B.ROPE_PAIRS, False, y)
    assert B.dvdq_last_device_status() == (B.ERR_SHAPE, 16)
    assert B.dvdq_last_device_status()[0] == B.OK     # reading clears it
    assert y[0, 1:3, :, :8].isnan().all() and torch.equal(y[..., 8:], q[..., 8:])
    assert y[0, [0, 3]].isfinite().all()


@gpu
def test_no_tokens():
    e = torch.empty(1, 0, 2, 8, device=DEV)
    B.dvdq_rope(e, None, make_table(1, 4), None, B.ROPE_PAIRS, False, e)


@gpu
@pytest.mark.parametrize("axes", [1, 3])
def test_table(axes):
    pairs, T, amp = 22, 700, 1.25
    freqs, _ = B.dvdq_rope_frequencies(2 * pairs, 10000.0)
    g = torch.Generator(device=DEV).manual_seed(5)
    pos = torch.randint(0, 1 << 20, (T, axes), generator=g, device=DEV, dtype=torch.int32)
    axis = [i * axes // pairs for i in range(pairs)]
    table = torch.empty(T, pairs, 2, device=DEV)
    B.dvdq_rope_table(freqs, pos[:, 0].contiguous() if axes == 1 else pos, table, axis if axes > 1 else None, amp)
    a = pos.double()[:, axis] * torch.tensor(freqs, dtype=torch.float64, device=DEV)
    want = amp * torch.stack([a.cos(), a.sin()], -1)
    bound = 2.0 ** -24 * want.abs() + 2.0 ** -50 * (1 + a.abs()[..., None]) * amp * 4
    assert ((table.double() - want).abs() <= bound).all()
    plain = torch.empty(T, pairs, 2, device=DEV)
    B.dvdq_rope_table(freqs, None, plain)
    a = torch.arange(T, dtype=torch.float64, device=DEV)[:, None] * torch.tensor(freqs, dtype=torch.float64, device=DEV)
    assert ((plain.double() - torch.stack([a.cos(), a.sin()], -1)).abs() <= 2.0 ** -24 + 2.0 ** -45).all()


# ------------------------------------------------------------------ host

def test_frequencies():
    f, a = B.dvdq_rope_frequencies(8, 100.0)
    assert a == 1.0 and all(math.isclose(x, y, rel_tol=1e-14) for x, y in zip(f, [1.0, 100 ** -0.25, 0.1, 100 ** -0.75]))
    g, a = B.dvdq_rope_frequencies(8, 100.0, B.ROPE_LINEAR, 4.0)
    assert a == 1.0 and all(math.isclose(x, y / 4, rel_tol=1e-14) for x, y in zip(g, f))
    g, a = B.dvdq_rope_frequencies(8, 100.0, B.ROPE_BASE, 4.0)
    assert a == 1.0 and g[0] == 1.0 and math.isclose(g[3], f[3] / 4, rel_tol=1e-12) and f[1] / 4 < g[1] < f[1]
    # by parts: over 4096 positions, pair i turns 4096 / (2 pi 10000^(i/32)) times
    f, _ = B.dvdq_rope_frequencies(64, 10000.0)
    g, a = B.dvdq_rope_frequencies(64, 10000.0, B.ROPE_BY_PARTS, 8.0, 4096.0, 32.0, 1.0)
    assert math.isclose(a, 0.1 * math.log(8.0) + 1.0)
    turns = [4096 * x / (2 * math.pi) for x in f]
    for i in range(32):
        if turns[i] > 40:
            assert g[i] == f[i]
        elif turns[i] < 0.7:
            assert math.isclose(g[i], f[i] / 8, rel_tol=1e-12)
        else:
            assert f[i] / 8 * 0.999999 <= g[i] <= f[i]
    assert g[0] == f[0] and sorted(g, reverse=True) == g
    for bad in (dict(rot_dim=3), dict(rot_dim=0), dict(rot_dim=514), dict(rot_dim=8, theta=0.0), dict(rot_dim=8, scaling=9),
                dict(rot_dim=8, scaling=1, factor=0.5), dict(rot_dim=8, scaling=3, factor=2.0), dict(rot_dim=2, scaling=2, factor=2.0),
                dict(rot_dim=8, theta=1.0, scaling=3, factor=2.0, original_length=4096.0, beta_fast=32.0, beta_slow=1.0),
                dict(rot_dim=8, theta=100.0, scaling=3, factor=2.0, original_length=float("inf"), beta_fast=32.0, beta_slow=1.0)):
        with pytest.raises(B.DvdqError):
            B.dvdq_rope_frequencies(**bad)


def rope(q=None, k=None, **kw):
    base = dict(x=4096, y=8192, heads=2, x_batch=640, x_token=128, x_head=64, y_batch=640, y_token=128, y_head=64)
    qt = None if q is None else B.RopeTensor(**{**base, **q})
    kt = None if k is None else B.RopeTensor(**{**base, **k})
    a = dict(B=2, S=5, D=64, rot=64, table=4096, rows=5, index=None, index_batch=0, layout=0, inverse=0, dtype=0, stream=None)
    a.update(kw)
    return B.load().dvdq_rope(qt, kt, *a.values())


@pytest.mark.parametrize("q,kw,status", [
    (None, {}, B.ERR_NULL), ({}, dict(D=0), B.ERR_SHAPE), ({}, dict(rot=66), B.ERR_SHAPE), ({}, dict(rot=31), B.ERR_SHAPE),
    ({}, dict(rot=0), B.ERR_SHAPE), ({}, dict(layout=2), B.ERR_UNSUPPORTED), ({}, dict(dtype=3), B.ERR_UNSUPPORTED),
    ({}, dict(table=None), B.ERR_NULL), ({}, dict(table=4100), B.ERR_ALIGN), ({}, dict(rows=4), B.ERR_SHAPE), ({}, dict(S=-1), B.ERR_SHAPE),
    (dict(heads=0), {}, B.ERR_SHAPE), (dict(x=None), {}, B.ERR_NULL), (dict(y=None), {}, B.ERR_NULL), (dict(x=4097), {}, B.ERR_ALIGN),
    (dict(y_head=0), {}, B.ERR_SHAPE), (dict(x_token=-128), {}, B.ERR_SHAPE), (dict(y=4096, y_token=256), {}, B.ERR_SHAPE),
    ({}, dict(S=0), B.OK), ({}, dict(B=0), B.OK)])
def test_rope_refuses(q, kw, status):
    assert rope(q, **kw) == status


def test_a_table_without_rows_is_refused():
    """A token whose row lies outside the table loads row 0 (and gets NaN): there has to be one."""
    assert rope({}, index=4096, rows=0) == B.ERR_SHAPE


def test_rope_table_refuses():
    f = (C.c_double * 4)(1, 1, 1, 1)
    call = B.load().dvdq_rope_table
    assert call(None, None, 4, None, 5, 1, 1.0, 4096, None) == B.ERR_NULL
    assert call(f, None, 0, None, 5, 1, 1.0, 4096, None) == B.ERR_SHAPE
    assert call(f, None, 257, None, 5, 1, 1.0, 4096, None) == B.ERR_SHAPE
    assert call(f, None, 4, None, 5, 3, 1.0, 4096, None) == B.ERR_NULL
    assert call(f, (C.c_int32 * 4)(0, 1, 2, 3), 4, 4096, 5, 3, 1.0, 4096, None) == B.ERR_SHAPE
    assert call(f, None, 4, None, 5, 1, 1.0, None, None) == B.ERR_NULL
    assert call(f, None, 4, None, 5, 1, 1.0, 4104, None) == B.ERR_ALIGN
    assert call(f, None, 4, None, 0, 1, 1.0, None, None) == B.OK

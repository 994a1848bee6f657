"""dvdq_linear_int8 against the formula in 64 bits (where its sums are exact).

Tolerances, element by element, with u the unit roundoff of the type (2^-8 bf16, 2^-11 fp16) and e = 2^-24:
  the sum over k is exact; its rounding to fp32, the scales' product and the fma onto the bias      3 e |acc s t| + e |z|
  activation in fp32                             slope <= 1.13 passes z's error on; ex2 / rcp add 2^-18 |z|
  the residual's addition e |y|, one rounding of the output u |y|, or half the smallest fp16 number
"""
import math

import pytest
import torch

from paper_2505_18663_b200 import binding as B

gpu = pytest.mark.gpu
DEV = "cuda"
DTYPES = [torch.bfloat16, torch.float16]
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
E = 2.0 ** -24


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def padded(r, c, dt, pitch=None):
    """[r, c] whose rows start on 16 bytes; what lies between rows is NaN (codes: 113), so that a read of it shows."""
    per = 16 // torch.empty(0, dtype=dt).element_size()
    return torch.full((r, pitch or -(-c // per) * per), 113 if dt == torch.int8 else float("nan"), dtype=dt, device=DEV)[:, :c]


def codes(r, c, g, pitch=None, lo=-128):
    t = padded(r, c, torch.int8, pitch)
    t.copy_(torch.randint(lo, 128, (r, c), device=DEV, generator=g, dtype=torch.int32))
    return t


def rows(r, c, dt, g, pitch=None, scale=1.0):
    t = padded(r, c, dt, pitch)
    t.copy_(torch.randn(r, c, device=DEV, generator=g) * scale)
    return t


def workspace(M, N, K):
    n = B.dvdq_linear_int8_workspace_bytes(M, N, K)
    return torch.full((n,), 255, dtype=torch.uint8, device=DEV) if n else None


def act64(z, act):
    if act == B.ACT_SILU:
        return z * torch.sigmoid(z)
    if act == B.ACT_GELU_TANH:
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def check(got, want, bound, what="y"):
    got = got.double()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = ((got - want).abs() - bound).max()
    assert float(over) <= 0, f"{what}: {float((got - want).abs().max()):.3e} off, {float(over):.3e} over the bound"


def status_ok():
    assert B.dvdq_last_device_status()[0] == B.OK


# one token; tiles and their edges (256 x 256 x 128); sizes that no piece divides; one column; long contractions (cut into pieces); many tiles
SIZES = [(1, 256, 256), (1, 1541, 1030), (7, 8, 8), (3, 1, 1), (8, 300, 700), (2, 9000, 2100), (5, 700, 5000), (9, 33, 3000), (16, 40, 64), (16, 9000, 40), (17, 255, 127), (33, 257, 129),
         (64, 1536, 1536), (128, 512, 4100), (129, 768, 3000), (256, 256, 128), (257, 264, 200), (300, 1000, 136), (1021, 1541, 515), (2500, 2300, 72),
         (6000, 1130, 130), (6000, 1130, 900)]


@gpu
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("act,bias,residual", [(0, False, False), (1, True, True), (2, True, False), (0, True, True), (2, False, True)])
def test_forward(dt, M, N, K, act, bias, residual):
    g = gen(M * 7 + N * 3 + K)
    a, w = codes(M, K, g), codes(N, K, g)
    s = torch.rand(M, device=DEV, generator=g) * 0.02
    t = torch.rand(N, device=DEV, generator=g) / (100 * math.sqrt(K))
    b = rows(1, N, dt, g)[0] if bias else None
    r = rows(M, N, dt, g, pitch=-(-N // 8) * 8 + 16) if residual else None
    y = padded(M, N, dt)
    B.dvdq_linear_int8(a, s, w, t, b, r, act, y, workspace(M, N, K))
    status_ok()
    scaled = (a.double() @ w.double().T) * (s.double()[:, None] * t.double())
    z = scaled + b.double() if bias else scaled
    y6 = act64(z, act)
    inner = 3 * E * scaled.abs() + E * z.abs()
    if act:
        inner = 1.13 * inner + 2.0 ** -18 * z.abs()
    if residual:
        y6 = y6 + r.double()
        inner = inner + E * (y6.abs() + inner)
    check(y, y6, inner + U[dt] * (y6.abs() + inner) + TINY[dt])


# up to 16 and up to 32 tokens without tiles: whole and partial groups of 8 tokens and of 16 channels, rows that end in any warp; and in tiles: short rows,
# many channels, rows too long for so few channels, 33 tokens
FEW = [(9, 1, 1), (10, 17, 63), (12, 2368, 1024), (13, 40, 5003), (15, 4736, 1090), (16, 4737, 1500), (16, 100, 16384), (10, 40, 16385), (16, 5000, 200), (9, 9600, 333), (14, 19000, 70), (16, 38000, 130),
       (17, 33, 65), (20, 2367, 1031), (24, 1540, 9237), (25, 171, 1024), (31, 1541, 515), (31, 1541, 1039), (32, 2368, 2100), (17, 2369, 1300), (32, 64, 9217), (33, 500, 1100)]


@gpu
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("M,N,K", FEW)
@pytest.mark.parametrize("act,bias,residual", [(0, False, False), (1, True, True), (2, False, True)])
def test_nine_to_thirty_three_tokens(dt, M, N, K, act, bias, residual):
    test_forward(dt, M, N, K, act, bias, residual)


@gpu
@pytest.mark.parametrize("N,K", [(520, 1100), (2304, 640), (6000, 300)])
def test_a_token_among_nine_to_forty_has_the_bits_it_has_alone(N, K):
    dt, g = torch.bfloat16, gen(N * 5 + K)
    a, w = codes(40, K, g), codes(N, K, g)
    s, t = torch.rand(40, device=DEV, generator=g) * 0.02, torch.rand(N, device=DEV, generator=g) / (100 * math.sqrt(K))
    alone = padded(40, N, dt)
    for m in range(40):
        B.dvdq_linear_int8(a[m:m + 1], s[m:m + 1], w, t, None, None, 1, alone[m:m + 1], workspace(1, N, K))
    for M in (9, 16, 17, 24, 32, 33, 40):
        y = padded(M, N, dt)
        B.dvdq_linear_int8(a[:M], s[:M], w, t, None, None, 1, y, workspace(M, N, K))
        assert torch.equal(y, alone[:M]), M
    status_ok()


@gpu
@pytest.mark.parametrize("M,N,K", [(1, 64, 131071), (5, 40, 131071), (40, 64, 131071), (300, 96, 131071)])
def test_the_longest_sums_do_not_wrap(M, N, K):
    """All codes -128 (and one row of 127): sums of up to 2^31 - 16384 in size."""
    a, w = padded(M, K, torch.int8).fill_(-128), padded(N, K, torch.int8).fill_(-128)
    w[1] = 127
    one = 2.0 ** -20
    y = padded(M, N, torch.bfloat16)
    B.dvdq_linear_int8(a, torch.full((M,), one, device=DEV), w, torch.ones(N, device=DEV), None, None, 0, y, workspace(M, N, K))
    want = torch.full((M, N), 16384 * K * one, dtype=torch.float64, device=DEV)
    want[:, 1] = -128 * 127 * K * one
    check(y, want, (U[torch.bfloat16] + 3 * E) * want.abs())
    status_ok()


@gpu
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("N,K", [(520, 1100), (96, 6000), (2304, 640)])
def test_a_row_does_not_depend_on_the_rows_beside_it(dt, N, K, act):
    """The kernel for few tokens, the tiles, their pieces along k and the widths of tiles give the same bits."""
    g = gen(N + K)
    M = 700
    a, w = codes(M, K, g), codes(N, K, g)
    s, t = torch.rand(M, device=DEV, generator=g) * 0.02, torch.rand(N, device=DEV, generator=g) / (100 * math.sqrt(K))
    b, r = rows(1, N, dt, g)[0], rows(M, N, dt, g)
    whole = padded(M, N, dt)
    B.dvdq_linear_int8(a, s, w, t, b, r, act, whole, workspace(M, N, K))
    for first, count in ((0, 1), (3, 7), (100, 8), (200, 9), (31, 40), (128, 130), (5, 400)):
        y = padded(count, N, dt)
        part = slice(first, first + count)
        B.dvdq_linear_int8(a[part], s[part], w, t, b, r[part], act, y, workspace(count, N, K))
        assert torch.equal(y, whole[part]), (first, count)
    status_ok()


@gpu
@pytest.mark.parametrize("M", [3, 40, 700])
def test_wide_pitches_and_a_residual_in_place(M):
    dt, N, K = torch.bfloat16, 136, 200
    g = gen(5)
    a, w = codes(M, K, g, pitch=K + 40), codes(N, K, g, pitch=K + 8)
    s, t = torch.rand(M, device=DEV, generator=g) * 0.01, torch.rand(N, device=DEV, generator=g) * 0.01
    y = rows(M, N, dt, g, pitch=N + 64)
    whole = torch.as_strided(y, (M, N + 64), (N + 64, 1))
    before = y.clone()
    B.dvdq_linear_int8(a, s, w, t, None, y, 0, y, workspace(M, N, K))
    scaled = (a.double() @ w.double().T) * (s.double()[:, None] * t.double())
    want = before.double() + scaled
    check(y, want, (U[dt] + 2 * E) * want.abs() + 4 * E * scaled.abs())
    assert whole[:, N:].isnan().all()   # what lies between rows is not written
    status_ok()


@gpu
@pytest.mark.parametrize("M", [2, 50])
def test_scales_that_are_not_finite_reach_their_row_or_channel_only(M):
    g = gen(6)
    N, K = 48, 72
    a, w = codes(M, K, g, lo=1), codes(N, K, g, lo=1)
    s, t = torch.ones(M, device=DEV), torch.full((N,), 1e-3, device=DEV)
    s[1], t[7] = float("nan"), float("inf")
    y = padded(M, N, torch.bfloat16)
    B.dvdq_linear_int8(a, s, w, t, None, None, 0, y, workspace(M, N, K))
    assert y[1].isnan().all()
    others, channels = [i for i in range(M) if i != 1], [i for i in range(N) if i != 7]
    assert (y[others, 7] == float("inf")).all() and y[others][:, channels].isfinite().all()


@gpu
def test_no_tokens_and_refusals_of_the_binding():
    g = gen(7)
    w, t = codes(24, 40, g), torch.ones(24, device=DEV)
    e, none = torch.empty(0, 40, dtype=torch.int8, device=DEV), torch.empty(0, device=DEV)
    B.dvdq_linear_int8(e, none, w, t, None, None, 0, torch.empty(0, 24, dtype=torch.float16, device=DEV))
    a, s, y = codes(4, 40, g), torch.ones(4, device=DEV), padded(4, 24, torch.float16)
    for bad in (lambda: B.dvdq_linear_int8(a.float(), s, w, t, None, None, 0, y), lambda: B.dvdq_linear_int8(a, s[:3], w, t, None, None, 0, y),
                lambda: B.dvdq_linear_int8(a, s, w[:, :39], t, None, None, 0, y), lambda: B.dvdq_linear_int8(a, s, w, t, t, None, 0, y),
                lambda: B.dvdq_linear_int8(a, s, w, t, None, None, 0, y.float()), lambda: B.dvdq_linear_int8(a, s.half(), w, t, None, None, 0, y),
                lambda: B.dvdq_linear_int8(a, s, w, t, None, y[:3], 0, y), lambda: B.dvdq_linear_int8(a, s, w, t.cpu(), None, None, 0, y)):
        with pytest.raises((TypeError, ValueError)):
            bad()
    with pytest.raises(B.DvdqError) as err:
        B.dvdq_linear_int8(a[:, :24], s, torch.empty(24, 24, dtype=torch.int8, device=DEV), t, None, None, 0, y)  # rows of 24 bytes
    assert err.value.status == B.ERR_ALIGN


def test_refusals_before_any_cuda_call():
    lib = B.load()
    one, two = 256, 512   # never dereferenced: validation fails first

    def call(M=20, N=16, K=32, a=one, s=one, lda=32, w=one, t=one, ldw=32, bias=0, r=0, ldr=16, act=0, y=two, ldy=16, dt=B.BF16, ws=0, room=0):
        return lib.dvdq_linear_int8(B.LINEAR_INT8_ARGS.pack(a or 0, lda, w or 0, ldw, s or 0, t or 0, bias, r, ldr, y or 0, ldy, M, N, K, ws, room, act, dt), None)

    assert lib.dvdq_linear_int8(None, None) == B.ERR_NULL
    assert call(M=-1) == call(N=0) == call(K=0) == call(K=131072, lda=131072, ldw=131072) == call(M=1 << 31) == call(N=(1 << 25) + 1, ldy=1 << 26) == B.ERR_SHAPE
    assert call(act=3) == call(dt=B.F32) == call(dt=-1) == B.ERR_UNSUPPORTED
    assert call(a=None) == call(w=None) == call(s=None) == call(t=None) == call(y=None) == B.ERR_NULL
    assert call(lda=16) == call(ldw=31) == call(ldy=8) == call(r=one, ldr=8) == call(r=two, ldr=24) == B.ERR_SHAPE
    assert call(lda=40) == call(ldw=33) == call(ldy=20) == call(a=8) == call(w=264) == call(y=520) == call(s=258) == call(bias=257) == B.ERR_ALIGN
    assert call(M=0, a=None, s=None, y=None) == B.OK
    need = B.dvdq_linear_int8_workspace_bytes(200, 256, 65536)
    assert need > 0 and need % 256 == 0
    long = dict(M=200, N=256, K=65536, lda=65536, ldw=65536, ldy=256)
    assert call(**long) == B.ERR_NULL and call(**long, ws=384, room=need) == B.ERR_ALIGN and call(**long, ws=one, room=need - 1) == B.ERR_WORKSPACE
    assert B.dvdq_linear_int8_workspace_bytes(4, 256, 65536) == 0 and B.dvdq_linear_int8_workspace_bytes(200, 256, 131072) == 0

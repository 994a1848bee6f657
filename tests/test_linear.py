"""dvdq_linear and dvdq_linear_backward against the formulas in 64 bits.

Tolerances, element by element, with u the unit roundoff of the type (2^-8 bf16, 2^-11 fp16):
  fp32 accumulation of K products in any order   (K + 8) 2^-23 sum |x||w|   (each add may truncate: one ulp, not half)
  activation in fp32                             slope <= 1.13 passes z's error on; ex2 / rcp add 2^-18 |z|
  one rounding of the output                     u |y|, or half the smallest fp16 number
  backward: dz is rounded to the type first      u sum |dz||w|
"""
import math

import pytest
import torch

from paper_2505_18663_b200 import binding as B

gpu = pytest.mark.gpu
DEV = "cuda"
DTYPES = [torch.bfloat16, torch.float16]
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


def rows(r, c, dt, g=None, scale=1.0, pitch=None, device=DEV):
    """[r, c] whose rows start on 16 bytes; what lies between rows is NaN, so that a read of it shows."""
    pitch = pitch or -(-c // 8) * 8
    t = torch.full((r, pitch), float("nan"), dtype=dt, device=device)
    v = t[:, :c]
    if g is not None:
        v.copy_(torch.randn(r, c, generator=g, device=device) * scale)
    return v


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def act64(z, act):
    if act == B.ACT_SILU:
        return z * torch.sigmoid(z)
    if act == B.ACT_GELU_TANH:
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def slope64(z, act):
    z = z.detach().clone().requires_grad_(True)
    with torch.enable_grad():
        act64(z, act).sum().backward()
    return z.grad


def workspace(n, fill=255):
    return torch.full((n,), fill, dtype=torch.uint8, device=DEV) if n else None


def check(got, want, bound, what):
    got = got.double()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = ((got - want).abs() - bound).max()
    assert float(over) <= 0, f"{what}: {float((got - want).abs().max()):.3e} off, {float(over):.3e} over the bound"


def status_ok():
    assert B.dvdq_last_device_status()[0] == B.OK


# sizes: one token; tiles and their edges (256 x 256 x 64); sizes that are no multiple of 8; one column;
# long contractions (cut into pieces); many tiles
FORWARD = [(1, 256, 256), (1, 1541, 1030), (7, 8, 8), (3, 1, 1), (16, 40, 64), (2, 100, 1537), (8, 300, 700), (9, 33, 3000), (5, 12000, 96), (16, 9000, 40), (17, 255, 63), (33, 257, 65), (128, 512, 4100),
           (256, 256, 64), (257, 264, 200), (300, 1000, 136), (129, 768, 3000), (1021, 1541, 515), (2500, 2300, 72),
           (6000, 1130, 130), (6000, 1130, 450)]


@gpu
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("M,N,K", FORWARD)
@pytest.mark.parametrize("act,bias,residual,save_z", [(0, False, False, False), (1, True, True, True), (2, True, False, True), (0, True, True, False),
                                                       (2, False, True, False)])
def test_forward(dt, M, N, K, act, bias, residual, save_z):
    g = gen(M * 7 + N * 3 + K)
    x, w = rows(M, K, dt, g), rows(N, K, dt, g, 1 / math.sqrt(K))
    b = rows(1, N, dt, g)[0] if bias else None
    r = rows(M, N, dt, g, pitch=-(-N // 8) * 8 + 16) if residual else None
    y, z = rows(M, N, dt), rows(M, N, dt) if save_z else None
    B.dvdq_linear(x, w, b, r, act, y, z, workspace(B.dvdq_linear_workspace_bytes(M, N, K)))
    status_ok()
    x6, w6 = x.double(), w.double()
    z6 = x6 @ w6.T
    acc = (K + 8) * 2.0 ** -23 * (x6.abs() @ w6.abs().T)
    if bias:
        z6 = z6 + b.double()
        acc = acc + 2.0 ** -23 * z6.abs()
    if save_z:
        check(z, z6, acc + U[dt] * z6.abs() * 1.001 + TINY[dt], "z")
    y6 = act64(z6, act)
    inner = 1.13 * acc + 2.0 ** -18 * z6.abs() * (act != 0)
    if residual:
        y6 = y6 + r.double()
        inner = inner + 2.0 ** -23 * y6.abs()
    check(y, y6, inner + U[dt] * (y6.abs() + inner) + TINY[dt], "y")


@gpu
def test_rows_with_wide_pitches_and_a_residual_in_place():
    dt, M, N, K = torch.bfloat16, 200, 136, 96
    g = gen(5)
    x, w = rows(M, K, dt, g, pitch=K + 40), rows(N, K, dt, g, 0.1, pitch=K + 8)
    y = rows(M, N, dt, g, pitch=N + 64)
    whole = torch.as_strided(y, (M, N + 64), (N + 64, 1))
    before = y.clone()
    B.dvdq_linear(x, w, None, y, 0, y, None, workspace(B.dvdq_linear_workspace_bytes(M, N, K)))
    want = before.double() + x.double() @ w.double().T
    check(y, want, 2.0 ** -8 * want.abs() + (K + 9) * 2.0 ** -23 * (x.double().abs() @ w.double().abs().T + want.abs()), "y")
    assert whole[:, N:].isnan().all()   # what lies between rows is not written
    status_ok()


@gpu
def test_infinities_and_nan_reach_their_row_only():
    dt, M, N, K = torch.bfloat16, 40, 48, 72
    g = gen(6)
    x, w, y = rows(M, K, dt, g), rows(N, K, dt, g), rows(M, N, dt)
    x[3, 5], x[9, 0] = float("nan"), float("inf")
    B.dvdq_linear(x, w, None, None, 0, y, None, workspace(B.dvdq_linear_workspace_bytes(M, N, K)))
    assert y[3].isnan().all() and not y[9].isfinite().any()
    rest = [i for i in range(M) if i not in (3, 9)]
    assert y[rest].isfinite().all()


@gpu
def test_no_tokens():
    dt = torch.float16
    g = gen(7)
    w = rows(24, 40, dt, g)
    e = torch.empty(0, 40, dtype=dt, device=DEV)
    B.dvdq_linear(e, w, None, None, 0, torch.empty(0, 24, dtype=dt, device=DEV))
    dw, db = rows(24, 40, dt, g), torch.ones(24, device=DEV)
    B.dvdq_linear_backward(torch.empty(0, 24, dtype=dt, device=DEV), None, e, w, 0, None, dw, db, None)
    assert (dw == 0).all() and (db == 0).all()


@gpu
def test_the_same_bits_every_time_and_on_another_stream():
    dt, M, N, K = torch.bfloat16, 100, 300, 5000   # cut into pieces
    assert B.dvdq_linear_workspace_bytes(M, N, K) > 0
    g = gen(8)
    x, w, y, y2 = rows(M, K, dt, g), rows(N, K, dt, g), rows(M, N, dt), rows(M, N, dt)
    ws = workspace(B.dvdq_linear_workspace_bytes(M, N, K))
    B.dvdq_linear(x, w, None, None, 1, y, None, ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    B.dvdq_linear(x, w, None, None, 1, y2, None, ws, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(y, y2)


BACKWARD = [(1, 64, 72), (1, 1541, 1030), (5, 8, 8), (2, 1, 3), (3, 700, 1100), (4, 257, 130), (16, 90, 2500), (17, 129, 65), (64, 256, 256), (65, 255, 130), (300, 264, 200), (1021, 515, 258), (4100, 72, 64),
            (700, 2100, 1100), (4200, 130, 1200), (200, 2600, 1100)]


@gpu
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("M,N,K", BACKWARD)
@pytest.mark.parametrize("act", [0, 1, 2])
def test_backward(dt, M, N, K, act):
    g = gen(M + N + K)
    dy, x, w = rows(M, N, dt, g), rows(M, K, dt, g), rows(N, K, dt, g, 1 / math.sqrt(K))
    z = rows(M, N, dt, g, 2.0) if act else None
    dx, dw, db = rows(M, K, dt), rows(N, K, dt), torch.full((N,), float("nan"), device=DEV)
    ws = workspace(B.dvdq_linear_backward_workspace_bytes(M, N, K, act))
    B.dvdq_linear_backward(dy, z, x, w, act, dx, dw, db, ws)
    status_ok()
    dz = dy.double() * (slope64(z.double(), act) if act else 1.0)
    x6, w6, a = x.double(), w.double(), dz.abs()
    # dz: fp32 slope (ex2 / rcp: 2^-18 of |dy| |z|), then one rounding; its smallest fp16 step counts as well
    rough = (U[dt] * a + TINY[dt] + 2.0 ** -18 * dy.double().abs() * (1 + z.double().abs()) * 1.2) if act else torch.zeros_like(a)
    for name, got, want, spread, terms, mag in (
            ("dx", dx, dz @ w6, rough @ w6.abs(), N, a @ w6.abs()), ("dw", dw, dz.T @ x6, rough.T @ x6.abs(), M, a.T @ x6.abs())):
        inner = spread * 1.01 + (terms + 8) * 2.0 ** -23 * mag
        check(got, want, inner + U[dt] * (want.abs() + inner) + TINY[dt], name)
    exact_dz = 2.0 ** -18 * dy.double().abs() * (1 + z.double().abs()) * 1.2 if act else torch.zeros_like(a)
    check(db, dz.sum(0), exact_dz.sum(0) + (M + 8) * 2.0 ** -24 * a.sum(0), "db")


@gpu
def test_each_gradient_alone_is_the_same():
    dt, M, N, K = torch.bfloat16, 130, 200, 72
    g = gen(11)
    dy, x, w, z = rows(M, N, dt, g), rows(M, K, dt, g), rows(N, K, dt, g), rows(M, N, dt, g)
    ws = workspace(B.dvdq_linear_backward_workspace_bytes(M, N, K, 2))
    full = rows(M, K, dt), rows(N, K, dt), torch.empty(N, device=DEV)
    B.dvdq_linear_backward(dy, z, x, w, 2, *full, ws)
    dx, dw, db = rows(M, K, dt), rows(N, K, dt), torch.empty(N, device=DEV)
    B.dvdq_linear_backward(dy, z, None, w, 2, dx, None, None, ws)
    B.dvdq_linear_backward(dy, z, x, None, 2, None, dw, None, ws)
    B.dvdq_linear_backward(dy, z, None, None, 2, None, None, db, workspace(B.dvdq_linear_backward_workspace_bytes(M, N, 8, 2)))
    assert torch.equal(dx, full[0]) and torch.equal(dw, full[1]) and torch.equal(db, full[2])


@gpu
def test_gradients_against_differences():
    """f = sum of c * y over the forward call's own (fp16) outputs: a central difference along a random direction of x
    and of w.  Steps of 1/4 on entries of about 1 make the products' change exact to about 2^-11 relative per entry;
    summed over M N = 2304 entries with random signs, 2 % of the difference is ten times what rounding leaves."""
    dt, M, N, K, act = torch.float16, 48, 48, 64, B.ACT_SILU
    g = gen(12)
    x, w = rows(M, K, dt, g), rows(N, K, dt, g, 0.25)
    c = rows(M, N, dt, g)
    y, z = rows(M, N, dt), rows(M, N, dt)

    def forward(xx, ww):
        B.dvdq_linear(xx, ww, None, None, act, y, z, workspace(B.dvdq_linear_workspace_bytes(M, N, K)))
        return float((y.double() * c.double()).sum())

    forward(x, w)
    dx, dw = rows(M, K, dt), rows(N, K, dt)
    B.dvdq_linear_backward(c, z.clone(), x, w, act, dx, dw, None, workspace(B.dvdq_linear_backward_workspace_bytes(M, N, K, act)))
    for t, grad, step in ((x, dx, 2.0 ** -5), (w, dw, 2.0 ** -7)):
        d = torch.sign(grad.float()).to(dt)     # every entry counts the same way: no cancellation
        up, down = (t + d * step).to(dt), (t - d * step).to(dt)
        diff = forward(up, w) - forward(down, w) if t is x else forward(x, up) - forward(x, down)
        want = float((grad.double() * (up.double() - down.double())).sum())
        assert abs(diff - want) <= 0.02 * abs(want), (diff, want)


# ------------------------------------------------------------------ refusals (no GPU needed)

P = 4096  # an address that is never dereferenced: the call is refused first


def linear(**k):
    a = dict(X=P, M=10, ldx=64, W=P, N=32, K=64, ldw=64, bias=None, R=None, ldr=0, act=0, Y=P, ldy=32, Z=None, ldz=0, dtype=0, ws=None, n=0,
             stream=None)
    a.update(k)
    return B.load().dvdq_linear(*a.values())


def backward(**k):
    a = dict(dY=P, lddy=32, Z=P, ldz=32, X=P, ldx=64, W=P, ldw=64, M=10, N=32, K=64, act=1, dX=P, lddx=64, dW=P, lddw=64, db=P, dtype=0, ws=P,
             n=1 << 30, stream=None)
    a.update(k)
    return B.load().dvdq_linear_backward(*a.values())


@pytest.mark.parametrize("change,status", [
    (dict(M=-1), B.ERR_SHAPE), (dict(N=0), B.ERR_SHAPE), (dict(K=0), B.ERR_SHAPE), (dict(K=1 << 31), B.ERR_SHAPE),
    (dict(act=3), B.ERR_UNSUPPORTED), (dict(act=-1), B.ERR_UNSUPPORTED), (dict(dtype=2), B.ERR_UNSUPPORTED), (dict(dtype=7), B.ERR_UNSUPPORTED),
    (dict(X=None), B.ERR_NULL), (dict(W=None), B.ERR_NULL), (dict(Y=None), B.ERR_NULL),
    (dict(ldx=63), B.ERR_SHAPE), (dict(ldw=60), B.ERR_SHAPE), (dict(ldx=65), B.ERR_ALIGN), (dict(ldy=36), B.ERR_ALIGN),
    (dict(X=P + 2), B.ERR_ALIGN), (dict(Y=P + 8), B.ERR_ALIGN), (dict(bias=P + 1), B.ERR_ALIGN), (dict(R=P, ldr=31), B.ERR_SHAPE),
    (dict(R=P, ldr=33), B.ERR_ALIGN), (dict(R=P, ldr=40), B.ERR_SHAPE), (dict(Z=P, ldz=8), B.ERR_SHAPE), (dict(Z=P + 4, ldz=32), B.ERR_ALIGN),
    (dict(M=20, K=6400, ldx=6400, ldw=6400), B.ERR_NULL), (dict(M=20, K=6400, ldx=6400, ldw=6400, ws=P, n=16), B.ERR_WORKSPACE),
    (dict(M=20, K=6400, ldx=6400, ldw=6400, ws=P + 16, n=1 << 30), B.ERR_ALIGN), (dict(M=0, X=None, Y=None, W=None), B.OK)])
def test_linear_refuses(change, status):
    assert linear(**change) == status


@pytest.mark.parametrize("change,status", [
    (dict(M=-1), B.ERR_SHAPE), (dict(act=5), B.ERR_UNSUPPORTED), (dict(dtype=2), B.ERR_UNSUPPORTED), (dict(dY=None), B.ERR_NULL),
    (dict(Z=None), B.ERR_NULL), (dict(X=None), B.ERR_NULL), (dict(W=None), B.ERR_NULL), (dict(ws=None), B.ERR_NULL),
    (dict(n=100), B.ERR_WORKSPACE), (dict(ws=P + 8), B.ERR_ALIGN), (dict(lddy=30), B.ERR_SHAPE), (dict(lddx=65), B.ERR_ALIGN),
    (dict(dW=P + 2), B.ERR_ALIGN), (dict(db=P + 2), B.ERR_ALIGN)])
def test_backward_refuses(change, status):
    assert backward(**change) == status


def test_sizes_of_workspaces():
    assert B.dvdq_linear_workspace_bytes(0, 64, 64) == 0 and B.dvdq_linear_workspace_bytes(-1, 64, 64) == 0
    assert B.dvdq_linear_workspace_bytes(32760, 1536, 1536) == 0          # more tiles than CTA pairs: nothing is cut
    n = B.dvdq_linear_workspace_bytes(20, 32, 6400)
    assert n > 0 and n % 256 == 0
    a, b = (B.dvdq_linear_backward_workspace_bytes(1000, 512, 512, k) for k in (0, 1))
    assert b >= a + 1000 * 512 * 2


def test_the_binding_refuses_what_is_no_cuda_matrix():
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        B.dvdq_linear(x, x, None, None, 0, x)
    with pytest.raises(TypeError):
        B.dvdq_linear(x.float(), x, None, None, 0, x)
    with pytest.raises(TypeError):
        B.dvdq_linear(x[:, ::2], x, None, None, 0, x)


@gpu
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("M,N,K", [(1, 70, 300), (3, 151, 1090), (16, 64, 90), (17, 130, 72), (32, 600, 200), (17, 73, 79), (63, 64, 300), (300, 13, 40)])
def test_gradients_of_few_tokens_do_not_round_dz(dt, M, N, K):
    """Up to 32 tokens, and in small layers, the gradients are formed from dz in two parts (what is left after both is below
    u^2 |dz|, or half the smallest fp16 step), or from fp32: one rounding of the result, as if dz were exact."""
    g = gen(N)
    dy, x, w, z = rows(M, N, dt, g), rows(M, K, dt, g), rows(N, K, dt, g), rows(M, N, dt, g, 2.0)
    dx, dw = rows(M, K, dt), rows(N, K, dt)
    B.dvdq_linear_backward(dy, z, x, w, B.ACT_SILU, dx, dw, None, workspace(B.dvdq_linear_backward_workspace_bytes(M, N, K, B.ACT_SILU)))
    dz = dy.double() * slope64(z.double(), B.ACT_SILU)
    fine = 2.0 ** -18 * dy.double().abs() * (1 + z.double().abs()) * 1.2 + U[dt] ** 2 * dz.abs() + TINY[dt]
    outs = [(dx, dz @ w.double(), fine @ w.double().abs(), 2 * N, dz.abs() @ w.double().abs()),
            (dw, dz.T @ x.double(), fine.T @ x.double().abs(), 2 * M, dz.abs().T @ x.double().abs())]
    for got, want, spread, terms, mag in outs:
        inner = spread + (terms + 8) * 2.0 ** -23 * mag
        check(got, want, inner + U[dt] * (want.abs() + inner) + TINY[dt], "gradient")


@gpu
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("M,N,K", [(5, 40, 72), (20, 130, 96)])
def test_an_infinite_gradient_stays_in_its_token_and_channel(dt, M, N, K):
    """Nothing is left of an infinity to round, and no row of dz's second part reaches a sum that it does not belong to."""
    g = gen(N + 1)
    dy, x, w, z = rows(M, N, dt, g), rows(M, K, dt, g), rows(N, K, dt, g), rows(M, N, dt, g)
    dy[2, 3], z[2, 3] = float("inf"), 1.0
    dx, dw, db = rows(M, K, dt), rows(N, K, dt), torch.empty(N, device=DEV)
    B.dvdq_linear_backward(dy, z, x, w, B.ACT_SILU, dx, dw, db, workspace(B.dvdq_linear_backward_workspace_bytes(M, N, K, B.ACT_SILU)))
    status_ok()
    assert torch.equal(dx[2].float(), torch.sign(w[3].float()) * math.inf) and torch.equal(dw[3].float(), torch.sign(x[2].float()) * math.inf)
    assert dx[[i for i in range(M) if i != 2]].isfinite().all() and dw[[i for i in range(N) if i != 3]].isfinite().all()
    assert db[3] == math.inf and db[[i for i in range(N) if i != 3]].isfinite().all()


# layers whose own workspace is smaller than the one of the same tokens and channels with a K of 8
LAYERS = [(1021, 1541, 1030, 0), (4096, 4096, 4096, 0), (4096, 4096, 4096, 1), (8192, 5120, 5120, 0), (100, 300, 5000, 2)]


@pytest.mark.parametrize("M,N,K,act", LAYERS)
def test_a_bias_gradient_alone_needs_no_more_than_the_layer(M, N, K, act):
    """Sized for the layer, with a K of 8 in the call: refused here for want of a GPU, not for want of room."""
    n = B.dvdq_linear_backward_workspace_bytes(M, N, K, act)
    need = dict(M=M, N=N, K=8, lddy=-(-N // 8) * 8, ldz=-(-N // 8) * 8, act=act, X=None, W=None, dX=None, dW=None, n=n)
    if not torch.cuda.is_available():  # (these addresses are for no GPU)
        assert backward(**need) not in (B.OK, B.ERR_WORKSPACE)
    assert backward(**dict(need, n=M)) == B.ERR_WORKSPACE


@gpu
@pytest.mark.parametrize("M,N,K,act", LAYERS)
def test_a_bias_gradient_alone(M, N, K, act):
    g = gen(M)
    dt = torch.bfloat16
    dy, z = rows(M, N, dt, g), rows(M, N, dt, g) if act else None
    db = torch.empty(N, device=DEV)
    B.dvdq_linear_backward(dy, z, None, None, act, None, None, db, workspace(B.dvdq_linear_backward_workspace_bytes(M, N, K, act)))
    dz = dy.double() * (slope64(z.double(), act) if act else 1.0)
    rough = 2.0 ** -18 * dy.double().abs() * (1 + z.double().abs()) * 1.2 if act else torch.zeros_like(dz)
    check(db, dz.sum(0), rough.sum(0) + (M + 8) * 2.0 ** -24 * dz.abs().sum(0), "db")


@gpu
@pytest.mark.parametrize("M", [1, 4, 5, 20])
@pytest.mark.parametrize("act", [1, 2])
def test_slopes_far_below_zero(M, act):
    """Where the slope of the activation is small but a large dy still makes something of it (in bf16; fp16 has no such range).
    The slope is right to |z| 2^-22 of itself, what two parts of dz leave to 2^-15, the output to 2^-8: 2^-7 of sum |dz||x| holds
    them all."""
    dt, N, K = torch.bfloat16, 72, 40
    g = gen(M)
    x, w, dy, z = rows(M, K, dt, g), rows(N, K, dt, g), rows(M, N, dt), rows(M, N, dt)
    dy.fill_(2.0 ** 15)
    far = 6.0 if act == 1 else 60.0
    z.copy_(-torch.linspace(far / 6, far, N, device=DEV).expand(M, N))
    dw, db = rows(N, K, dt), torch.empty(N, device=DEV)
    B.dvdq_linear_backward(dy, z, x, w, act, None, dw, db, workspace(B.dvdq_linear_backward_workspace_bytes(M, N, K, act)))
    z6 = z.double()
    u, du = (z6, torch.ones_like(z6)) if act == 2 else (2 * math.sqrt(2 / math.pi) * (z6 + 0.044715 * z6 ** 3),
                                                       2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z6 ** 2))
    f = torch.sigmoid(u)   # 1 + tanh would cancel here
    dz = dy.double() * (f + z6 * du * f * (1 - f))
    mag = dz.abs().T @ x.double().abs()
    check(dw, dz.T @ x.double(), 2.0 ** -7 * mag, "dw")
    check(db, dz.sum(0), 2.0 ** -14 * dz.abs().sum(0), "db")


@gpu
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("M,N,K", [(1, 40, 72), (3, 40, 72), (5, 40, 72), (20, 130, 96), (63, 64, 300), (300, 13, 40)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_infinities_in_the_other_operand_of_the_gradients(dt, M, N, K, sign):
    """w and x with an infinity each: what it is multiplied with decides its sign, whether dz comes whole or in two parts (one dz
    here is a power of two, which is its own first part)."""
    g = gen(N + 1)
    dy, x, w, z = rows(M, N, dt, g), rows(M, K, dt, g), rows(N, K, dt, g), rows(M, N, dt, g)
    dy[0, 3], z[0, 3] = 0.5, 0.0    # dz = 0.25
    w[3, 5], x[M // 2, 7] = sign * math.inf, sign * math.inf
    dx, dw = rows(M, K, dt), rows(N, K, dt)
    B.dvdq_linear_backward(dy, z, x, w, B.ACT_SILU, dx, dw, None, workspace(B.dvdq_linear_backward_workspace_bytes(M, N, K, B.ACT_SILU)))
    dz = dy.double() * slope64(z.double(), B.ACT_SILU)
    assert torch.equal(dx[:, 5].double(), torch.sign(dz[:, 3]) * sign * math.inf)
    assert torch.equal(dw[:, 7].double(), torch.sign(dz[M // 2]) * sign * math.inf)
    assert dx[:, [c for c in range(K) if c != 5]].isfinite().all() and dw[:, [c for c in range(K) if c != 7]].isfinite().all()


@gpu
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("M,N,K", [(1024, 4, 200), (5000, 16, 130), (2000, 1, 64), (700, 32, 300)])
def test_gradients_of_few_channels_do_not_round_dz(dt, M, N, K):
    """dX sums over channels: with up to 32 of them it has one rounding of the result too, however many tokens there are, and so has dW."""
    g = gen(N)
    dy, x, w, z = rows(M, N, dt, g), rows(M, K, dt, g), rows(N, K, dt, g), rows(M, N, dt, g, 2.0)
    dx, dw = rows(M, K, dt), rows(N, K, dt)
    B.dvdq_linear_backward(dy, z, x, w, B.ACT_SILU, dx, dw, None, workspace(B.dvdq_linear_backward_workspace_bytes(M, N, K, B.ACT_SILU)))
    dz = dy.double() * slope64(z.double(), B.ACT_SILU)
    fine = 2.0 ** -18 * dy.double().abs() * (1 + z.double().abs()) * 1.2 + U[dt] ** 2 * dz.abs() + TINY[dt]
    outs = [(dx, dz @ w.double(), fine @ w.double().abs(), 2 * N, dz.abs() @ w.double().abs()),
            (dw, dz.T @ x.double(), fine.T @ x.double().abs(), 2 * M, dz.abs().T @ x.double().abs())]
    for got, want, spread, terms, mag in outs:
        inner = spread + (terms + 8) * 2.0 ** -23 * mag
        check(got, want, inner + U[dt] * (want.abs() + inner) + TINY[dt], "gradient")
    status_ok()

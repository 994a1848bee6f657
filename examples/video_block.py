"""One block of a video transformer and one block of its latent decoder, forward and a training step, on the C ABI.

    python examples/video_block.py [frames height width]        (patches; default 3 12 20)

Transformer block: modulation from one conditioning vector (dvdq_linear, one token), fused projection with 4-bit weights and
4-bit activations (dvdq_qlinear), rotary positions over (frame, row, column) in place on the projection's output
(dvdq_rope), attention (torch), output projection added onto the residual stream (dvdq_linear), and the gradients of that
projection (dvdq_linear_backward, dvdq_rope with inverse=True).  Decoder block: group norm with SiLU, a 1x1
convolution as a linear layer with residual, and their gradients (dvdq_group_norm, dvdq_linear).  Every step is compared with the
same formula in fp32; the worst relative errors are returned.
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2505_18663_b200 import binding as B  # noqa: E402
from paper_2505_18663_b200 import workloads as W  # noqa: E402

DEV, DT = "cuda", torch.bfloat16


def rel(got, want):
    return float((got.float() - want).norm() / want.norm())


def linear(x, w, bias=None, residual=None, act=B.ACT_NONE, keep_z=False):
    y = torch.empty(x.shape[0], w.shape[0], dtype=x.dtype, device=DEV)
    z = torch.empty_like(y) if keep_z else None
    need = B.dvdq_linear_workspace_bytes(x.shape[0], w.shape[0], x.shape[1])
    ws = torch.empty(need, dtype=torch.uint8, device=DEV) if need else None
    B.dvdq_linear(x, w, bias, residual, act, y, z, ws)
    return (y, z) if keep_z else y


def linear_backward(dy, z, x, w, act):
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(w.shape[0], device=DEV)
    ws = torch.empty(B.dvdq_linear_backward_workspace_bytes(x.shape[0], w.shape[0], x.shape[1], act), dtype=torch.uint8, device=DEV)
    B.dvdq_linear_backward(dy, z, x, w, act, dx, dw, db, ws)
    return dx, dw, db


def randn(*shape, scale=1.0, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(*shape, generator=g, device=DEV) * scale).to(DT)


def transformer_block(frames, height, width, dim=256, heads=4):
    T, D = frames * height * width, dim // heads
    errors = {}
    # modulation: shift, scale and gate from one conditioning vector
    c, wm = randn(1, dim, seed=1), randn(3 * dim, dim, scale=dim ** -0.5, seed=2)
    m = linear(c, wm, act=B.ACT_SILU)
    errors["modulation"] = rel(m, torch.nn.functional.silu(c.float() @ wm.float().T))
    shift, scale, gate = m.view(3, dim)
    h = randn(T, dim, seed=3)
    x = (torch.nn.functional.layer_norm(h.float(), (dim,)) * (1 + scale.float()) + shift.float()).to(DT)

    # fused projection: 4-bit weights, 4-bit rotated activations
    layer = W.Layer(K=dim, N=3 * dim, rot_block=256, bits=4)
    u, d, z = W.make_weight_codes(layer, seed=4, device=DEV)
    blob = torch.empty(B.dvdq_weight_blob_bytes(layer.N, layer.K), dtype=torch.uint8, device=DEV)
    qw = B.dvdq_pack_weights(u, d, z, layer.rot_block, blob)
    q = B.ActQuant(layer.bits, layer.rot_block, 0, 8)
    ws = torch.empty(B.dvdq_qlinear_workspace_bytes(T, dim, q), dtype=torch.uint8, device=DEV)
    qkv = torch.empty(T, 3 * dim, dtype=DT, device=DEV)
    B.dvdq_qlinear(x, q, qw, None, 0, qkv, ws)

    # rotary positions, in place on the projection's output: a third of the pairs for each axis
    pairs = D // 2
    freqs, amplitude = B.dvdq_rope_frequencies(D)
    axis = [min(2, 3 * i // pairs) for i in range(pairs)]
    n = torch.arange(T, device=DEV)
    positions = torch.stack([n // (height * width), n // width % height, n % width], 1).to(torch.int32).contiguous()
    table = torch.empty(T, pairs, 2, device=DEV)
    B.dvdq_rope_table(freqs, positions, table, axis, amplitude)
    heads_view = qkv.view(1, T, 3, heads, D)
    qh, kh, vh = heads_view.unbind(2)
    angle = positions.double()[:, axis] * torch.tensor(freqs, dtype=torch.float64, device=DEV)
    turn = torch.polar(torch.ones_like(angle), angle)[None, :, None]
    wants = [torch.view_as_real(torch.view_as_complex(t.double().contiguous().unflatten(-1, (pairs, 2))) * turn).flatten(-2).float() for t in (qh, kh)]
    B.dvdq_rope(qh, kh, table, None, B.ROPE_PAIRS, False, qh, kh)
    errors["rope"] = max(rel(qh, wants[0]), rel(kh, wants[1]))

    a = torch.nn.functional.scaled_dot_product_attention(*(t.transpose(1, 2) for t in (qh, kh, vh))).transpose(1, 2).reshape(T, dim)

    # output projection onto the residual stream
    wo, bo = randn(dim, dim, scale=dim ** -0.5, seed=5), randn(dim, scale=0.1, seed=6)
    out = linear(a, wo, bo, residual=h)
    errors["out projection"] = rel(out, a.float() @ wo.float().T + bo.float() + h.float())

    # its gradients, and those of the rotated queries back through the rotation
    dy = randn(T, dim, seed=7)
    da, dw, db = linear_backward(dy, None, a, wo, B.ACT_NONE)
    errors["out projection gradients"] = max(rel(da, dy.float() @ wo.float()), rel(dw, dy.float().T @ a.float()), rel(db, dy.float().sum(0)))
    dq = da.view(1, T, heads, D)
    back = torch.empty_like(dq)
    B.dvdq_rope(dq, None, table, None, B.ROPE_PAIRS, True, back)
    want = torch.view_as_real(torch.view_as_complex(dq.double().unflatten(-1, (pairs, 2))) * turn.conj()).flatten(-2).float()
    errors["rope gradient"] = rel(back, want)
    return errors


def decoder_block(frames, height, width, channels=128, groups=32):
    S = frames * height * width * 4
    errors = {}
    x, gamma, beta = randn(1, S, channels, seed=8), randn(channels, seed=9), randn(channels, seed=10)
    w, b = randn(channels, channels, scale=channels ** -0.5, seed=11), randn(channels, scale=0.1, seed=12)
    n = torch.empty_like(x)
    mean, rstd = torch.empty(1, groups, device=DEV), torch.empty(1, groups, device=DEV)
    ws = torch.empty(B.dvdq_group_norm_workspace_bytes(1, S, channels, groups), dtype=torch.uint8, device=DEV)
    B.dvdq_group_norm(x, groups, gamma, beta, 1e-6, B.ACT_SILU, n, mean, rstd, ws)
    y = linear(n[0], w, b, residual=x[0])

    # the same in fp32, with torch's gradients
    xf, gf, bf, wf, cf = (t.float().requires_grad_(True) for t in (x, gamma, beta, w, b))
    nf = torch.nn.functional.silu(torch.nn.functional.group_norm(xf.transpose(1, 2), groups, gf, bf, 1e-6).transpose(1, 2))
    yf = nf[0] @ wf.T + cf + xf[0]
    errors["group norm"], errors["decoder block"] = rel(n, nf.detach()), rel(y, yf.detach())

    dy = randn(S, channels, seed=13)
    yf.backward(dy.float())
    dn, dw, db = linear_backward(dy, None, n[0], w, B.ACT_NONE)
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty(channels, device=DEV), torch.empty(channels, device=DEV)
    B.dvdq_group_norm_backward(dn.view(1, S, channels), x, mean, rstd, groups, gamma, beta, B.ACT_SILU, dx, dgamma, dbeta, ws)
    errors["decoder gradients"] = max(rel(dx.float() + dy.float(), xf.grad), rel(dw, wf.grad), rel(db, cf.grad), rel(dgamma, gf.grad),
                                      rel(dbeta, bf.grad))
    return errors


def main(frames=3, height=12, width=20):
    errors = {**transformer_block(frames, height, width), **decoder_block(frames, height, width)}
    status, detail = B.dvdq_last_device_status()
    if status != B.OK:
        raise B.DvdqError(status, f"device status (detail {detail})")
    return errors


if __name__ == "__main__":
    for name, e in main(*(int(a) for a in sys.argv[1:4])).items():
        print(f"{name:28s} relative error against fp32 {e:.2e}")

"""A feed-forward block whose two layers are in 8 bits, and the norms of queries and keys, on the C ABI; with the norm's gradients.

    python examples/int8_block.py [tokens]        (default 700)

Block: the residual stream takes the attention's output and is normalised into 8-bit codes in one call (dvdq_rms_norm), the up layer with GELU
(dvdq_linear_int8), its output in 8 bits row by row (dvdq_quantize_rows), the down layer added onto the residual stream in place
(dvdq_linear_int8).  Weights: rows in 8 bits, a scale for each output channel (dvdq_quantize_rows).  Queries and keys: each head
normalised where it lies in a fused projection's output (dvdq_rms_norm), then rotated (dvdq_rope).  A training step through the norm: dvdq_rms_norm_backward.
Every step is compared with the same formula in fp64; the worst relative errors are returned.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2505_18663_b200 import binding as B  # noqa: E402

DEV, DT, EPS = "cuda", torch.bfloat16, 1e-6


def rel(got, want):
    return float((got.double() - want).norm() / want.norm())


def randn(*shape, scale=1.0, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(*shape, generator=g, device=DEV) * scale).to(DT)


def codes_for(rows, channels):
    """Room for rows in 8 bits: each starts on 16 bytes, as dvdq_linear_int8 wants them."""
    return torch.empty(rows, -(-channels // 16) * 16, dtype=torch.int8, device=DEV)[:, :channels], torch.empty(rows, device=DEV)


def quantized(x):
    codes, scales = codes_for(*x.shape)
    B.dvdq_quantize_rows(x, codes, scales)
    return codes, scales


def linear_int8(x, w, bias, out, residual=None, act=B.ACT_NONE):
    need = B.dvdq_linear_int8_workspace_bytes(x[0].shape[0], w[0].shape[0], x[0].shape[1])
    ws = torch.empty(need, dtype=torch.uint8, device=DEV) if need else None
    B.dvdq_linear_int8(*x, *w, bias, residual, act, out, ws)
    return out


def values(codes_and_scales):
    return codes_and_scales[0].double() * codes_and_scales[1].double()[:, None]


def rms64(h, gamma):
    return h * (h.square().mean(-1, keepdim=True) + EPS).rsqrt() * gamma.double()


def feed_forward(tokens, dim=320, inner=1000):
    errors = {}
    stream, attention = randn(tokens, dim, seed=1), randn(tokens, dim, seed=2)
    gamma, up, down = randn(dim, seed=3), randn(inner, dim, scale=dim ** -0.5, seed=4), randn(dim, inner, scale=inner ** -0.5, seed=5)
    b_up, b_down = randn(inner, scale=0.1, seed=6), randn(dim, scale=0.1, seed=7)
    w_up, w_down = quantized(up), quantized(down)
    errors["weights in 8 bits"] = max(rel(values(w_up), up.double()), rel(values(w_down), down.double()))

    want_h = stream.double() + attention.double()
    codes, scales = codes_for(tokens, dim)
    B.dvdq_rms_norm(stream, attention, gamma, EPS, H=stream, codes=codes, scales=scales)   # the stream in place
    want_y = rms64(want_h, gamma)
    errors["residual stream"], errors["norm in 8 bits"] = rel(stream, want_h), rel(values((codes, scales)), want_y)

    hidden = linear_int8((codes, scales), w_up, b_up, torch.empty(tokens, inner, dtype=DT, device=DEV), act=B.ACT_GELU_TANH)
    z = values((codes, scales)) @ values(w_up).T + b_up.double()
    errors["up"] = rel(hidden, torch.nn.functional.gelu(z, approximate="tanh"))
    q = quantized(hidden)
    want = values(q) @ values(w_down).T + b_down.double() + stream.double()
    linear_int8(q, w_down, b_down, stream, residual=stream)
    errors["down onto the stream"] = rel(stream, want)
    # the block against the same block in full precision: three roundings to 8 bits, each half a step of a row's largest value over 127
    exact = torch.nn.functional.gelu(want_y @ up.double().T + b_up.double(), approximate="tanh") @ down.double().T + b_down.double() + want_h
    return errors, rel(stream, exact)


def heads(tokens, count=5, width=64):
    qkv = randn(tokens, 3 * count, width, seed=8)
    q, k = qkv[:, :count], qkv[:, count:2 * count]
    errors = {}
    for name, t, gamma in (("queries", q, randn(width, seed=9)), ("keys", k, randn(width, seed=10))):
        want = rms64(t.double(), gamma)
        B.dvdq_rms_norm(t, None, gamma, EPS, Y=t)   # in place
        errors[name] = rel(t, want)
    freqs, amplitude = B.dvdq_rope_frequencies(width)
    table = torch.empty(tokens, width // 2, 2, device=DEV)
    B.dvdq_rope_table(freqs, None, table, None, amplitude)
    lengths = q.float().norm(dim=-1)
    B.dvdq_rope(q.unsqueeze(0), k.unsqueeze(0), table, None, B.ROPE_HALVES, False, q.unsqueeze(0), k.unsqueeze(0))
    errors["a rotation keeps lengths"] = rel(q.float().norm(dim=-1), lengths.double())
    return errors


def training_step(tokens, dim=320):
    x, r, gamma = randn(tokens, dim, seed=11), randn(tokens, dim, seed=12), randn(dim, seed=13)
    h, y, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(tokens, device=DEV)
    B.dvdq_rms_norm(x, r, gamma, EPS, h, y, None, None, rstd)
    dy, dh = randn(tokens, dim, seed=14), randn(tokens, dim, seed=15)
    dx, dgamma = torch.empty_like(x), torch.empty(dim, device=DEV)
    ws = torch.empty(B.dvdq_rms_norm_backward_workspace_bytes(1, tokens, dim), dtype=torch.uint8, device=DEV)
    B.dvdq_rms_norm_backward(dy, h, rstd, gamma, dh, dx, dgamma, ws)
    # torch's gradients of the formula at the same h
    h6, g6 = h.double().requires_grad_(True), gamma.double().requires_grad_(True)
    y6 = h6 * (h6.square().mean(-1, keepdim=True) + EPS).rsqrt() * g6
    y6.backward(dy.double())
    return {"norm": rel(y, rms64(x.double() + r.double(), gamma)), "norm gradient": rel(dx, h6.grad + dh.double()), "gamma gradient": rel(dgamma, g6.grad)}


def main(tokens=700):
    errors, block = feed_forward(tokens)
    errors.update(heads(tokens))
    errors.update(training_step(tokens))
    status, detail = B.dvdq_last_device_status()
    if status != B.OK:
        raise B.DvdqError(status, f"device status (detail {detail})")
    return errors, block


if __name__ == "__main__":
    errors, block = main(*(int(a) for a in sys.argv[1:2]))
    for name, e in errors.items():
        print(f"{name:28s} relative error {e:.2e}")
    print(f"{'the block in full precision':28s} relative error {block:.2e}")

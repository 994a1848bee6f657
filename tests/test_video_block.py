"""The operators run together as in examples/video_block.py; and their offsets past 32 bits."""
import importlib.util
import os

import pytest
import torch

from paper_2505_18663_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_example():
    """bf16 rounds an output by at most 2^-8, about 0.17 % in the mean square; a chain of three roundings (group norm, linear,
    group norm's gradient) stays below 1 %."""
    spec = importlib.util.spec_from_file_location("video_block", os.path.join(ROOT, "examples", "video_block.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    errors = example.main(2, 7, 9)
    assert len(errors) == 8
    assert all(e < 0.01 for e in errors.values()), errors


FAR = (1 << 31) + 4096  # elements


def test_linear_rows_past_2_31_elements():
    M, N, K, dt = 70000, 32768, 64, torch.bfloat16
    g = torch.Generator(device=DEV).manual_seed(0)
    x, w = torch.randn(M, K, generator=g, device=DEV).to(dt), torch.randn(N, K, generator=g, device=DEV).to(dt)
    y = torch.empty(M, N, dtype=dt, device=DEV)
    assert y.numel() > FAR
    B.dvdq_linear(x, w, None, y.zero_(), 0, y)
    want = x[-300:].double() @ w.double().T
    assert (y[-300:].double() - want).abs().le(2.0 ** -8 * want.abs() + (K + 8) * 2.0 ** -23 * (x[-300:].double().abs() @ w.double().abs().T)).all()
    # the gradient reads those rows: only the last rows of dy differ from zero
    y.zero_()
    y[-20:] = torch.randn(20, N, generator=g, device=DEV).to(dt)
    dx, dw, db = torch.empty(M, K, dtype=dt, device=DEV), torch.empty(N, K, dtype=dt, device=DEV), torch.empty(N, device=DEV)
    ws = torch.empty(B.dvdq_linear_backward_workspace_bytes(M, N, K, 0), dtype=torch.uint8, device=DEV)
    B.dvdq_linear_backward(y, None, x, w, 0, dx, dw, db, ws)
    last, lx = y[-20:].double(), x[-20:].double()
    assert (dx[:-20] == 0).all()
    for got, want, mag in ((dx[-20:], last @ w.double(), last.abs() @ w.double().abs()), (dw, last.T @ lx, last.abs().T @ lx.abs())):
        assert (got.double() - want).abs().le(2.0 ** -8 * want.abs() * 1.01 + N * 2.0 ** -23 * mag).all()
    assert (db.double() - last.sum(0)).abs().le(2.0 ** -18 * last.abs().sum(0)).all()
    assert B.dvdq_last_device_status()[0] == B.OK


def test_rope_and_group_norm_past_2_31_elements():
    dt = torch.bfloat16
    flat = torch.empty(FAR + (1 << 20), dtype=dt, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    # two sequences of 16 tokens, the second one past 2^31 elements
    x = torch.as_strided(flat, (2, 16, 4, 64), (FAR, 256, 64, 1))
    x.copy_(torch.randn(2, 16, 4, 64, generator=g, device=DEV))
    dense, out = x.clone(), torch.empty(2, 16, 4, 64, dtype=dt, device=DEV)
    table = torch.randn(16, 32, 2, generator=g, device=DEV)
    B.dvdq_rope(dense, None, table, None, B.ROPE_HALVES, False, out)
    B.dvdq_rope(x, None, table, None, B.ROPE_HALVES, False, x)
    assert torch.equal(x, out)
    # two samples (the small kernel), and one whose places are far apart (more than 2^31 elements in all)
    for shape, strides in (((2, 50, 64), (FAR, 64, 1)), ((1, 65, 64), (0, 1 << 25, 1))):
        v = torch.as_strided(flat, shape, strides)
        v.copy_(torch.randn(*shape, generator=g, device=DEV))
        dense = v.clone()
        ws = torch.empty(B.dvdq_group_norm_workspace_bytes(*shape, 4), dtype=torch.uint8, device=DEV)
        y = torch.empty_like(dense)
        B.dvdq_group_norm(dense, 4, None, None, 1e-5, 2, y, None, None, ws)
        B.dvdq_group_norm(v, 4, None, None, 1e-5, 2, v, None, None, ws)
        assert torch.equal(v, y)
    del flat, x, v
    # a large sample in the one-launch kernel for large tensors, last places past 2^31 elements
    S, C = 17_000_000, 128
    big = torch.zeros(1, S, C, dtype=dt, device=DEV)
    assert big.numel() > FAR
    big[:, -1000:] = torch.randn(1, 1000, C, generator=g, device=DEV).to(dt)
    tail = big[0, -1000:].double().view(1000, 32, 4)
    n = S * 4
    mean = tail.sum((0, 2)) / n
    rstd = (tail.square().sum((0, 2)) / n - mean.square() + 1e-3).rsqrt()
    want = ((tail - mean[None, :, None]) * rstd[None, :, None]).view(1000, C)
    ws = torch.empty(B.dvdq_group_norm_workspace_bytes(1, S, C, 32), dtype=torch.uint8, device=DEV)
    B.dvdq_group_norm(big, 32, None, None, 1e-3, 0, big, None, None, ws)
    got = big[0, -1000:].double()
    assert (got - want).abs().le(2.0 ** -8 * want.abs() + 1e-3).all()
    assert B.dvdq_last_device_status()[0] == B.OK


def test_in_a_captured_graph():
    """Every operator (one launch, cooperative launch, dependent launches, pieces that are joined) captured once and replayed on
    new inputs: the bits of the same calls outside the graph."""
    dt = torch.bfloat16
    g = torch.Generator(device=DEV).manual_seed(2)
    x = torch.randn(1, 20000, 128, generator=g, device=DEV).to(dt)       # group norm: cooperative
    t = torch.randn(100, 5120, generator=g, device=DEV).to(dt)           # linear: cut along k
    w = (torch.randn(320, 5120, generator=g, device=DEV) / 70).to(dt)
    q = torch.randn(1, 100, 5, 64, generator=g, device=DEV).to(dt)
    table = torch.randn(100, 32, 2, generator=g, device=DEV)
    dy = torch.randn(100, 320, generator=g, device=DEV).to(dt)
    y, n, qo, dx, dw, db = (torch.empty(100, 320, dtype=dt, device=DEV), torch.empty_like(x), torch.empty_like(q), torch.empty_like(t),
                            torch.empty_like(w), torch.empty(320, device=DEV))
    rooms = [torch.empty(max(256, k), dtype=torch.uint8, device=DEV) for k in (
        B.dvdq_linear_workspace_bytes(100, 320, 5120), B.dvdq_linear_backward_workspace_bytes(100, 320, 5120, 2),
        B.dvdq_group_norm_workspace_bytes(1, 20000, 128, 32))]
    assert B.dvdq_linear_workspace_bytes(100, 320, 5120) > 0

    def run():
        B.dvdq_linear(t, w, None, None, 2, y, None, rooms[0])
        B.dvdq_linear_backward(dy, y, t, w, 2, dx, dw, db, rooms[1])
        B.dvdq_rope(q, None, table, None, B.ROPE_PAIRS, False, qo)
        B.dvdq_group_norm(x, 32, None, None, 1e-5, 2, n, None, None, rooms[2])

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for seed in (3, 4):
        g.manual_seed(seed)
        for a in (x, t, q, dy):
            a.copy_(torch.randn(a.shape, generator=g, device=DEV))
        outs = (y, n, qo, dx, dw, db)
        for o in outs:
            o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs))
    assert B.dvdq_last_device_status()[0] == B.OK

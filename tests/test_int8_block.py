"""The 8-bit linear layer, the norm that feeds it and the rows' quantization together, as in examples/int8_block.py; their offsets past 32 bits,
captured graphs, other streams."""
import importlib.util
import os

import pytest
import torch

from paper_2505_18663_b200 import binding as B

gpu = pytest.mark.gpu
DEV = "cuda"
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
E = 2.0 ** -24


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def status_ok():
    assert B.dvdq_last_device_status()[0] == B.OK


@gpu
@pytest.mark.parametrize("tokens", [3, 700])
def test_example(tokens):
    """bf16 rounds an output by at most 2^-8, about 0.17 % in the mean square.  A row in 8 bits is off by top / 127 / sqrt(12) in the mean square.
    Weights: a normal row's top is below 4.5 of its root mean square at these lengths, 4.5 / 127 / sqrt(12) = 1.0 %.  The norm's output is a product of two normal
    values (gamma is one), which exceeds t of its root mean square with a probability below exp(-t): the top of 320 lies near ln 320 = 5.8, in the
    mean square below 8.8: 8.8 / 127 / sqrt(12) = 2.0 %."""
    spec = importlib.util.spec_from_file_location("int8_block", os.path.join(ROOT, "examples", "int8_block.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    errors, block = example.main(tokens)
    assert len(errors) == 11
    in_8_bits = {"weights in 8 bits": 0.012, "norm in 8 bits": 0.02}
    assert all(e < in_8_bits.get(name, 0.004) for name, e in errors.items()), errors
    assert block < 0.05   # four such roundings, each passed on by a layer


FAR = (1 << 31) + 4096  # elements


@gpu
def test_norm_rows_past_2_31_elements():
    dt = torch.bfloat16
    flat = torch.empty(FAR + (1 << 20), dtype=dt, device=DEV)
    g = gen(1)
    gamma = torch.randn(64, generator=g, device=DEV)
    for shape, strides in (((2, 12, 64), (FAR, 64, 1)), ((1, 65, 64), (0, 1 << 25, 1)), ((300, 2, 64), (1 << 22, FAR - (300 << 22), 1))):
        x = torch.as_strided(flat, shape, strides)
        x.copy_(torch.randn(shape, generator=g, device=DEV))
        dense, want = x.clone(), torch.empty(shape, dtype=dt, device=DEV)
        q = torch.empty(shape[:-1], device=DEV)
        B.dvdq_rms_norm(dense, None, gamma, 1e-6, None, want, None, None, q)
        y = torch.empty_like(want)
        B.dvdq_rms_norm(x, None, gamma, 1e-6, None, y)
        assert torch.equal(y, want)
        dy = torch.randn(shape, generator=g, device=DEV).to(dt)
        dx, far = torch.empty_like(want), x   # the gradient over the far rows themselves
        B.dvdq_rms_norm_backward(dy, dense, q, gamma, None, dx, None)
        B.dvdq_rms_norm_backward(dy, x, q, gamma, None, far, None)
        assert torch.equal(far, dx)
    del flat, x, far
    # many rows: the last ones lie past 2^31 elements of inputs, outputs and codes
    rows, C = 1_100_000, 2048
    x = torch.zeros(rows, C, dtype=dt, device=DEV)
    assert x.numel() > FAR
    x[-500:] = torch.randn(500, C, generator=g, device=DEV).to(dt)
    c, s = torch.empty(rows, C, dtype=torch.int8, device=DEV), torch.empty(rows, device=DEV)
    B.dvdq_rms_norm(x, None, None, 1e-6, None, x, c, s)
    tail = torch.Generator(device=DEV).manual_seed(1)
    y6 = c[-500:].double() * s[-500:].double()[:, None]
    assert (x[-500:].double() - y6).abs().le(s[-500:].double()[:, None] * 0.501 + 2.0 ** -8 * x[-500:].double().abs()).all()
    assert (x[:-500:1000] == 0).all() and (c[:-500:1000] == 0).all() and (s[:-500] == 0).all() and (s[-500:] > 0).all()
    c2, s2 = torch.empty_like(c), torch.empty_like(s)
    B.dvdq_quantize_rows(x, c2, s2)
    small = (torch.empty(500, C, dtype=torch.int8, device=DEV), torch.empty(500, device=DEV))
    B.dvdq_quantize_rows(x[-500:].clone(), *small)
    assert torch.equal(c2[-500:], small[0]) and torch.equal(s2[-500:], small[1])
    status_ok()


@gpu
def test_linear_rows_past_2_31_elements():
    M, N, K, dt = 70000, 32768, 64, torch.bfloat16
    g = gen(0)
    a = torch.randint(-127, 128, (M, K), device=DEV, generator=g, dtype=torch.int32).to(torch.int8)
    w = torch.randint(-127, 128, (N, K), device=DEV, generator=g, dtype=torch.int32).to(torch.int8)
    s, t = torch.rand(M, device=DEV, generator=g) * 0.01, torch.rand(N, device=DEV, generator=g) * 0.01
    y = torch.empty(M, N, dtype=dt, device=DEV)
    assert y.numel() > FAR
    B.dvdq_linear_int8(a, s, w, t, None, y.zero_(), 0, y)
    want = (a[-300:].double() @ w.double().T) * (s[-300:].double()[:, None] * t.double())
    assert (y[-300:].double() - want).abs().le((2.0 ** -8 + 5 * E) * want.abs()).all()
    del y, w, want
    # codes past 2^31 bytes
    M, N, K = 70000, 8, 32768
    a = torch.zeros(M, K, dtype=torch.int8, device=DEV)
    assert a.numel() > FAR
    a[-20:] = torch.randint(-127, 128, (20, K), device=DEV, generator=g, dtype=torch.int32).to(torch.int8)
    w = torch.randint(-127, 128, (N, K), device=DEV, generator=g, dtype=torch.int32).to(torch.int8)
    y = torch.empty(M, N, dtype=dt, device=DEV)
    need = B.dvdq_linear_int8_workspace_bytes(M, N, K)
    B.dvdq_linear_int8(a, s, w, t[:N], None, None, 0, y, torch.empty(need, dtype=torch.uint8, device=DEV) if need else None)
    want = (a[-20:].double() @ w.double().T) * (s[-20:].double()[:, None] * t[:N].double())
    assert (y[-20:].double() - want).abs().le((2.0 ** -8 + 5 * E) * want.abs()).all() and (y[:-20] == 0).all()
    # a few tokens against weights past 2^31 bytes: the weights are those rows
    few = torch.randint(-127, 128, (2, K), device=DEV, generator=g, dtype=torch.int32).to(torch.int8)
    y = torch.empty(2, M, dtype=dt, device=DEV)
    B.dvdq_linear_int8(few, s[:2], a, s, None, None, 0, y)
    want = (few.double() @ a[-20:].double().T) * (s[:2].double()[:, None] * s[-20:].double())
    assert (y[:, -20:].double() - want).abs().le((2.0 ** -8 + 5 * E) * want.abs()).all() and (y[:, :-20] == 0).all()
    status_ok()


class Chain:
    """Norm into codes, layer, codes of its output, layer onto the stream, the norm's gradients: a step's calls on fixed buffers."""

    def __init__(self, M, dim, inner, seed, shared=None):
        g = gen(seed)
        dt = torch.bfloat16
        self.x, self.r, self.dy = (torch.empty(M, dim, dtype=dt, device=DEV) for _ in range(3))
        self.gamma = torch.randn(dim, device=DEV, generator=g)
        self.up, self.down = ((torch.randint(-127, 128, s, device=DEV, generator=g, dtype=torch.int32).to(torch.int8), torch.rand(s[0], device=DEV, generator=g) * 1e-3)
                              for s in ((inner, dim), (dim, inner)))
        self.h, self.y, self.out, self.dx = (torch.empty_like(self.x) for _ in range(4))
        self.hidden = torch.empty(M, inner, dtype=dt, device=DEV)
        self.c, self.c2 = torch.empty(M, dim, dtype=torch.int8, device=DEV), torch.empty(M, inner, dtype=torch.int8, device=DEV)
        self.s, self.s2, self.q = (torch.empty(M, device=DEV) for _ in range(3))
        self.dg = torch.empty(dim, device=DEV)
        need = max(B.dvdq_linear_int8_workspace_bytes(M, inner, dim), B.dvdq_linear_int8_workspace_bytes(M, dim, inner), B.dvdq_rms_norm_backward_workspace_bytes(1, M, dim))
        self.ws = shared if shared is not None else torch.empty(need, dtype=torch.uint8, device=DEV)
        assert self.ws.numel() >= need

    def fill(self, seed):
        g = gen(seed)
        for t in (self.x, self.r, self.dy):
            t.copy_(torch.randn(t.shape, device=DEV, generator=g))

    def run(self, stream=None):
        B.dvdq_rms_norm(self.x, self.r, self.gamma, 1e-6, self.h, self.y, self.c, self.s, self.q, stream)
        B.dvdq_linear_int8(self.c, self.s, *self.up, None, None, B.ACT_SILU, self.hidden, self.ws, stream)
        B.dvdq_quantize_rows(self.hidden, self.c2, self.s2, stream)
        B.dvdq_linear_int8(self.c2, self.s2, *self.down, None, self.h, B.ACT_NONE, self.out, self.ws, stream)
        B.dvdq_rms_norm_backward(self.dy, self.h, self.q, self.gamma, self.out, self.dx, self.dg, self.ws, stream)

    def results(self):
        return [t.clone() for t in (self.h, self.y, self.c, self.s, self.q, self.hidden, self.c2, self.s2, self.out, self.dx, self.dg)]

    def spoil(self):
        for t in (self.h, self.y, self.hidden, self.out, self.dx, self.s, self.s2, self.q, self.dg):
            t.fill_(float("nan"))
        self.c.fill_(99), self.c2.fill_(99)


# few tokens; pieces along k; rows in lanes, warps and CTAs, with and without a ring
@gpu
@pytest.mark.parametrize("M,dim,inner", [(5, 96, 704), (200, 512, 8192), (1500, 1536, 640), (2000, 2560, 256), (700, 1552, 2064)])
def test_in_captured_graphs(M, dim, inner):
    """Captured once and replayed on new inputs: the bits of the same calls outside the graph.  Two graphs of other sizes that share a
    workspace, one after the other on a stream, do not disturb each other."""
    a = Chain(M, dim, inner, 3)
    b = Chain(M // 2 + 1, dim, inner, 4, a.ws)
    for chain in (a, b):
        chain.fill(0)
        chain.run()
    torch.cuda.synchronize()
    graphs = []
    for chain in (a, b):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            chain.run()
        graphs.append(graph)
    for seed in (1, 2):
        for chain in (a, b):
            chain.fill(seed)
            chain.spoil()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        got = [chain.results() for chain in (a, b)]
        for chain, replayed in zip((a, b), got):
            chain.run()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(chain.results(), replayed))
    status_ok()


@gpu
def test_on_other_streams_at_the_same_time():
    """Two chains on two streams at once, given by argument and as the current one: each gives the bits that it gives alone."""
    chains = [Chain(1500, 1536, 640, 5), Chain(900, 512, 8192, 6)]
    alone = []
    for i, chain in enumerate(chains):
        chain.fill(i)
        chain.run()
        torch.cuda.synchronize()
        alone.append(chain.results())
        chain.spoil()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        chains[0].run(streams[0])
        with torch.cuda.stream(streams[1]):
            chains[1].run()
    torch.cuda.synchronize()
    for chain, want in zip(chains, alone):
        assert all(torch.equal(x, y) for x, y in zip(chain.results(), want))
    status_ok()


@gpu
def test_tensors_of_another_device_are_refused():
    x = torch.randn(4, 16, device=DEV)

    class Elsewhere(torch.Tensor):   # a tensor that says it is on another GPU; its memory is not
        def get_device(self):
            return 1

    other = torch.randn(4, 16, device=DEV).as_subclass(Elsewhere)
    with pytest.raises(ValueError):
        B.dvdq_rms_norm(x, None, None, 1e-6, None, other)
    with pytest.raises(ValueError):
        B.dvdq_rms_norm(other, None, None, 1e-6, None, x)
    c, s = torch.empty(4, 16, dtype=torch.int8, device=DEV), torch.empty(4, device=DEV)
    with pytest.raises(ValueError):
        B.dvdq_quantize_rows(x, c, s.as_subclass(Elsewhere))
    with pytest.raises(ValueError):
        B.dvdq_linear_int8(c, s, c.as_subclass(Elsewhere), s, None, None, 0, torch.empty(4, 4, dtype=torch.float16, device=DEV))

"""Cases of the 8-bit linear layer and of the RMS norm that feeds it.

Operators:

  linear_int8    y = act(s_m t_n sum_k a_mk w_nk + bias) + residual with int8 codes a, w and a scale for each token and
                 output channel; "values": the activations arrive in 16 bits and are quantized row by row first
  norm           RMS norm of rows, or of the heads inside a fused projection's output, with the residual's addition; its output in
                 the inputs' type, or in 8 bits with a scale for each row
  norm_grad      its gradients

`run` computes them in plain torch operations in 32 bits, or, where `own` is true, through the package's entry points.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
ACTS = {"none": 0, "gelu": 1, "silu": 2}
DEV = "cuda"
EPS = 1e-6


# ------------------------------------------------------------------ cases

def listed():
    return [
        # three timesteps' embeddings through a small layer: latency counts
        {"name": "int8 linear 3 tokens", "op": "linear_int8", "dtype": "fp16", "M": 3, "N": 1536, "K": 1536, "act": "silu",
         "bias": True, "residual": False, "values": False},
        # one token of the text model that writes the prompt, through its widest layer: the weights are what is read
        {"name": "int8 linear 1 token wide", "op": "linear_int8", "dtype": "bf16", "M": 1, "N": 13824, "K": 5120, "act": "none",
         "bias": False, "residual": False, "values": True},
        # a prompt's tokens, odd sizes throughout (rows padded to 16 bytes)
        {"name": "int8 linear text ragged", "op": "linear_int8", "dtype": "fp16", "M": 517, "N": 4101, "K": 2049, "act": "silu",
         "bias": True, "residual": True, "values": False},
        # the small video model's feed-forward down: hidden activations quantized, then onto the residual stream
        {"name": "int8 linear down from values", "op": "linear_int8", "dtype": "bf16", "M": 32760, "N": 1536, "K": 8960, "act": "none",
         "bias": True, "residual": True, "values": True},
        # the large video model's feed-forward up, codes from the norm in front of it
        {"name": "int8 linear feed-forward up", "op": "linear_int8", "dtype": "bf16", "M": 32760, "N": 13824, "K": 5120, "act": "gelu",
         "bias": True, "residual": False, "values": False},
        # a few tokens of the text model: residual added, both outputs and the statistics: latency counts
        {"name": "norm few rows", "op": "norm", "dtype": "fp16", "params": "fp16", "N": 1, "S": 7, "C": 1536, "fused": 0,
         "residual": True, "y": True, "codes": False, "stats": True},
        # the queries of every token, head by head, inside the fused projection's output (12 + 12 + 12 heads)
        {"name": "norm queries", "op": "norm", "dtype": "bf16", "params": "bf16", "N": 32760, "S": 12, "C": 128, "fused": 36,
         "residual": False, "y": True, "codes": False, "stats": False},
        # in front of the large model's feed-forward: residual added and kept, normalised rows in 8 bits
        {"name": "norm residual to int8", "op": "norm", "dtype": "bf16", "params": "bf16", "N": 1, "S": 32760, "C": 5120, "fused": 0,
         "residual": True, "y": False, "codes": True, "stats": False},
        # a training step's forward in fp32, rows that start nowhere in particular
        {"name": "norm fp32 ragged", "op": "norm", "dtype": "fp32", "params": "fp32", "N": 2, "S": 1001, "C": 2049, "fused": 0,
         "residual": True, "y": True, "codes": False, "stats": True},
        # training the large model: the gradient that comes along the residual stream is added
        {"name": "norm gradients", "op": "norm_grad", "dtype": "bf16", "params": "fp32", "N": 1, "S": 32760, "C": 5120, "fused": 0,
         "residual": True},
        # training the norm of the queries on a short clip
        {"name": "norm gradients queries", "op": "norm_grad", "dtype": "bf16", "params": "bf16", "N": 4680, "S": 12, "C": 128, "fused": 36,
         "residual": False},
        # a prompt's rows, an odd width
        {"name": "norm gradients ragged", "op": "norm_grad", "dtype": "fp16", "params": "fp32", "N": 1, "S": 509, "C": 1541, "fused": 0,
         "residual": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear_int8", "linear_int8", "linear_int8", "norm", "norm", "norm_grad"])
    if op == "linear_int8":
        while True:
            M, N, K = _log(rng, 1, 32760), _log(rng, 64, 13824), _log(rng, 64, 13824)
            if M * N * K <= 32760 * 13824 * 5120:
                break
        return {"op": op, "dtype": rng.choice(["bf16", "fp16"]), "M": M, "N": N, "K": K, "act": rng.choice(sorted(ACTS)),
                "bias": rng.random() < 0.8, "residual": rng.random() < 0.4, "values": rng.random() < 0.4}
    while True:
        heads = rng.random() < 0.4
        C = rng.choice([64, 72, 80, 96, 128, 256]) if heads else _log(rng, 64, 16384)
        N, S = (_log(rng, 1, 32760), rng.choice([1, 2, 8, 12, 24])) if heads else (rng.choice([1, 1, 2, 3]), _log(rng, 1, 32760))
        if N * S * C <= 32760 * 5120:
            break
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    case = {"op": op, "dtype": dtype, "params": rng.choice([dtype, "fp32"]), "N": N, "S": S, "C": C, "fused": 3 * S if heads else 0,
            "residual": not heads and rng.random() < 0.7}
    if op == "norm":
        codes = rng.random() < 0.4
        case.update(y=not codes or rng.random() < 0.2, codes=codes, stats=rng.random() < 0.3)
    return case


# ------------------------------------------------------------------ inputs

def _rows(rows, cols, dt):
    """An uninitialised [rows, cols] matrix whose rows start on 16 bytes."""
    per = 16 // torch.empty(0, dtype=dt).element_size()
    return torch.empty(rows, -(-cols // per) * per, dtype=dt, device=DEV)[:, :cols]


def _normal(rows, cols, dt, g, scale=1.0):
    t = _rows(rows, cols, dt)
    t.copy_(torch.randn(rows, cols, device=DEV, generator=g, dtype=torch.float32).mul_(scale))
    return t


def _codes_of(values):
    """Codes and scales of rows in fp32, as a program has them in hand."""
    scales = values.abs().amax(1) / 127
    codes = _rows(*values.shape, torch.int8)
    codes.copy_(torch.round(values / scales[:, None]))
    return codes, scales


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt, op = DTYPES[case["dtype"]], case["op"]
    s = dict(case, seed=seed)
    if op == "linear_int8":
        M, N, K = case["M"], case["N"], case["K"]
        x = torch.randn(M, K, device=DEV, generator=g).mul_(0.5 + torch.rand(M, 1, device=DEV, generator=g))
        if case["values"]:  # what the program quantizes, and where it keeps the codes
            s["x"] = _rows(M, K, dt)
            s["x"].copy_(x)
            s["a"], s["sa"] = _rows(M, K, torch.int8), torch.empty(M, device=DEV)
        else:
            s["a"], s["sa"] = _codes_of(x)
        del x
        s["w"], s["sw"] = _codes_of(torch.randn(N, K, device=DEV, generator=g).mul_(1 / math.sqrt(K)))
        s["b"] = _normal(1, N, dt, g, 0.1)[0] if case["bias"] else None
        s["r"] = _normal(M, N, dt, g) if case["residual"] else None
        s["out_y"] = _rows(M, N, dt)
        return s
    N, S, C, pt = case["N"], case["S"], case["C"], DTYPES[case["params"]]
    # activations: some channels are several times as large as the rest, as in a trained model's residual stream
    channel = torch.exp(0.7 * torch.randn(C, device=DEV, generator=g))

    def tensor(fill):
        t = torch.empty(N, case["fused"] or S, C, dtype=dt, device=DEV)[:, :S]
        if fill:
            t.copy_(torch.randn(N, S, C, device=DEV, generator=g).mul_(channel))
        return t

    s["x"] = tensor(True)
    s["gamma"] = (1 + 0.2 * torch.randn(C, device=DEV, generator=g)).to(pt)
    if op == "norm":
        s["r"] = tensor(True) if case["residual"] else None
        s["out_h"] = torch.empty(N, S, C, dtype=dt, device=DEV) if case["residual"] else None
        s["out_y"] = torch.empty(N, S, C, dtype=dt, device=DEV) if case["y"] else None
        s["out_codes"] = _rows(N * S, C, torch.int8).unflatten(0, (N, S)) if case["codes"] else None
        s["out_scales"] = torch.empty(N, S, device=DEV) if case["codes"] else None
        s["out_values"] = torch.empty(N, S, C, dtype=_of_codes(dt), device=DEV) if case["codes"] else None
        s["out_rstd"] = torch.empty(N, S, device=DEV) if case["stats"] else None
        return s
    s["rstd"] = torch.rsqrt(s["x"].float().square().mean(-1, dtype=torch.float64) + EPS).float()
    s["dy"] = torch.randn(N, S, C, device=DEV, generator=g).to(dt)
    s["dh"] = torch.randn(N, S, C, device=DEV, generator=g).to(dt) if case["residual"] else None
    s["out_dx"], s["out_dgamma"] = tensor(False), torch.empty(C, device=DEV)
    return s


def _of_codes(dt):
    """The type in which the values that codes stand for are given."""
    return torch.bfloat16 if dt is torch.float32 else dt


# ------------------------------------------------------------------ one pass

def run(state):
    if own:
        return _own(state)
    return {"linear_int8": _linear_int8, "norm": _norm, "norm_grad": _norm_grad}[state["op"]](state)


def _workspace(s, n):
    if "workspace" not in s:
        s["workspace"] = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None
    return s["workspace"]


def _own(s):
    from paper_2505_18663_b200 import binding as B
    op = s["op"]
    if op == "linear_int8":
        ws = s["workspace"] if "workspace" in s else _workspace(s, B.dvdq_linear_int8_workspace_bytes(s["M"], s["N"], s["K"]))
        if s["values"]:
            B.dvdq_quantize_rows(s["x"], s["a"], s["sa"])
        B.dvdq_linear_int8(s["a"], s["sa"], s["w"], s["sw"], s["b"], s["r"], ACTS[s["act"]], s["out_y"], ws)
        return {"y": s["out_y"]}
    if op == "norm":
        B.dvdq_rms_norm(s["x"], s["r"], s["gamma"], EPS, s["out_h"], s["out_y"], s["out_codes"], s["out_scales"], s["out_rstd"])
        out = {"h": s["out_h"], "y": s["out_y"], "rstd": s["out_rstd"]}
        if s["codes"]:
            out["values"] = torch.mul(s["out_codes"], s["out_scales"][..., None], out=s["out_values"])
        return out
    ws = s["workspace"] if "workspace" in s else _workspace(s, B.dvdq_rms_norm_backward_workspace_bytes(s["N"], s["S"], s["C"]))
    B.dvdq_rms_norm_backward(s["dy"], s["x"], s["rstd"], s["gamma"], s["dh"], s["out_dx"], s["out_dgamma"], ws)
    return {"dx": s["out_dx"], "dgamma": s["out_dgamma"]}


def _act(z, act):
    if act == "gelu":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z * torch.sigmoid(z) if act == "silu" else z


def _quantize(v):
    """(codes as fp32 numbers, scales) of rows."""
    scales = v.abs().amax(-1, keepdim=True) / 127
    return torch.where(scales > 0, torch.round(v / scales), 0.0), scales


def _linear_int8(s):
    a, sa = _quantize(s["x"].float()) if s["values"] else (s["a"].float(), s["sa"][:, None])
    z = (a @ s["w"].float().T) * (sa * s["sw"])
    if s["b"] is not None:
        z = z + s["b"].float()
    y = _act(z, s["act"])
    if s["r"] is not None:
        y = y + s["r"].float()
    return {"y": y.to(s["out_y"].dtype)}


def _norm(s):
    dt = s["x"].dtype
    h = s["x"].float()
    if s["r"] is not None:
        h = h + s["r"].float()
    rstd = torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS)
    y = h * rstd * s["gamma"].float()
    out = {"h": h.to(dt) if s["residual"] else None, "y": y.to(dt) if s["y"] else None, "rstd": rstd[..., 0] if s["stats"] else None}
    if s["codes"]:
        codes, scales = _quantize(y)
        out["values"] = (codes * scales).to(_of_codes(dt))
    return out


def _norm_grad(s):
    rstd = s["rstd"][..., None]
    hh = s["x"].float() * rstd
    dy = s["dy"].float()
    dh = dy * s["gamma"].float()
    dx = rstd * (dh - hh * (dh * hh).mean(-1, keepdim=True))
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    return {"dx": dx.to(s["x"].dtype), "dgamma": (dy * hh).sum((0, 1))}


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    op, e = case["op"], {"bf16": 2, "fp16": 2, "fp32": 4}[case["dtype"]]
    if op == "linear_int8":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": (e if case["values"] else 1) * M * K + N * K + e * (M * N * (1 + case["residual"]) + N * case["bias"]) + 4 * (M + N),
                "flops": 2 * M * N * K}
    rows, p = case["N"] * case["S"], 4 if case["params"] == "fp32" else 2
    n = rows * case["C"]
    if op == "norm":
        return {"bytes": n * (e * (1 + 2 * case["residual"] + case["y"]) + case["codes"]) + p * case["C"] + 4 * rows * (case["codes"] + case["stats"]),
                "flops": 6 * n}
    return {"bytes": e * n * (3 + case["residual"]) + (p + 4) * case["C"] + 4 * rows, "flops": 10 * n}


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "linear_int8":
        if case["values"]:
            x = s["x"].double()
            step = torch.linalg.vector_norm(x, math.inf, dim=1, keepdim=True).div_(127)
            a = x.div_(step).round_().mul_(step)
        else:
            a = torch.mul(s["a"], s["sa"].double().unsqueeze(1))
        y = torch.mm(a, torch.mul(s["w"], s["sw"].double().unsqueeze(1)).t())
        del a
        if case["bias"]:
            y += s["b"].double()
        if case["act"] == "silu":
            y = y / (1 + torch.exp(-y))
        elif case["act"] == "gelu":
            y = y / (1 + torch.exp(y * (1 + 0.044715 * y.square()) * (-2 * math.sqrt(2 / math.pi))))
        if case["residual"]:
            y += s["r"].double()
        return {"y": y}
    C, gamma, x = case["C"], s["gamma"].double(), s["x"].double()
    if op == "norm":
        if case["residual"]:
            x = x + s["r"].double()
        size = torch.linalg.vector_norm(x, dim=-1, keepdim=True)
        length = torch.sqrt(size.square() / C + EPS)
        y = torch.div(x, length) * gamma
        out = {"h": x if case["residual"] else None, "y": y if case["y"] else None, "rstd": length.reciprocal().squeeze(-1) if case["stats"] else None}
        if case["codes"]:
            top = torch.linalg.vector_norm(y, math.inf, dim=-1, keepdim=True)
            out["values"] = torch.round(y * 127 / top) * top / 127
        return out
    rstd, dy = s["rstd"].double().unsqueeze(-1), s["dy"].double()
    along = torch.einsum("nsc,nsc,c->ns", dy, x, gamma).unsqueeze(-1)  # of the row's direction
    dx = rstd * dy * gamma - x * along * rstd ** 3 / C
    if case["residual"]:
        dx += s["dh"].double()
    return {"dx": dx, "dgamma": torch.einsum("nsc,nsc,ns->c", dy, x, rstd.squeeze(-1))}

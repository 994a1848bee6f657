"""Cases of the operators around the quantized linear layers of a video transformer.

Three operators, each forward and backward:

  linear         y = act(x w^T + bias) + residual in 16-bit floating point: the layers that stay unquantized
                 (embedders, modulation, output projections, the last layer), and its gradients
  rope           rotary positions of queries and keys, in pairs or in halves, over part of the head or all of it;
                 its gradient is the rotation the other way round
  group_norm     group norm with an activation, channels last: the latent decoder's normalisation, and its gradients

`run` computes them in plain torch operations in 32 bits, or, where `own` is true, through the package's entry points.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
ACTS = {"none": 0, "gelu": 1, "silu": 2}
DEV = "cuda"
EPS = 1e-5


# ------------------------------------------------------------------ cases

def listed():
    return [
        # the modulation of one denoising step: one conditioning vector to six shifts, scales and gates
        {"name": "linear modulation 1 token", "op": "linear", "dtype": "bf16", "M": 1, "N": 18432, "K": 3072,
         "act": "none", "bias": True, "residual": False, "save_z": False},
        # a prompt's embeddings through a text projection in training: ragged length, an inner size that is no
        # multiple of anything (rows padded to 16 bytes), the pre-activation kept for the backward pass
        {"name": "linear text ragged", "op": "linear", "dtype": "fp16", "M": 509, "N": 5120, "K": 4100,
         "act": "silu", "bias": True, "residual": False, "save_z": True},
        # attention's output projection added onto the residual stream, at the token count of a small video model
        {"name": "linear out projection", "op": "linear", "dtype": "bf16", "M": 32760, "N": 1536, "K": 1536,
         "act": "none", "bias": True, "residual": True, "save_z": False},
        # the widest feed-forward layer of a large video model, left in 16 bits
        {"name": "linear feed-forward up", "op": "linear", "dtype": "bf16", "M": 32760, "N": 13824, "K": 5120,
         "act": "gelu", "bias": True, "residual": False, "save_z": False},
        # fine-tuning that feed-forward layer in the small model
        {"name": "linear gradients", "op": "linear_grad", "dtype": "bf16", "M": 32760, "N": 8960, "K": 1536, "act": "gelu"},
        # fine-tuning a projection on a short clip: odd sizes throughout, few tiles
        {"name": "linear gradients ragged", "op": "linear_grad", "dtype": "fp16", "M": 1021, "N": 1541, "K": 1030, "act": "none"},
        # every block of the small video model: queries and keys inside the fused projection's output, three-axis positions
        {"name": "rope video", "op": "rope", "dtype": "bf16", "B": 1, "S": 32760, "Hq": 12, "Hk": 12, "D": 128, "rot": 128,
         "layout": "pairs", "inverse": False, "fused": True, "gather": False, "axes": 3, "stretch": 1.0},
        # a text model that writes the prompt, one token for each of seven requests, at positions of their own,
        # grouped heads, half of the head rotated, a stretched context
        {"name": "rope one token", "op": "rope", "dtype": "fp16", "B": 7, "S": 1, "Hq": 32, "Hk": 8, "D": 128, "rot": 64,
         "layout": "halves", "inverse": False, "fused": False, "gather": True, "axes": 1, "stretch": 4.0},
        # the backward pass over a long sequence
        {"name": "rope gradient long", "op": "rope", "dtype": "bf16", "B": 1, "S": 65536, "Hq": 24, "Hk": 8, "D": 96, "rot": 96,
         "layout": "halves", "inverse": True, "fused": False, "gather": False, "axes": 1, "stretch": 8.0},
        # the last stage of a latent video decoder: few channels, many places
        {"name": "group norm decoder", "op": "group_norm", "dtype": "bf16", "params": "bf16", "N": 1, "S": 499200, "C": 128,
         "G": 32, "act": "silu", "stats": False},
        # a small feature map with an odd channel count, no activation: latency counts
        {"name": "group norm small", "op": "group_norm", "dtype": "fp32", "params": "fp32", "N": 3, "S": 77, "C": 180,
         "G": 12, "act": "none", "stats": True},
        # training an inner stage of that decoder
        {"name": "group norm gradients", "op": "group_norm_grad", "dtype": "bf16", "params": "fp32", "N": 2, "S": 18720,
         "C": 512, "G": 32, "act": "silu"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "linear", "linear_grad", "rope", "rope", "group_norm", "group_norm_grad"])
    if op in ("linear", "linear_grad"):
        most = 32760 * 13824 * 5120 if op == "linear" else 32760 * 8960 * 1536
        while True:
            M, N, K = _log(rng, 1, 32760), _log(rng, 64, 13824), _log(rng, 64, 13824)
            if M * N * K <= most:
                break
        case = {"op": op, "dtype": rng.choice(["bf16", "fp16"]), "M": M, "N": N, "K": K, "act": rng.choice(sorted(ACTS))}
        if op == "linear":
            case.update(bias=rng.random() < 0.8, residual=rng.random() < 0.4, save_z=rng.random() < 0.2)
        return case
    if op == "rope":
        while True:
            B, S, D = rng.choice([1, 1, 2, 5]), _log(rng, 1, 65536), rng.choice([64, 72, 80, 96, 128, 256])
            Hk = rng.choice([1, 2, 8, 12])
            Hq = Hk * rng.choice([1, 2, 3])
            if B * S * (Hq + Hk) * D <= 65536 * 32 * 96:
                break
        return {"op": op, "dtype": rng.choice(["bf16", "bf16", "fp16", "fp32"]), "B": B, "S": S, "Hq": Hq, "Hk": Hk, "D": D,
                "rot": rng.choice([D, D, D // 2, D // 4 * 2 - 2]), "layout": rng.choice(["pairs", "halves"]),
                "inverse": rng.random() < 0.4, "fused": rng.random() < 0.5, "gather": rng.random() < 0.5,
                "axes": rng.choice([1, 3]), "stretch": rng.choice([1.0, 4.0, 8.0])}
    while True:
        N, S, G, per = rng.choice([1, 1, 2, 3, 4]), _log(rng, 1, 499200), rng.choice([1, 4, 12, 32]), _log(rng, 1, 40)
        if S * per >= 64 and N * S * G * per <= 499200 * 128:
            break
    case = {"op": op, "dtype": rng.choice(["bf16", "bf16", "fp16", "fp32"]), "params": "fp32", "N": N, "S": S, "C": G * per,
            "G": G, "act": rng.choice(sorted(ACTS))}
    case["params"] = rng.choice([case["dtype"], "fp32"])
    if op == "group_norm":
        case["stats"] = rng.random() < 0.3
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


def _table(case, rows_wanted, g):
    """Cosines and sines of every position, [positions, rot / 2, 2] in 32 bits, from angles in 64."""
    half = case["rot"] // 2
    i = torch.arange(half, dtype=torch.float64, device=DEV)
    freq = 10000.0 ** (-i / max(1, half)) / case["stretch"]
    n = torch.arange(rows_wanted, dtype=torch.float64, device=DEV)
    if case["axes"] == 3:  # (frame, row, column) of each token of a video, 52 columns and 30 rows of patches
        axis = torch.clamp((i * 3 / max(1, half)).floor(), max=2).long()
        pos = torch.stack([torch.floor(n / 1560), torch.floor(n / 52) % 30, n % 52], 1)[:, axis]
    else:
        pos = n[:, None]
    angle = pos * freq
    return torch.stack([torch.cos(angle), torch.sin(angle)], -1).float().contiguous()


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt, op = DTYPES[case["dtype"]], case["op"]
    s = dict(case, seed=seed)
    if op in ("linear", "linear_grad"):
        M, N, K = case["M"], case["N"], case["K"]
        s["x"], s["w"] = _normal(M, K, dt, g), _normal(N, K, dt, g, 1.0 / math.sqrt(K))
        if op == "linear":
            s["b"] = _normal(1, N, dt, g, 0.1)[0] if case["bias"] else None
            s["r"] = _normal(M, N, dt, g) if case["residual"] else None
            s["y"], s["z"] = _rows(M, N, dt), _rows(M, N, dt) if case["save_z"] else None
        else:
            s["dy"] = _normal(M, N, dt, g)
            s["z"] = _normal(M, N, dt, g) if case["act"] != "none" else None
            s["dx"], s["dw"], s["db"] = _rows(M, K, dt), _rows(N, K, dt), torch.empty(N, device=DEV)
    elif op == "rope":
        B, S, Hq, Hk, D = (case[k] for k in ("B", "S", "Hq", "Hk", "D"))
        heads = Hq + 2 * Hk if case["fused"] else Hq + Hk
        t = torch.randn(B, S, heads, D, device=DEV, generator=g).to(dt) if case["fused"] else None
        s["q"] = t[:, :, :Hq] if case["fused"] else torch.randn(B, S, Hq, D, device=DEV, generator=g).to(dt)
        s["k"] = t[:, :, Hq:Hq + Hk] if case["fused"] else torch.randn(B, S, Hk, D, device=DEV, generator=g).to(dt)
        positions = max(S, 32768) if case["gather"] else S
        s["table"] = _table(case, positions, g)
        s["rows"] = torch.randint(0, positions, (B, S), device=DEV, generator=g, dtype=torch.int32) if case["gather"] else None
        s["q_out"], s["k_out"] = torch.empty(B, S, Hq, D, dtype=dt, device=DEV), torch.empty(B, S, Hk, D, dtype=dt, device=DEV)
    else:
        N, S, C, G = (case[k] for k in ("N", "S", "C", "G"))
        pt = DTYPES[case["params"]]
        offset = torch.randn(N, 1, C, device=DEV, generator=g).mul_(0.5).add_(0.3)
        s["x"] = torch.randn(N, S, C, device=DEV, generator=g).add_(offset).to(dt)
        s["gamma"] = (1 + 0.2 * torch.randn(C, device=DEV, generator=g)).to(pt)
        s["beta"] = (0.2 * torch.randn(C, device=DEV, generator=g)).to(pt)
        if op == "group_norm":
            s["y"] = torch.empty(N, S, C, dtype=dt, device=DEV)
            s["mean"], s["rstd"] = ((torch.empty(N, G, device=DEV), torch.empty(N, G, device=DEV)) if case["stats"] else (None, None))
        else:
            s["dy"] = torch.randn(N, S, C, device=DEV, generator=g).to(dt)
            v = s["x"].reshape(N, S, G, C // G).float()
            mean = v.mean((1, 3), dtype=torch.float64)
            s["mean"] = mean.float()
            s["rstd"] = ((v - s["mean"][:, None, :, None]).square_().mean((1, 3), dtype=torch.float64) + EPS).rsqrt().float()
            s["dx"] = torch.empty(N, S, C, dtype=dt, device=DEV)
            s["dgamma"], s["dbeta"] = torch.empty(C, device=DEV), torch.empty(C, device=DEV)
    return s


# ------------------------------------------------------------------ one pass

def run(state):
    if own:
        return _own(state)
    return {"linear": _linear, "linear_grad": _linear_grad, "rope": _rope, "group_norm": _group_norm,
            "group_norm_grad": _group_norm_grad}[state["op"]](state)


def _workspace(s, n):
    if "workspace" not in s:
        s["workspace"] = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None
    return s["workspace"]


def _own(s):
    from paper_2505_18663_b200 import binding as B
    op, act = s["op"], ACTS[s.get("act", "none")]
    if op == "linear":
        ws = s["workspace"] if "workspace" in s else _workspace(s, B.dvdq_linear_workspace_bytes(s["M"], s["N"], s["K"]))
        B.dvdq_linear(s["x"], s["w"], s["b"], s["r"], act, s["y"], s["z"], ws)
        return {"y": s["y"], "z": s["z"]} if s["save_z"] else {"y": s["y"]}
    if op == "linear_grad":
        ws = (s["workspace"] if "workspace" in s else
              _workspace(s, B.dvdq_linear_backward_workspace_bytes(s["M"], s["N"], s["K"], act)))
        B.dvdq_linear_backward(s["dy"], s["z"], s["x"], s["w"], act, s["dx"], s["dw"], s["db"], ws)
        return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}
    if op == "rope":
        layout = B.ROPE_PAIRS if s["layout"] == "pairs" else B.ROPE_HALVES
        B.dvdq_rope(s["q"], s["k"], s["table"], s["rows"], layout, s["inverse"], s["q_out"], s["k_out"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "group_norm":
        ws = (s["workspace"] if "workspace" in s else
              _workspace(s, B.dvdq_group_norm_workspace_bytes(s["N"], s["S"], s["C"], s["G"])))
        B.dvdq_group_norm(s["x"], s["G"], s["gamma"], s["beta"], EPS, act, s["y"], s["mean"], s["rstd"], ws)
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]} if s["stats"] else {"y": s["y"]}
    ws = (s["workspace"] if "workspace" in s else
          _workspace(s, B.dvdq_group_norm_workspace_bytes(s["N"], s["S"], s["C"], s["G"])))
    B.dvdq_group_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["G"], s["gamma"], s["beta"], act, s["dx"],
                               s["dgamma"], s["dbeta"], ws)
    return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}


def _act(z, act):
    if act == "gelu":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z * torch.sigmoid(z) if act == "silu" else z


def _act_slope(z, act):
    if act == "gelu":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    sig = torch.sigmoid(z)
    return sig * (1 + z * (1 - sig))


def _linear(s):
    dt = s["x"].dtype
    z = s["x"].float() @ s["w"].float().T
    if s["b"] is not None:
        z = z + s["b"].float()
    y = _act(z, s["act"])
    if s["r"] is not None:
        y = y + s["r"].float()
    return {"y": y.to(dt), "z": z.to(dt)} if s["save_z"] else {"y": y.to(dt)}


def _linear_grad(s):
    dt = s["x"].dtype
    dz = s["dy"].float()
    if s["act"] != "none":
        dz = dz * _act_slope(s["z"].float(), s["act"])
    return {"dx": (dz @ s["w"].float()).to(dt), "dw": (dz.T @ s["x"].float()).to(dt), "db": dz.sum(0)}


def _rotate(t, table, rot, layout, inverse):
    v = t.float()
    cos, sin = table[..., 0], table[..., 1]
    if inverse:
        sin = -sin
    if layout == "pairs":
        a, b = v[..., 0:rot:2], v[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = v[..., :rot // 2], v[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, v[..., rot:]], -1).to(t.dtype)


def _rope(s):
    table = s["table"][s["rows"].long()] if s["rows"] is not None else s["table"][None]
    table = table[:, :, None]
    return {n: _rotate(s[n], table, s["rot"], s["layout"], s["inverse"]) for n in ("q", "k")}


def _group_norm(s):
    N, S, C, G = s["N"], s["S"], s["C"], s["G"]
    x = s["x"].float().view(N, S, G, C // G)
    mean = x.mean((1, 3), keepdim=True)
    d = x - mean
    rstd = torch.rsqrt((d * d).mean((1, 3), keepdim=True) + EPS)
    z = (d * rstd).view(N, S, C) * s["gamma"].float() + s["beta"].float()
    y = _act(z, s["act"]).to(s["x"].dtype)
    return {"y": y, "mean": mean.view(N, G), "rstd": rstd.view(N, G)} if s["stats"] else {"y": y}


def _group_norm_grad(s):
    N, S, C, G = s["N"], s["S"], s["C"], s["G"]
    mean, rstd = s["mean"].view(N, 1, G, 1), s["rstd"].view(N, 1, G, 1)
    h = (s["x"].float().view(N, S, G, C // G) - mean) * rstd
    gamma = s["gamma"].float()
    dz = s["dy"].float()
    if s["act"] != "none":
        dz = dz * _act_slope(h.view(N, S, C) * gamma + s["beta"].float(), s["act"])
    dh = (dz * gamma).view(N, S, G, C // G)
    dx = rstd * (dh - dh.mean((1, 3), keepdim=True) - h * (dh * h).mean((1, 3), keepdim=True))
    return {"dx": dx.view(N, S, C).to(s["x"].dtype), "dgamma": (dz * h.view(N, S, C)).sum((0, 1)), "dbeta": dz.sum((0, 1))}


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    op, e = case["op"], {"bf16": 2, "fp16": 2, "fp32": 4}[case["dtype"]]
    if op == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        outs = 1 + case["save_z"] + case["residual"]
        return {"bytes": e * (M * K + N * K + outs * M * N + N * case["bias"]), "flops": 2 * M * N * K}
    if op == "linear_grad":
        M, N, K = case["M"], case["N"], case["K"]
        read = M * K + N * K + M * N * (1 if case["act"] == "none" else 2)
        return {"bytes": e * (read + M * K + N * K) + 4 * N, "flops": 4 * M * N * K}
    if op == "rope":
        tokens = case["B"] * case["S"]
        angles = tokens if case["gather"] else case["S"]
        return {"bytes": 2 * e * tokens * (case["Hq"] + case["Hk"]) * case["D"] + angles * (4 * case["rot"] + 4 * case["gather"]),
                "flops": 3 * tokens * (case["Hq"] + case["Hk"]) * case["rot"]}
    n = case["N"] * case["S"] * case["C"]
    p = 4 if case["params"] == "fp32" else 2
    if op == "group_norm":
        return {"bytes": 2 * e * n + 2 * p * case["C"] + 8 * case["N"] * case["G"] * case["stats"], "flops": 10 * n}
    return {"bytes": 3 * e * n + (2 * p + 8) * case["C"] + 8 * case["N"] * case["G"], "flops": 25 * n}


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    wide = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()
            and k not in ("y", "dx", "dw", "db", "dgamma", "dbeta", "q_out", "k_out")}
    op = case["op"]
    if op == "linear":
        z = torch.mm(wide["x"], wide["w"].t())
        if case["bias"]:
            z += wide["b"]
        out = {"z": z} if case["save_z"] else {}
        y = _value64(z, case["act"])
        out["y"] = y + wide["r"] if case["residual"] else y
        return out
    if op == "linear_grad":
        dz = wide["dy"] * _slope64(wide["z"], case["act"]) if case["act"] != "none" else wide["dy"]
        return {"dx": torch.mm(dz, wide["w"]), "dw": torch.mm(dz.t(), wide["x"]),
                "db": torch.mv(dz.t(), torch.ones(case["M"], dtype=torch.float64, device=DEV))}
    if op == "rope":
        turn = torch.complex(wide["table"][..., 0], wide["table"][..., 1])
        turn = turn.conj().resolve_conj() if case["inverse"] else turn
        turn = (turn[s["rows"].long()] if case["gather"] else turn.unsqueeze(0)).unsqueeze(2)
        half, out = case["rot"] // 2, {}
        for name in ("q", "k"):
            v = wide[name].clone(memory_format=torch.contiguous_format)
            r = v[..., :case["rot"]]
            r = r.unflatten(-1, (half, 2)) if case["layout"] == "pairs" else r.unflatten(-1, (2, half)).transpose(-1, -2)
            c = torch.complex(r[..., 0].contiguous(), r[..., 1].contiguous()) * turn
            c = torch.stack([c.real, c.imag], -1 if case["layout"] == "pairs" else -2).flatten(-2)
            v[..., :case["rot"]] = c
            out[name] = v
        return out
    N, S, C, G = (case[k] for k in ("N", "S", "C", "G"))
    per = C // G
    by_group = wide["x"].unflatten(-1, (G, per)).transpose(1, 2).flatten(2)  # [N, G, S * per]
    gamma, beta = (wide[k].view(1, G, 1, per).expand(N, G, S, per).flatten(2) for k in ("gamma", "beta"))

    def back(t):
        return t.unflatten(-1, (S, per)).transpose(1, 2).flatten(2)

    if op == "group_norm":
        var, mean = torch.var_mean(by_group, -1, correction=0)
        rstd = 1.0 / torch.sqrt(var + EPS)
        y = _value64(gamma * (by_group - mean[..., None]) * rstd[..., None] + beta, case["act"])
        return {"y": back(y), "mean": mean, "rstd": rstd} if case["stats"] else {"y": back(y)}
    rstd = wide["rstd"][..., None]
    h = (by_group - wide["mean"][..., None]) * rstd
    dz = wide["dy"].unflatten(-1, (G, per)).transpose(1, 2).flatten(2)
    if case["act"] != "none":
        dz = dz * _slope64(gamma * h + beta, case["act"])
    dh = dz * gamma
    n = S * per
    dx = rstd / n * (n * dh - dh.sum(-1, keepdim=True) - h * (dh * h).sum(-1, keepdim=True))
    return {"dx": back(dx), "dgamma": back(dz * h).sum((0, 1)), "dbeta": back(dz).sum((0, 1))}


def _value64(z, act):
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return z / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * z * (1 + 0.044715 * z * z)))
    return z


def _slope64(z, act):
    """The derivative of z f(u(z)) with f the logistic function: f + z u' f (1 - f)."""
    u, du = (z, 1.0) if act == "silu" else (math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3), math.sqrt(8 / math.pi) * (1 + 0.134145 * z ** 2))
    f = 1 / (1 + torch.exp(-u))
    return f + z * du * f * (1 - f)

"""Quantized layers at work: the operators that take a solved layer (codes, scales, zeros) into a model, and what is measured of them.

``op`` names the operator of a case:

  linear    Y = act(X W_hat + bias) + residual with W_hat = a * Q + b of a quantized layer: the layer in a model that answers, from one
            token to a whole calibration batch (whose outputs are the next layer's calibration inputs)
  backward  gradients of that product for X, the scales a, the zeros b and the bias, the codes fixed: tuning of a quantized layer
  moe       a gated mixture-of-experts layer for a few tokens whose experts are quantized layers: router, top-k, gate and up, down, sum

``run`` computes them in plain torch in 32 bits where ``own`` is false, and through the library where it is true.  Sizes are those of the
layers that the library quantizes (256, 2048 x 16384, 4096 x 4096, 14336 x 4096, 18432 x 73728 and the odd 1350 x 677).
"""
from __future__ import annotations

import math

import torch
import torch.nn.functional as F

own = False

DEV = "cuda:0"
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_DEFAULTS = {"op": "linear", "n": 1, "d_in": 256, "d_out": 256, "bits": 4, "group": 0, "x": "bf16", "act": "none", "bias": False,
             "residual": False, "experts": 0, "top_k": 0}


def _case(**kw) -> dict:
    return {**_DEFAULTS, **kw}


def listed() -> list:
    return [
        # one token through the smallest layer: latency alone
        _case(name="token-tiny", d_in=256, d_out=256, bits=4),
        # one token, MLP up-projection of a small model, 3 bits per channel, its activation
        _case(name="token-up", d_in=2048, d_out=16384, bits=3, act="gelu_tanh"),
        # eight requests that decode together, attention projection in 2 bits and groups of 128, added to the residual stream
        _case(name="token-batch", n=8, d_in=4096, d_out=4096, bits=2, group=128, residual=True),
        # one token through the largest layer: the cache-less rate at which packed weights are read
        _case(name="token-largest", d_in=18432, d_out=73728, bits=3, group=128),
        # a ragged batch between decoding and prefill through the down-projection
        _case(name="ragged", n=61, d_in=14336, d_out=4096, bits=4, residual=True),
        # a prompt through the attention projection with bias and residual, 2 bits in groups
        _case(name="prompt", n=2048, d_in=4096, d_out=4096, bits=2, group=128, bias=True, residual=True),
        # calibration rows on their way to the next layer, 3 bits per channel
        _case(name="calibration", n=8192, d_in=2048, d_out=16384, bits=3, act="gelu_tanh"),
        # odd sizes throughout, in fp32
        _case(name="odd-f32", n=333, d_in=1350, d_out=677, bits=3, x="f32", bias=True, act="silu"),
        # a tuning step of the grouped scales of an attention projection
        _case(name="tune-grouped", op="backward", n=2048, d_in=4096, d_out=4096, bits=2, group=128, bias=True),
        # a tuning step of an up-projection with its activation, odd number of rows
        _case(name="tune-up", op="backward", n=1021, d_in=2048, d_out=16384, bits=3, act="silu", bias=True),
        # one token through large experts, two of eight
        _case(name="experts-token", op="moe", d_in=4096, d_out=14336, bits=4, act="silu", experts=8, top_k=2),
        # five tokens through many small experts, eight of 64, 3 bits in groups
        _case(name="experts-many", op="moe", n=5, d_in=2048, d_out=1024, bits=3, group=128, act="silu", experts=64, top_k=8),
    ]


def _log(rng, lo, hi) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng) -> dict:
    op = rng.choice(["linear", "linear", "linear", "backward", "moe"])
    group = rng.choice([0, 0, 32, 64, 128, 128, 256, 96])
    c = _case(op=op, bits=rng.choice([2, 3, 4, 4, 8, rng.randint(1, 8)]), group=group, x=rng.choice(["bf16", "bf16", "bf16", "f32"]),
              act=rng.choice(["none", "none", "relu", "gelu", "gelu_tanh", "silu"]))
    units = lambda v: max(1, round(v / group)) * group if group else v   # noqa: E731
    if op == "moe":
        c["d_in"], c["d_out"] = units(_log(rng, 128, 4096)), units(_log(rng, 128, 4096))
        c["n"] = rng.choice([1, 1, 2, rng.randint(1, 8), rng.randint(1, 32)])
        c["experts"] = _log(rng, 2, 64)
        c["top_k"] = rng.randint(1, min(8, c["experts"]))
        while c["d_in"] * c["d_out"] * c["n"] * c["top_k"] > 2e8 or c["d_in"] * c["d_out"] * c["experts"] > 2e8:
            c["experts"] = max(2, c["experts"] // 2)
            c["top_k"] = max(1, min(c["top_k"], c["experts"]) * 2 // 3)
            c["d_out"] = units(max(64, c["d_out"] // 2))
        return c
    c["bias"], c["residual"] = rng.random() < 0.5, op == "linear" and rng.random() < 0.5
    c["d_in"], c["d_out"] = units(_log(rng, 64, 16384)), _log(rng, 64, 16384)
    most = 2.0e11 / (8 if c["x"] == "f32" else 1) / (4 if op == "backward" else 1)
    c["n"] = min(rng.choice([1, rng.randint(1, 16), _log(rng, 16, 256), _log(rng, 64, 8192)]), max(1, int(most / (c["d_in"] * c["d_out"]))))
    return c


# ---------------------------------------------------------------------------------------------------------------------------------------
# inputs

def _quantized(lead, d_in, d_out, bits, group, gen):
    """Codes, scales and zeros as a min-max grid leaves them on normal weights of variance 1 / d_in: levels bell-shaped around the middle."""
    L, g = 2 ** bits - 1, group or d_in
    ng, sigma = d_in // g, d_in ** -0.5
    Q = torch.empty((*lead, d_in, d_out), dtype=torch.uint8, device=DEV)
    rows = Q.view(-1, d_out)
    step = max(1, (1 << 27) // d_out)
    for r in range(0, rows.shape[0], step):
        z = torch.randn(rows[r:r + step].shape, generator=gen, device=DEV)
        rows[r:r + step] = (z * (L / 6.0) + L / 2.0).round_().clamp_(0, L).to(torch.uint8)
    scale = (6 * sigma / L) * torch.exp(0.1 * torch.randn((*lead, ng, d_out), generator=gen, device=DEV))
    zero = -3 * sigma * (1 + 0.05 * torch.randn((*lead, ng, d_out), generator=gen, device=DEV))
    return Q, scale, zero


def _rows(n, d, dtype, gen):
    """Activations: normal entries, log-normal feature scales."""
    s = torch.exp(0.7 * torch.randn(d, generator=gen, device=DEV))
    return (torch.randn((n, d), generator=gen, device=DEV) * s).to(dtype)


def prepare(case, seed) -> dict:
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dt = _TYPES[case["x"]]
    n, d_in, d_out, bits, group = (case[k] for k in ("n", "d_in", "d_out", "bits", "group"))
    s = {"case": case, "X": _rows(n, d_in, dt, gen)}
    if case["op"] == "moe":
        E = case["experts"]
        s["router"] = (torch.randn((d_in, E), generator=gen, device=DEV) * (2.0 * d_in ** -0.5)).to(dt)
        for part, shape in (("gate", (d_in, d_out)), ("up", (d_in, d_out)), ("down", (d_out, d_in))):
            s[part] = _quantized((E,), *shape, bits, group, gen)
    else:
        s["layer"] = _quantized((), d_in, d_out, bits, group, gen)
        s["bias"] = 0.3 * torch.randn(d_out, generator=gen, device=DEV) if case["bias"] else None
        s["residual"] = _rows(n, d_out, dt, gen) if case["residual"] else None
        if case["op"] == "backward":
            s["dY"] = _rows(n, d_out, dt, gen)
            s["Z"] = torch.randn((n, d_out), generator=gen, device=DEV).to(dt) if case["act"] != "none" else None
    if own:   # a model keeps its weights packed: laid out once, when it is loaded
        from paper_2406_17542_b200 import binding as B
        grid = B.Grid(bits, group)
        if case["op"] == "moe":
            s["experts"] = B.PackedExperts(s["router"], *(B.cdq_pack(s[p][0], grid, s[p][1], s[p][2]) for p in ("gate", "up", "down")))
        else:
            s["packed"] = B.cdq_pack(s["layer"][0], grid, s["layer"][1], s["layer"][2])
    return s


# ---------------------------------------------------------------------------------------------------------------------------------------
# one pass

def _w_hat(Q, scale, zero):
    """W_hat = a * Q + b in 32 bits, groups along the rows."""
    lead, (d_in, d_out), ng = Q.shape[:-2], Q.shape[-2:], scale.shape[-2]
    W = Q.view(*lead, ng, d_in // ng, d_out).float()
    return W.mul_(scale[..., :, None, :]).add_(zero[..., :, None, :]).view(*lead, d_in, d_out)


_GT = math.sqrt(2.0 / math.pi)


def _act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(_GT * (z + 0.044715 * z * z * z)))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    t = torch.tanh(_GT * (z + 0.044715 * z * z * z))
    return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * _GT * (1 + 3 * 0.044715 * z * z)


def _plain_linear(s):
    c = s["case"]
    z = s["X"].float() @ _w_hat(*s["layer"])
    if s["bias"] is not None:
        z += s["bias"]
    y = _act(z, c["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["X"].dtype)


def _plain_backward(s):
    c = s["case"]
    Q, scale, zero = s["layer"]
    dz = s["dY"].float()
    if c["act"] != "none":
        dz = dz * _act_slope(s["Z"].float(), c["act"])
    dX = (dz @ _w_hat(Q, scale, zero).t()).to(s["X"].dtype)
    M = (s["X"].float().t() @ dz).view(scale.shape[0], -1, scale.shape[1])
    dscale = (M * Q.view(M.shape)).sum(1)
    out = {"dX": dX, "dscale": dscale, "dzero": M.sum(1)}
    if s["bias"] is not None:
        out["dbias"] = dz.sum(0)
    return out


def _plain_moe(s):
    c = s["case"]
    X, n, k = s["X"], c["n"], c["top_k"]
    logits = X.double() @ s["router"].double()       # in 64 bits: which experts are chosen hangs on the last digits
    best, ids = torch.sort(logits, dim=1, descending=True, stable=True)
    weights = torch.exp(best[:, :k] - best[:, :1])
    weights = (weights / weights.sum(1, keepdim=True)).float()
    ids = ids[:, :k]
    pairs = ids.reshape(-1)
    x = X.float().repeat_interleave(k, 0)[:, None, :]
    gate = torch.bmm(x, _w_hat(*(t[pairs] for t in s["gate"])))
    up = torch.bmm(x, _w_hat(*(t[pairs] for t in s["up"])))
    h = _act(gate, c["act"]) * up
    y = torch.bmm(h, _w_hat(*(t[pairs] for t in s["down"]))).view(n, k, -1)
    return {"Y": (y * weights[:, :, None]).sum(1).to(X.dtype), "ids": ids.to(torch.int32), "weights": weights}


def run(state):
    c = state["case"]
    if own:
        from paper_2406_17542_b200 import binding as B
        if c["op"] == "linear":
            return B.cdq_linear(state["X"], state["packed"], bias=state["bias"], act=c["act"], residual=state["residual"])
        if c["op"] == "backward":
            got = B.cdq_linear_backward(state["dY"], state["packed"], X=state["X"], Z=state["Z"], act=c["act"], want_bias=c["bias"])
            return {k: v for k, v in got.items() if v is not None}
        Y, ids, weights = B.cdq_moe(state["X"], state["experts"], c["top_k"], act=c["act"])
        return {"Y": Y, "ids": ids, "weights": weights}
    return {"linear": _plain_linear, "backward": _plain_backward, "moe": _plain_moe}[c["op"]](state)


def work(case) -> dict:
    """Bytes: the codes at their bits, scales and zeros, activations in and out, each once.  Flops: two per weight and row."""
    n, d_in, d_out, group = (case[k] for k in ("n", "d_in", "d_out", "group"))
    es = 2 if case["x"] == "bf16" else 4
    w = d_in * d_out
    layer = lambda a, b: a * b * case["bits"] / 8 + 8 * (a // (group or a)) * b   # noqa: E731
    if case["op"] == "moe":
        E, k = case["experts"], case["top_k"]
        active = E * (1 - (1 - k / E) ** n)          # experts that at least one token takes, on average
        return {"bytes": active * (2 * layer(d_in, d_out) + layer(d_out, d_in)) + es * (2 * n * d_in + d_in * E) + 8 * n * k,
                "flops": 2 * n * (3 * k * w + d_in * E)}
    b = layer(d_in, d_out) + es * n * (d_in + d_out) + 4 * d_out * case["bias"]
    if case["op"] == "backward":
        return {"bytes": b + es * n * (d_in + d_out * (case["act"] != "none")) + 8 * (d_in // (group or d_in)) * d_out, "flops": 4.0 * n * w}
    return {"bytes": b + es * n * d_out * case["residual"], "flops": 2.0 * n * w}


# ---------------------------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits

_F64_ACT = {"none": lambda z: z, "relu": F.relu, "silu": F.silu, "gelu": F.gelu, "gelu_tanh": lambda z: F.gelu(z, approximate="tanh")}


def _columns64(layer, j0, j1):
    """Columns [j0, j1) of W_hat in 64 bits, by repeating every group's scale and zero over its rows."""
    Q, scale, zero = (t[:, j0:j1].double() for t in layer)
    per = Q.shape[0] // scale.shape[0]
    return torch.addcmul(zero.repeat_interleave(per, 0), Q, scale.repeat_interleave(per, 0))


def _product64(X, layer, width=4096):
    X = X.double()
    return torch.cat([X @ _columns64(layer, j, j + width) for j in range(0, layer[0].shape[1], width)], 1)


def exact(case, seed):
    s = prepare(case, seed)
    f = _F64_ACT[case["act"]]
    if case["op"] == "linear":
        z = _product64(s["X"], s["layer"])
        z = z if s["bias"] is None else z + s["bias"].double()
        return f(z) if s["residual"] is None else f(z) + s["residual"].double()
    if case["op"] == "backward":
        dz = s["dY"].double()
        if s["Z"] is not None:
            z = s["Z"].double().requires_grad_()
            dz, = torch.autograd.grad(f(z), z, dz)
        Q, scale, zero = s["layer"]
        per = Q.shape[0] // scale.shape[0]
        dX = torch.zeros(s["X"].shape, dtype=torch.float64, device=DEV)
        for j in range(0, Q.shape[1], 4096):
            dX += dz[:, j:j + 4096] @ _columns64(s["layer"], j, j + 4096).t()
        X = s["X"].double()
        dscale, dzero = (torch.empty(scale.shape, dtype=torch.float64, device=DEV) for _ in range(2))
        for t in range(scale.shape[0]):      # a group's scale multiplies the product of its rows' inputs and codes
            rows = slice(t * per, (t + 1) * per)
            dscale[t] = (dz * (X[:, rows] @ Q[rows].double())).sum(0)
            dzero[t] = (dz * X[:, rows].sum(1, keepdim=True)).sum(0)
        out = {"dX": dX, "dscale": dscale, "dzero": dzero}
        if case["bias"]:
            out["dbias"] = dz.sum(0)
        return out
    X, k = s["X"].double(), case["top_k"]
    probs = torch.softmax(X @ s["router"].double(), 1)
    ids = torch.sort(probs, dim=1, descending=True, stable=True).indices[:, :k]
    weights = torch.gather(probs, 1, ids)
    weights = weights / weights.sum(1, keepdim=True)
    Y = torch.zeros_like(X)
    for t in range(case["n"]):
        for e, w in zip(ids[t].tolist(), weights[t]):
            x = X[t:t + 1]
            gate, up = (_product64(x, [v[e] for v in s[p]]) for p in ("gate", "up"))
            Y[t] += w * _product64(f(gate) * up, [v[e] for v in s["down"]])[0]
    return {"Y": Y, "ids": ids.to(torch.int32), "weights": weights}

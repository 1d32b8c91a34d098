"""Timed cases of the experts' feed-forward block as products of its own, with its gradients, and of clipping a step's gradients, through
the package's public entry points.

Rows are sorted by expert, ragged or padded to `capacity` rows per expert.  Four calls make the block: `moe_ffn_up` (both projections, the
activation and its product: g = x W1, u = x W3, h = silu(g) u), `moe_ffn_down` (y = h W2), `moe_ffn_down_backward` (dh = dy W2^T taken
through the activation to dg and du, and dW2 = h^T dy) and `moe_ffn_up_backward` (dx = dg W1^T + du W3^T, dW1 = x^T dg, dW3 = x^T du).
`moe_grad_norm` and `moe_grad_clip` take the norm of many gradients and scale them all to a largest norm.

The plain forms are elementary torch operations in 32 bits, one product per expert that has rows; `exact` is the definition in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

_DEFAULTS = dict(dtype="bf16", T=1, E=128, k=8, d=64, f=64, capacity=0, bias_std=0.5, keep=True, layers=1, limit=1.0)


def _case(**kw):
    return {**_DEFAULTS, **kw}


def listed():
    return [
        # one new token's eight experts: the weights of eight of 128 are read, latency
        _case(name="up_token", op="up", T=1, d=2048, f=768, keep=False),
        # the layer of many small experts, a training micro-batch of 4096 tokens: g and u are kept for the way back
        _case(name="up_prefill", op="up", T=4096, d=2048, f=768),
        # few large experts, the largest batch
        _case(name="up_large", op="up", T=16384, E=8, k=2, d=4096, f=14336, bias_std=0.0),
        # a decode batch: a few rows per expert, all weights are read
        _case(name="down_decode", op="down", T=128, d=2048, f=768),
        # dimensions that are no powers of two
        _case(name="down_odd_dims", op="down", T=4096, k=4, d=2880, f=2880),
        # gradients in a unit test or a reference run
        _case(name="down_grad_small_f32", op="down_grad", dtype="f32", T=256, E=8, k=2, d=512, f=1024, bias_std=0.0),
        # ... of the micro-batch on many small experts
        _case(name="down_grad_prefill", op="down_grad", T=4096, d=2048, f=768),
        # fp32 at odd sizes, rows padded to a capacity that some experts exceed
        _case(name="up_grad_odd_f32", op="up_grad", dtype="f32", T=1001, E=48, k=6, d=1040, f=368, capacity=256),
        # the micro-batch on many small experts
        _case(name="up_grad_prefill", op="up_grad", T=4096, d=2048, f=768),
        # the largest: few large experts
        _case(name="up_grad_large", op="up_grad", T=16384, E=8, k=2, d=4096, f=14336, bias_std=0.0),
        # a small model's gradients, 120 tensors of 8 to 32768 numbers: latency
        _case(name="clip_small", op="clip", E=8, d=64, f=64, layers=24, limit=0.1),
        # two layers of many small experts: what a step of that model clips at a time
        _case(name="clip_large", op="clip", d=2048, f=768, layers=2, limit=0.1),
    ]


def _log_uniform(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    """One more case: 1 to 16384 tokens, 2 to 256 experts, 1 to 16 per token, d from 64 to 7168, f to 14336, both types and layouts."""
    while True:
        op = rng.choice(["up", "down", "down_grad", "up_grad", "clip"])
        dtype = "f32" if rng.random() < 0.25 else "bf16"
        step = 16 if dtype == "f32" else 64
        T, E = _log_uniform(rng, 1, 16384), _log_uniform(rng, 2, 256)
        k = rng.choice([k for k in (1, 2, 3, 4, 6, 8, 8, 11, 16) if k <= E])
        d, f = _log_uniform(rng, 64, 7168, step), _log_uniform(rng, 64, 14336, step)
        if E * d * f > 4.7e8 / (2 if dtype == "f32" else 1):
            continue
        if op == "clip":
            layers = _log_uniform(rng, 1, 48)
            if layers * E * d * f > 4e8 / (2 if dtype == "f32" else 1):
                continue
            return _case(op=op, dtype=dtype, E=E, d=d, f=f, layers=layers, limit=rng.choice([0.01, 0.5, 2.0]))
        if T * k * d * f > 1.9e12 / (8 if dtype == "f32" else 1) or T * k * max(d, f) > 4.7e8:
            continue
        capacity = 0
        if rng.random() < 0.3:
            capacity = min(T, 64 * (int(2 * T * k / E) // 64 + 1))
            if E * capacity > 3 * T * k:
                continue
        return _case(op=op, dtype=dtype, T=T, E=E, k=k, d=d, f=f, capacity=capacity, bias_std=rng.choice([0.0, 0.5, 1.0]),
                     keep=op != "up" or rng.random() < 0.7)


def _rows(case):
    return case["E"] * case["capacity"] if case["capacity"] else case["T"] * case["k"]


def _grad_shapes(case):
    """Shapes and whether they are fp32 of one layer's gradients: gate, its bias, both projections, the way down."""
    E, d, f = case["E"], case["d"], case["f"]
    wide = case["dtype"] == "f32"
    return [((d, E), True), ((E,), True), ((E, d, f), wide), ((E, d, f), wide), ((E, f, d), wide)]


def _views(flat, sizes):
    return list(torch.split(flat, sizes))


def prepare(case, seed):
    T, E, k, d, f, C = (case[n] for n in ("T", "E", "k", "d", "f", "capacity"))
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0, dtype=dt):
        t = torch.empty(shape, dtype=dtype, device="cuda")
        t.normal_(0.0, std, generator=gen)
        return t

    def empty(*shape):
        return torch.empty(shape, dtype=dt, device="cuda")

    s = {"case": case, "dt": dt}
    if case["op"] == "clip":
        # a buffer for each type, a tensor a piece of it: what a program that keeps its gradients together has
        shapes = _grad_shapes(case) * case["layers"]
        s["grads"], s["outs"], s["flat"] = [None] * len(shapes), [None] * len(shapes), []
        for wide, t in ((True, torch.float32), (False, torch.bfloat16)):
            at = [i for i, (_, w) in enumerate(shapes) if w == wide]
            if not at:
                continue
            sizes = [math.prod(shapes[i][0]) for i in at]
            grads = normal(sum(sizes), std=1.0, dtype=t)
            outs = torch.empty_like(grads)
            for i, g, o in zip(at, _views(grads, sizes), _views(outs, sizes)):
                # sizes of gradients differ from tensor to tensor
                g.mul_(10.0 ** (-(i % 5) / 2.0 - 1.0))
                s["grads"][i], s["outs"][i] = g, o
            s["flat"].append(outs)
        total = sum(math.prod(shape) * 100.0 ** (-(i % 5) / 2.0 - 1.0) for i, (shape, _) in enumerate(shapes))
        s["max_norm"] = case["limit"] * math.sqrt(total)  # (the norm is near the square root)
        s["sum"], s["norm"] = torch.empty(1, dtype=torch.float64, device="cuda"), torch.empty(1, device="cuda")
        return s
    # the gate's choices, and the rows of every expert
    top = torch.topk(normal(T, E, dtype=torch.float32) + normal(E, std=max(case["bias_std"], 1e-6), dtype=torch.float32), k, dim=1)
    counts = torch.bincount(top.indices.reshape(-1), minlength=E)
    if C:
        counts = counts.clamp(max=C)
    s["counts"] = counts.to(torch.int32)
    n, spans, at = counts.tolist(), [], 0
    for e in range(E):
        first = e * C if C else at
        if n[e]:
            spans.append((e, first, first + n[e]))
        at += n[e]
    s["spans"] = spans  # (a program that calls torch's products has the experts' rows on the host)
    rows = _rows(case)
    if case["op"] in ("up", "up_grad"):
        s["x"], s["W1"], s["W3"] = normal(rows, d), normal(E, d, f, std=0.02), normal(E, d, f, std=0.02)
    else:
        s["W2"] = normal(E, f, d, std=0.02)
    if case["op"] == "up":
        s["h"] = empty(rows, f)
        s["gu"] = empty(rows, 2 * f) if case["keep"] else None
    elif case["op"] == "down":
        s["h"], s["y"] = normal(rows, f, std=0.3), empty(rows, d)
    elif case["op"] == "down_grad":
        s["dy"], s["gu"] = normal(rows, d), normal(rows, 2 * f)
        g = s["gu"][:, :f].float()
        s["h"] = (g * torch.sigmoid(g) * s["gu"][:, f:].float()).to(dt)
        s["dgu"], s["dW2"] = empty(rows, 2 * f), empty(E, f, d)
    else:
        s["dgu"] = normal(rows, 2 * f)
        s["dx"], s["dW1"], s["dW3"] = empty(rows, d), empty(E, d, f), empty(E, d, f)
    return s


def _plain(s):
    c, dt = s["case"], s["dt"]
    f = c["f"]
    if c["op"] == "clip":
        total = torch.stack([g.float().square().sum(dtype=torch.float64) for g in s["grads"]]).sum()
        norm = torch.sqrt(total)
        factor = torch.clamp(s["max_norm"] / norm, max=1.0)
        for g, o in zip(s["grads"], s["outs"]):
            o.copy_(g.float() * factor)
        return {"norm": norm.float().reshape(1), "grads": s["flat"]}
    if c["op"] == "up":
        h = torch.zeros_like(s["h"])
        gu = torch.zeros_like(s["gu"]) if c["keep"] else None
        for e, a, b in s["spans"]:
            x = s["x"][a:b].float()
            g, u = x @ s["W1"][e].float(), x @ s["W3"][e].float()
            h[a:b] = (g / (1.0 + torch.exp(-g)) * u).to(dt)
            if c["keep"]:
                gu[a:b, :f], gu[a:b, f:] = g.to(dt), u.to(dt)
        return {"h": h, "gu": gu} if c["keep"] else {"h": h}
    if c["op"] == "down":
        y = torch.zeros_like(s["y"])
        for e, a, b in s["spans"]:
            y[a:b] = (s["h"][a:b].float() @ s["W2"][e].float()).to(dt)
        return {"y": y}
    if c["op"] == "down_grad":
        dgu, dW2 = torch.zeros_like(s["dgu"]), torch.zeros_like(s["dW2"])
        for e, a, b in s["spans"]:
            dy, gu = s["dy"][a:b].float(), s["gu"][a:b].float()
            g, u = gu[:, :f], gu[:, f:]
            dh = dy @ s["W2"][e].float().t()
            sig = 1.0 / (1.0 + torch.exp(-g))
            dgu[a:b, :f], dgu[a:b, f:] = (dh * u * sig * (1.0 + g * (1.0 - sig))).to(dt), (dh * g * sig).to(dt)
            dW2[e] = (s["h"][a:b].float().t() @ dy).to(dt)
        return {"dgu": dgu, "dW2": dW2}
    dx, dW1, dW3 = torch.zeros_like(s["dx"]), torch.zeros_like(s["dW1"]), torch.zeros_like(s["dW3"])
    for e, a, b in s["spans"]:
        x, dg, du = s["x"][a:b].float(), s["dgu"][a:b, :f].float(), s["dgu"][a:b, f:].float()
        dx[a:b] = (dg @ s["W1"][e].float().t() + du @ s["W3"][e].float().t()).to(dt)
        dW1[e], dW3[e] = (x.t() @ dg).to(dt), (x.t() @ du).to(dt)
    return {"dx": dx, "dW1": dW1, "dW3": dW3}


def _framework(s):
    from paper_2605_00686_amd import binding as B
    c, f = s["case"], s["case"]["f"]
    if c["op"] == "clip":
        if "list" not in s:  # the list and the workspace that a program keeps
            s["list"] = B.tensor_list(s["grads"], s["outs"])
            s["workspace"] = torch.empty(B.moe_grad_workspace_bytes(s["list"]), dtype=torch.uint8, device="cuda")
        B.moe_grad_norm(s["list"], s["sum"], s["norm"], s["workspace"])
        B.moe_grad_clip(s["list"], s["sum"], s["max_norm"])
        return {"norm": s["norm"], "grads": s["flat"]}
    if "p" not in s:  # the problem and the workspace that a program keeps
        s["p"] = B.problem(c["T"], c["d"], c["E"], c["k"], f, 1, s["dt"], capacity=c["capacity"])
        s["workspace"] = torch.empty(B.moe_ffn_workspace_bytes(s["p"]), dtype=torch.uint8, device="cuda")
    p, counts, ws = s["p"], s["counts"], s["workspace"]
    if c["op"] == "up":
        gu = s["gu"]
        B.moe_ffn_up(p, s["x"], s["W1"], s["W3"], counts, gu[:, :f] if c["keep"] else None, gu[:, f:] if c["keep"] else None, s["h"], ws)
        return {"h": s["h"], "gu": gu} if c["keep"] else {"h": s["h"]}
    if c["op"] == "down":
        B.moe_ffn_down(p, s["h"], s["W2"], counts, s["y"], ws)
        return {"y": s["y"]}
    if c["op"] == "down_grad":
        B.moe_ffn_down_backward(p, s["dy"], s["W2"], s["h"], s["gu"][:, :f], s["gu"][:, f:], counts, None, s["dgu"][:, :f], s["dgu"][:, f:],
                                s["dW2"], ws)
        return {"dgu": s["dgu"], "dW2": s["dW2"]}
    B.moe_ffn_up_backward(p, s["x"], s["W1"], s["W3"], s["dgu"][:, :f], s["dgu"][:, f:], counts, s["dx"], s["dW1"], s["dW3"], ws)
    return {"dx": s["dx"], "dW1": s["dW1"], "dW3": s["dW3"]}


def run(s):
    if own:
        return _framework(s)
    return _plain(s)


def work(case):
    T, E, k, d, f = (case[n] for n in ("T", "E", "k", "d", "f"))
    N, rows, sz = T * k, _rows(case), 4 if case["dtype"] == "f32" else 2
    if case["op"] == "clip":
        shapes = _grad_shapes(case) * case["layers"]
        return {"bytes": sum(2 * math.prod(shape) * (4 if wide else 2) for shape, wide in shapes), "flops": sum(3 * math.prod(shape) for shape, _ in shapes)}
    N = min(N, rows)
    used = E * (1.0 - (1.0 - k / E) ** T)  # experts that have rows, about
    matrix = d * f * sz
    if case["op"] == "up":
        return {"bytes": N * d * sz + 2 * used * matrix + rows * f * sz * (3 if case["keep"] else 1), "flops": 4 * N * d * f}
    if case["op"] == "down":
        return {"bytes": N * f * sz + used * matrix + rows * d * sz, "flops": 2 * N * d * f}
    if case["op"] == "down_grad":
        return {"bytes": (N * d + 3 * N * f + 2 * rows * f) * sz + (used + E) * matrix, "flops": 4 * N * d * f}
    return {"bytes": (N * d + 2 * N * f + rows * d) * sz + 2 * (used + E) * matrix, "flops": 8 * N * d * f}


def exact(case, seed):
    """The definitions, in 64 bits; every row by the expert that has it."""
    s = prepare(case, seed)
    E, d, f, C, op = (case[n] for n in ("E", "d", "f", "capacity", "op"))
    if op == "clip":
        norm = math.sqrt(math.fsum(float(torch.linalg.vecdot(part, part)) for g in s["grads"] for part in (c.double() for c in g.split(1 << 26))))
        factor = min(1.0, s["max_norm"] / norm)
        for flat in s["flat"]:
            flat.zero_()
        wide = {t: [g.double() * factor for g in s["grads"] if g.dtype == t] for t in (torch.float32, torch.bfloat16)}
        return {"norm": torch.tensor([norm], dtype=torch.float64), "grads": [torch.cat(v) for v in wide.values() if v]}
    end = torch.cumsum(s["counts"].long(), 0)
    rows = _rows(case)
    r = torch.arange(rows, device="cuda")
    expert = r // C if C else torch.searchsorted(end, r, right=True)
    used = (r - expert * C < s["counts"].long()[expert]) if C else r < end[-1]
    of = [((expert == e) & used).nonzero()[:, 0] for e in range(E)]

    def zeros(*shape):
        return torch.zeros(shape, dtype=torch.float64, device="cuda")
    if op == "up":
        out = {"h": zeros(rows, f), "gu": zeros(rows, 2 * f)}
        for e, i in enumerate(of):
            gu = s["x"].index_select(0, i).double() @ torch.cat([s["W1"][e], s["W3"][e]], 1).double()
            g, u = gu.chunk(2, 1)
            out["h"][i] = u * g * torch.sigmoid(g)
            out["gu"][i] = gu
        return out if case["keep"] else {"h": out["h"]}
    if op == "down":
        y = zeros(rows, d)
        for e, i in enumerate(of):
            y[i] = torch.mm(s["h"].index_select(0, i).double(), s["W2"][e].double())
        return {"y": y}
    if op == "down_grad":
        dgu, dW2 = zeros(rows, 2 * f), zeros(E, f, d)
        for e, i in enumerate(of):
            dy = s["dy"].index_select(0, i).double()
            g, u = s["gu"].index_select(0, i).double().chunk(2, 1)
            dh = torch.mm(s["W2"][e].double(), dy.t()).t()
            silu = g * torch.sigmoid(g)
            dgu[i] = torch.cat([dh * u * (torch.sigmoid(g) + silu * torch.sigmoid(-g)), dh * silu], 1)
            dW2[e] = torch.mm(dy.t(), s["h"].index_select(0, i).double()).t()
        return {"dgu": dgu, "dW2": dW2}
    dx, dW1, dW3 = zeros(rows, d), zeros(E, d, f), zeros(E, d, f)
    for e, i in enumerate(of):
        x, dgu = s["x"].index_select(0, i).double(), s["dgu"].index_select(0, i).double()
        dx[i] = torch.mm(dgu, torch.cat([s["W1"][e], s["W3"][e]], 1).double().t())
        dW1[e], dW3[e] = torch.mm(x.t(), dgu).chunk(2, 1)
    return {"dx": dx, "dW1": dW1, "dW3": dW3}

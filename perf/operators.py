"""Timed cases of training the MoE layer around a program's own expert products, through the package's public entry points.

Five calls: rows sorted by expert back to their tokens (`moe_unsort`: the forward pass's end, and without weights the gradient of the
sort), the gradient of that with respect to rows and weights (`moe_unsort_backward`), the gradient of the gate (`moe_route_backward`),
and the experts' SwiGLU with its inputs kept in 8 bits (`moe_swiglu`) and its gradient from them (`moe_swiglu_backward`).

The plain forms are elementary torch operations in 32 bits; `exact` is the definition in 64 bits.  Rows sorted by expert are
ragged, or padded to `capacity` rows per expert; slots that an expert has no room for have no row (-1) there.
"""
from __future__ import annotations

import math

import torch

own = False

_DEFAULTS = dict(dtype="bf16", E=128, k=8, d=64, f=64, capacity=0, bias_std=0.5, weighted=True, addend=False)
_BLOCK = 32  # values that share a scale


def _case(**kw):
    return {**_DEFAULTS, **kw}


def listed():
    return [
        # one new token's eight expert rows are added up: latency
        _case(name="unsort_token", op="unsort", T=1, d=2048),
        # the forward pass's end on the layer of many small experts, 4096 tokens
        _case(name="unsort_prefill", op="unsort", T=4096, d=2048),
        # the gradient of the sort, added to the gate's: few large experts, the largest batch
        _case(name="sort_grad_large", op="unsort", T=16384, d=4096, E=8, k=2, bias_std=0.0, weighted=False, addend=True),
        # gradients of 4096 tokens' expert rows and of their weights
        _case(name="unsort_grad_prefill", op="unsort_grad", T=4096, d=2048),
        # the same in fp32 at odd sizes, rows padded to a capacity that some experts exceed
        _case(name="unsort_grad_odd_f32", op="unsort_grad", dtype="f32", T=1001, d=1040, E=48, k=6, capacity=256),
        # the gate's gradient in a unit test or a reference run
        _case(name="gate_grad_tiny_f32", op="gate_grad", dtype="f32", T=256, d=512, E=8, k=2, bias_std=0.0),
        # ... on the layer of many small experts
        _case(name="gate_grad_prefill", op="gate_grad", T=4096, d=2048),
        # ... and of a wide layer with all its experts
        _case(name="gate_grad_wide", op="gate_grad", T=2048, d=7168, E=256),
        # a short batch at odd sizes, padded rows
        _case(name="swiglu_odd", op="swiglu", T=1001, E=48, k=6, f=1408, capacity=256),
        # the experts' activations of 4096 tokens x 8
        _case(name="swiglu_prefill", op="swiglu", T=4096, f=768),
        # a micro-batch's gradient in fp32
        _case(name="swiglu_grad_small_f32", op="swiglu_grad", dtype="f32", T=256, E=8, k=2, f=1024, bias_std=0.0),
        # the largest: few large experts
        _case(name="swiglu_grad_large", op="swiglu_grad", T=16384, E=8, k=2, f=14336, bias_std=0.0),
    ]


def _log_uniform(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    """One more case: 1 to 16384 tokens, 2 to 256 experts, 1 to 16 per token, d from 64 to 7168, f to 14336, both types and layouts."""
    while True:
        op = rng.choice(["unsort", "unsort_grad", "gate_grad", "swiglu", "swiglu_grad"])
        dtype = "f32" if rng.random() < 0.25 else "bf16"
        step = 16 if dtype == "f32" else 64
        T, E = _log_uniform(rng, 1, 16384), _log_uniform(rng, 2, 256)
        # (one expert per token has weight one whatever its logit: no gradient for the gate)
        k = rng.choice([k for k in (1, 2, 3, 4, 6, 8, 8, 11, 16) if k <= E and (k > 1 or op != "gate_grad")])
        d = _log_uniform(rng, 64, 7168, step) if not op.startswith("swiglu") else 64
        f = _log_uniform(rng, 64, 14336, step) if op.startswith("swiglu") else 64
        if T * k * max(d, f) > (4.6e8 if op.startswith("swiglu") else 1.4e8) / (2 if dtype == "f32" else 1):
            continue
        capacity = 0
        if op != "gate_grad" and rng.random() < 0.3:
            capacity = min(T, 64 * (int(2 * T * k / E) // 64 + 1))
            if E * capacity > 3 * T * k:
                continue
        weighted = op != "unsort" or rng.random() < 0.6
        return _case(op=op, dtype=dtype, T=T, E=E, k=k, d=d, f=f, capacity=capacity, bias_std=rng.choice([0.0, 0.5, 1.0]),
                     weighted=weighted, addend=op == "unsort" and not weighted)


def _rows(case):
    return case["E"] * case["capacity"] if case["capacity"] else case["T"] * case["k"]


def _power_of_two(e):
    """2 to the e as fp32, from the bits of whole numbers e in [-126, 127]."""
    return ((e + 127) << 23).view(torch.float32)


def _exponents(x):
    """The power of two of every block of 32 values (of the last one of 16, where a row ends there): the least that brings them to 448."""
    b = torch.nn.functional.pad(x, (0, -x.shape[1] % _BLOCK)).reshape(x.shape[0], -1, _BLOCK)
    most = b.abs().amax(-1)
    m, a = torch.frexp(most)
    e = a.to(torch.int32) - 9 + (m > 0.875).to(torch.int32)
    return torch.where(most > 0, e, -127).clamp(min=-127)


def _spread(e, n):
    return e.repeat_interleave(_BLOCK, 1)[:, :n]


def _encode(x):
    """fp32 [rows, f] -> codes (float8_e4m3fn) and the powers of two of their blocks (float8_e8m0fnu)."""
    e = _exponents(x)
    codes = (x * _power_of_two(_spread(-e, x.shape[1]))).to(torch.float8_e4m3fn)
    return codes, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def prepare(case, seed):
    T, E, k, d, f, C = (case[n] for n in ("T", "E", "k", "d", "f", "capacity"))
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0, dtype=dt):
        t = torch.empty(shape, dtype=dtype, device="cuda")
        t.normal_(0.0, std, generator=gen)
        return t

    s = {"case": case, "dt": dt}
    rows = _rows(case)
    # the gate's choices, and where the sort puts every slot
    top = torch.topk(normal(T, E, dtype=torch.float32) + normal(E, std=max(case["bias_std"], 1e-6), dtype=torch.float32), k, dim=1)
    s["idx"] = top.indices.to(torch.int32).contiguous()
    s["w"] = torch.softmax(top.values, 1).contiguous()
    flat = s["idx"].reshape(-1).long()
    order = torch.argsort(flat, stable=True)
    place = torch.empty_like(order)
    place[order] = torch.arange(T * k, device="cuda")
    counts = torch.bincount(flat, minlength=E)
    if C:
        rank = place - (torch.cumsum(counts, 0) - counts)[flat]
        place = torch.where(rank < C, flat * C + rank, -1)
        counts = counts.clamp(max=C)
        s["used"] = (torch.arange(C, device="cuda")[None, :] < counts[:, None]).reshape(-1)
    s["inv_perm"], s["counts"] = place.to(torch.int32), counts.to(torch.int32)
    if case["op"] in ("unsort", "unsort_grad"):
        s["rows"] = normal(rows, d, std=0.5)
        s["addend"] = normal(T, d) if case["addend"] else None
        if case["op"] == "unsort":
            s["out"] = torch.empty((T, d), dtype=dt, device="cuda")
        else:
            s["dout"] = normal(T, d)
            s["drows"] = torch.empty((rows, d), dtype=dt, device="cuda")
            s["dw"] = torch.empty((T, k), dtype=torch.float32, device="cuda")
    elif case["op"] == "gate_grad":
        s["x"], s["Wg"], s["dw"] = normal(T, d), normal(d, E, std=0.02), normal(T, k, dtype=torch.float32)
        s["dx"] = torch.empty((T, d), dtype=dt, device="cuda")
        s["dWg"] = torch.empty((d, E), dtype=torch.float32, device="cuda")
        s["dbias"] = torch.empty(E, dtype=torch.float32, device="cuda")
    else:
        # one product gives both halves of a row, side by side; columns differ in size as a trained layer's do
        gu = normal(rows, 2 * f)
        gu *= torch.exp(normal(2 * f, std=0.5, dtype=torch.float32)).to(dt)
        if case["op"] == "swiglu":
            s["gu"] = gu
            s["h"] = torch.empty((rows, f), dtype=dt, device="cuda")
            s["codes"] = torch.empty((rows, 2, f), dtype=torch.uint8, device="cuda")
            s["scales"] = torch.empty((rows, 2, -(-f // _BLOCK)), dtype=torch.uint8, device="cuda")
        else:
            codes, scales = _encode(gu.float().reshape(rows * 2, f))
            s["codes"] = codes.view(torch.uint8).reshape(rows, 2, f)
            s["scales"] = scales.view(torch.uint8).reshape(rows, 2, -1)
            del gu, codes, scales
            s["dh"] = normal(rows, f)
            s["dgu"] = torch.empty((rows, 2 * f), dtype=dt, device="cuda")
            s["h"] = torch.empty((rows, f), dtype=dt, device="cuda")
        if C:
            s["codes"][~s["used"]] = 0
            s["scales"][~s["used"]] = 0
    return s


def _gathered(s, rows):
    """fp32 [T, k, d]: the row of every slot, zero where it has none."""
    inv = s["inv_perm"].long()
    got = rows.float()[inv.clamp(min=0)]
    if s["case"]["capacity"]:
        got = torch.where((inv >= 0)[:, None], got, 0.0)
    return got.reshape(s["case"]["T"], s["case"]["k"], -1)


def _plain(s):
    c = s["case"]
    T, E, k, f, C, dt = c["T"], c["E"], c["k"], c["f"], c["capacity"], s["dt"]
    if c["op"] == "unsort":
        out = _gathered(s, s["rows"])
        out = (out * s["w"][:, :, None] if c["weighted"] else out).sum(1)
        return {"out": (out + s["addend"].float() if c["addend"] else out).to(dt)}
    if c["op"] == "unsort_grad":
        dout, inv = s["dout"].float(), s["inv_perm"].long()
        dw = (_gathered(s, s["rows"]) * dout[:, None]).sum(-1)
        drows = torch.zeros((_rows(c) + 1, c["d"]), dtype=dt, device=dout.device)  # (the last: slots without a row)
        drows[torch.where(inv >= 0, inv, _rows(c))] = (s["w"][:, :, None] * dout[:, None]).reshape(T * k, -1).to(dt)
        return {"drows": drows[:-1], "dw": dw}
    if c["op"] == "gate_grad":
        dl = s["w"] * (s["dw"] - (s["w"] * s["dw"]).sum(1, keepdim=True))
        dense = torch.zeros((T, E), dtype=torch.float32, device=dl.device).scatter_(1, s["idx"].long(), dl)
        return {"dx": (dense @ s["Wg"].float().t()).to(dt), "dWg": s["x"].float().t() @ dense, "dbias": dense.sum(0)}
    if c["op"] == "swiglu":
        gu = s["gu"].float()
        if C:
            gu = torch.where(s["used"][:, None], gu, 0.0)
        g, u = gu[:, :f], gu[:, f:]
        codes, scales = _encode(gu.reshape(-1, f))
        return {"h": (g / (1.0 + torch.exp(-g)) * u).to(dt), "codes": codes.reshape(-1, 2, f), "scales": scales.reshape(codes.shape[0] // 2, 2, -1)}
    e = s["scales"].to(torch.int32) - 127
    # (two factors: the power of an empty block lies below fp32's normal numbers)
    low = e.clamp(min=-64)
    scale = (_power_of_two(low) * _power_of_two(e - low)).repeat_interleave(_BLOCK, 2)[:, :, :f]
    gu = s["codes"].view(torch.float8_e4m3fn).float() * scale
    g, u, dh = gu[:, 0], gu[:, 1], s["dh"].float()
    if C:
        dh = torch.where(s["used"][:, None], dh, 0.0)
    sig = 1.0 / (1.0 + torch.exp(-g))
    return {"dgu": torch.cat([dh * u * sig * (1.0 + g * (1.0 - sig)), dh * g * sig], 1).to(dt), "h": (g * sig * u).to(dt)}


def _framework(s):
    from paper_2605_00686_amd import binding as B
    c = s["case"]
    if "p" not in s:  # the problem and the workspace that a program keeps
        s["p"] = B.problem(c["T"], c["d"], c["E"], c["k"], c["f"], 1, s["dt"], capacity=c["capacity"])
        s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
        if c["op"] == "gate_grad":
            s["workspace"] = torch.empty(max(256, B.moe_backward_workspace_bytes(s["p"])), dtype=torch.uint8, device="cuda")
    p, f, counts = s["p"], c["f"], s["counts"] if c["capacity"] else None
    if c["op"] == "unsort":
        B.moe_unsort(p, s["rows"], s["inv_perm"], s["w"] if c["weighted"] else None, s["addend"], s["out"], s["status"])
        return {"out": s["out"]}
    if c["op"] == "unsort_grad":
        B.moe_unsort_backward(p, s["dout"], s["rows"], s["inv_perm"], s["w"], counts, s["drows"], s["dw"], s["status"])
        return {"drows": s["drows"], "dw": s["dw"]}
    if c["op"] == "gate_grad":
        B.moe_route_backward(p, s["x"], s["Wg"], s["idx"], s["w"], s["dw"], s["dx"], s["dWg"], s["dbias"], s["status"], s["workspace"])
        return {"dx": s["dx"], "dWg": s["dWg"], "dbias": s["dbias"]}
    if c["op"] == "swiglu":
        B.moe_swiglu(p, s["gu"][:, :f], s["gu"][:, f:], counts, s["h"], s["codes"], s["scales"])
        return {"h": s["h"], "codes": s["codes"].view(torch.float8_e4m3fn), "scales": s["scales"].view(torch.float8_e8m0fnu)}
    B.moe_swiglu_backward(p, s["dh"], s["codes"], s["scales"], counts, s["dgu"][:, :f], s["dgu"][:, f:], s["h"])
    return {"dgu": s["dgu"], "h": s["h"]}


def run(s):
    if own:
        return _framework(s)
    return _plain(s)


def work(case):
    T, E, k, d, f = (case[n] for n in ("T", "E", "k", "d", "f"))
    N, rows, sz = T * k, _rows(case), 4 if case["dtype"] == "f32" else 2
    kept = 2 * (f + -(-f // _BLOCK))  # bytes of a row in 8 bits, both halves
    if case["op"] == "unsort":
        return {"bytes": (N + T + T * case["addend"]) * d * sz + N * (4 + 4 * case["weighted"]), "flops": 2 * N * d}
    if case["op"] == "unsort_grad":
        return {"bytes": (T + N + rows) * d * sz + 12 * N, "flops": 3 * N * d}
    if case["op"] == "gate_grad":
        return {"bytes": 2 * T * d * sz + d * E * (sz + 4) + 12 * N + 4 * E, "flops": 4 * N * d}
    used = N if not case["capacity"] else min(N, rows)
    if case["op"] == "swiglu":
        return {"bytes": used * 2 * f * sz + rows * (f * sz + kept), "flops": 12 * used * f}
    return {"bytes": used * (f * sz + kept) + rows * 3 * f * sz, "flops": 14 * used * f}


def exact(case, seed):
    """The definitions, in 64 bits; sums over slots and experts one choice after the other."""
    s = prepare(case, seed)
    T, E, k, f, op = (case[n] for n in ("T", "E", "k", "f", "op"))
    w, inv, idx = s["w"].double(), s["inv_perm"].long().reshape(T, k), s["idx"].long()
    has = inv >= 0
    if op == "unsort":
        out = s["addend"].double() if case["addend"] else torch.zeros_like(s["out"], dtype=torch.float64)
        for j in range(k):
            row = s["rows"][inv[:, j].clamp(min=0)].double().masked_fill(~has[:, j, None], 0.0)
            out = out + (w[:, j, None] * row if case["weighted"] else row)
        return {"out": out}
    if op == "unsort_grad":
        dout = s["dout"].double()
        drows, dw = torch.zeros_like(s["drows"], dtype=torch.float64), torch.zeros_like(w)
        for j in range(k):
            at = has[:, j].nonzero()[:, 0]
            to = inv[at, j]
            drows[to] = w[at, j, None] * dout[at]
            dw[at, j] = torch.linalg.vecdot(s["rows"][to].double(), dout[at])
        return {"drows": drows, "dw": dw}
    if op == "gate_grad":
        x, W, dw = s["x"].double(), s["Wg"].double(), s["dw"].double()
        dx, dWg, dbias = torch.zeros_like(x), torch.zeros_like(W), torch.zeros(E, dtype=torch.float64, device=x.device)
        mean = torch.linalg.vecdot(w, dw)
        for j in range(k):
            dl = w[:, j] * (dw[:, j] - mean)
            dx.addcmul_(W.t()[idx[:, j]], dl[:, None])
            dbias.index_add_(0, idx[:, j], dl)
        for e in range(E):
            t, j = (idx == e).nonzero(as_tuple=True)
            dWg[:, e] = (w[t, j] * (dw[t, j] - mean[t])) @ x[t]
        return {"dx": dx, "dWg": dWg, "dbias": dbias}
    used = s["used"][:, None].double() if case["capacity"] else 1.0
    if op == "swiglu":
        gu = (s["gu"].double() * used).reshape(-1, 2, f)
        g, u = gu[:, 0], gu[:, 1]
        h = g * torch.sigmoid(g) * u
        scales = torch.empty(s["scales"].shape, dtype=torch.float64, device=gu.device)
        codes = torch.empty_like(gu)
        for b in range(scales.shape[2]):
            part = gu[:, :, b * _BLOCK:(b + 1) * _BLOCK]
            # the least power of two that all values of the block, divided by it, stay within 448
            scale = torch.exp2(torch.ceil(torch.log2(part.abs().amax(-1).clamp(min=2.0 ** -119) / 448.0)))
            scale = torch.where(part.abs().amax(-1) > 448.0 * scale, 2.0 * scale, scale).clamp(min=2.0 ** -127)
            scale = torch.where(part.abs().amax(-1) > 0, scale, 2.0 ** -127)
            v = part / scale[:, :, None]
            # three bits behind the leading one, at least in steps of 2^-9; halves go to the even one
            step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3.0)
            codes[:, :, b * _BLOCK:(b + 1) * _BLOCK], scales[:, :, b] = torch.round(v / step) * step, scale
        return {"h": h, "codes": codes, "scales": scales}
    value = s["codes"].view(torch.float8_e4m3fn).double()
    value *= torch.exp2(s["scales"].double() - 127.0).repeat_interleave(_BLOCK, 2)[:, :, :f]
    g, u, dh = value[:, 0], value[:, 1], s["dh"].double() * used
    sig = torch.sigmoid(g)
    silu = g * sig
    return {"dgu": torch.cat([dh * u * (sig + silu * (1.0 - sig)), dh * silu], 1), "h": silu * u}

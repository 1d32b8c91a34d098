#!/usr/bin/env python3
"""Trains one MoE layer, with a residual connection, to follow another of the same shape: the gate, the sort, the experts' activation and
the way back are this package's calls, forward and backward; the experts' matrix products are torch's.  What a step keeps of the
experts' inputs g and u is 8 bits a number.

  python examples/train_layer.py [--tokens T] [--dim d] [--experts E] [--top-k k] [--ffn f] [--dtype bf16|f32] [--steps N] [--lr R]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2605_00686_amd import binding as B  # noqa: E402


class Layer:
    """out = x + sum_j w[t,j] expert_j(x); parameters Wg [d,E], bias [E] (fp32), W13 [E,d,2f] (W1 and W3 side by side), W2 [E,f,d]."""

    def __init__(self, T, d, E, k, f, dtype, seed=0):
        self.p = B.problem(T, d, E, k, f, 1, dtype)
        self.T, self.d, self.E, self.k, self.f, self.dtype = T, d, E, k, f, dtype
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, std):
            return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)
        self.Wg, self.bias = normal(d, E, std=d ** -0.5), torch.zeros(E, device="cuda")
        self.W13, self.W2 = normal(E, d, 2 * f, std=d ** -0.5), normal(E, f, d, std=f ** -0.5)
        N = T * k

        def empty(*shape, dtype=dtype):
            return torch.empty(shape, dtype=dtype, device="cuda")
        i32 = torch.int32
        self.idx, self.w = empty(T, k, dtype=i32), empty(T, k, dtype=torch.float32)
        self.counts, self.offsets = empty(E, dtype=i32), empty(E + 1, dtype=i32)
        self.perm, self.inv_perm = empty(N, dtype=i32), empty(N, dtype=i32)
        self.x_perm, self.gu, self.h, self.y = empty(N, d), empty(N, 2 * f), empty(N, f), empty(N, d)
        self.codes, self.scales = empty(N, 2, f, dtype=torch.uint8), empty(N, 2, -(-f // 32), dtype=torch.uint8)
        self.out, self.dx, self.dw = empty(T, d), empty(T, d), empty(T, k, dtype=torch.float32)
        self.dWg, self.dbias = empty(d, E, dtype=torch.float32), empty(E, dtype=torch.float32)
        self.dW13, self.dW2 = torch.zeros_like(self.W13), torch.zeros_like(self.W2)
        self.status = torch.zeros(1, dtype=i32, device="cuda")
        self.workspace = empty(B.moe_workspace_bytes(self.p), dtype=torch.uint8)
        B.moe_workspace_init(self.p, self.workspace)
        self.grad_workspace = empty(max(256, B.moe_backward_workspace_bytes(self.p)), dtype=torch.uint8)

    def _experts(self):
        """(expert, its rows) of those that have any."""
        ends = self.offsets.tolist()
        return [(e, slice(ends[e], ends[e + 1])) for e in range(self.E) if ends[e + 1] > ends[e]]

    def forward(self, x):
        p, f = self.p, self.f
        B.moe_route(p, x, self.Wg, self.bias, self.idx, self.w)
        B.moe_dispatch(p, x, self.idx, self.counts, self.offsets, self.perm, self.inv_perm, self.x_perm, self.status, self.workspace)
        self.rows = self._experts()
        for e, r in self.rows:
            torch.mm(self.x_perm[r], self.W13[e], out=self.gu[r])
        B.moe_swiglu(p, self.gu[:, :f], self.gu[:, f:], None, self.h, self.codes, self.scales)
        for e, r in self.rows:
            torch.mm(self.h[r], self.W2[e], out=self.y[r])
        # (from here on gu and h are free: the backward pass reads the codes, and writes both anew)
        B.moe_unsort(p, self.y, self.inv_perm, self.w, x, self.out, self.status)
        self.x = x
        return self.out

    def backward(self, dout):
        """Gradients of the parameters (dWg, dbias, dW13, dW2) and of x, which is returned."""
        p, f = self.p, self.f
        B.moe_unsort_backward(p, dout, self.y, self.inv_perm, self.w, None, self.y, self.dw, self.status)  # y becomes dy
        dh = torch.empty_like(self.h)
        for e, r in self.rows:
            torch.mm(self.y[r], self.W2[e].t(), out=dh[r])
        B.moe_swiglu_backward(p, dh, self.codes, self.scales, None, self.gu[:, :f], self.gu[:, f:], self.h)
        self.dW13.zero_()
        self.dW2.zero_()
        dx_perm = torch.empty_like(self.x_perm)
        for e, r in self.rows:
            torch.mm(self.h[r].t(), self.y[r], out=self.dW2[e])
            torch.mm(self.x_perm[r].t(), self.gu[r], out=self.dW13[e])
            torch.mm(self.gu[r], self.W13[e].t(), out=dx_perm[r])
        B.moe_route_backward(p, self.x, self.Wg, self.idx, self.w, self.dw, self.dx, self.dWg, self.dbias, self.status, self.grad_workspace)
        B.moe_unsort(p, dx_perm, self.inv_perm, None, self.dx, self.dx, self.status)
        return self.dx.add_(dout)

    def step(self, lr):
        for value, grad in ((self.Wg, self.dWg), (self.bias, self.dbias), (self.W13, self.dW13), (self.W2, self.dW2)):
            value.add_(grad.to(value.dtype), alpha=-lr)

    def check(self):
        """What the calls had to report, once the device is done with them."""
        status = int(self.status.item())
        if status:
            raise B.MoeError(status, "layer")


def train(T=1024, d=256, E=16, k=2, f=512, dtype=torch.bfloat16, steps=50, lr=100.0, seed=0, say=None):
    teacher, layer = Layer(T, d, E, k, f, dtype, seed + 1), Layer(T, d, E, k, f, dtype, seed + 2)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    losses = []
    for i in range(steps):
        x = torch.randn((T, d), generator=gen, device="cuda").to(dtype)
        target = teacher.forward(x).clone()
        diff = layer.forward(x).float() - target.float()
        losses.append(diff.square().mean())
        layer.backward((diff * (2.0 / diff.numel())).to(dtype))
        layer.step(lr)
        if say and (i % 10 == 0 or i == steps - 1):
            say(f"step {i}: mean squared difference {float(losses[-1]):.4f}")
    layer.check()
    teacher.check()
    return [float(v) for v in losses]


def main():
    a = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("--tokens", 1024), ("--dim", 256), ("--experts", 16), ("--top-k", 2), ("--ffn", 512), ("--steps", 50)):
        a.add_argument(name, type=int, default=value)
    a.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    a.add_argument("--lr", type=float, default=100.0)
    o = a.parse_args()
    train(o.tokens, o.dim, o.experts, o.top_k, o.ffn, torch.float32 if o.dtype == "f32" else torch.bfloat16, o.steps, o.lr, say=print)


if __name__ == "__main__":
    main()

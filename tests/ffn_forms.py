"""What the tests of the experts' products share: rows of experts, the definitions in 64 bits on the CPU, and what rounding may move."""
import torch

from tests.train_forms import HALF_STEP, dtype_of, routing

# (T, E, k, d, f, capacity, dtype): one token; few, dozens and hundreds of rows per expert; lengths of no round number; experts without rows; padded
# rows, some with a capacity that experts exceed or that ends inside a row block
SHAPES = [
    (1, 8, 2, 64, 64, 0, "bf16"), (1, 256, 1, 64, 128, 0, "bf16"), (1, 1, 1, 64, 64, 0, "f32"), (3, 200, 3, 128, 320, 0, "bf16"),
    (40, 8, 2, 192, 448, 0, "bf16"), (200, 6, 2, 320, 192, 0, "bf16"), (517, 4, 2, 192, 320, 0, "bf16"), (700, 2, 1, 576, 640, 0, "bf16"),
    (1030, 3, 2, 64, 64, 0, "bf16"), (100, 6, 3, 128, 64, 48, "bf16"), (333, 5, 2, 192, 128, 200, "bf16"), (400, 3, 3, 128, 192, 300, "bf16"),
    (40, 8, 2, 48, 80, 0, "f32"), (301, 4, 2, 144, 208, 0, "f32"), (150, 6, 3, 80, 272, 72, "f32"), (2, 3, 2, 16, 16, 0, "f32"),
]


class Rows:
    """Rows sorted by expert: `of[e]` the numbers of expert e's, `used` which are anybody's."""

    def __init__(self, gen, T, E, k, d, f, capacity, dtype, skew=1.0, lost=0):
        self.T, self.E, self.k, self.d, self.f, self.capacity, self.dt = T, E, k, d, f, capacity, dtype_of(dtype)
        self.half = HALF_STEP[self.dt]
        _, _, counts = routing(gen, T, E, k, capacity, skew)
        if lost:  # a program that dropped rows and kept them ragged
            counts[int(torch.argmax(counts))] -= lost
        self.counts = counts
        self.n = E * capacity if capacity else T * k
        c = counts.long().clamp(max=capacity) if capacity else counts.long()
        first = torch.arange(E) * capacity if capacity else torch.cumsum(c, 0) - c
        self.of = [torch.arange(int(a), int(a) + int(b)) for a, b in zip(first, c)]
        self.used = torch.zeros(self.n, dtype=torch.bool)
        for i in self.of:
            self.used[i] = True

    def problem(self):
        from paper_2605_00686_amd import binding as B
        return B.problem(self.T, self.d, self.E, self.k, self.f, 1, self.dt, capacity=self.capacity)

    def draw(self, gen, cols, std=1.0):
        """[n, cols], NaN in unused rows."""
        x = (torch.randn(self.n, cols, generator=gen) * std).to(self.dt)
        x[~self.used] = float("nan")
        return x

    def weights(self, gen, rows, cols, std=0.05):
        return (torch.randn(self.E, rows, cols, generator=gen) * std).to(self.dt)

    def zeros(self, cols):
        return torch.zeros(self.n, cols, dtype=torch.float64)


def product(a, b):
    """a b in 64 bits, and what K fp32 sums may be off: each step by a unit in the last place of the sum of the magnitudes (the matrix cores
    may cut where the vector ALU rounds)."""
    a, b = a.double(), b.double()
    return a @ b, (a.shape[1] + 1) * 2.0 ** -23 * (a.abs() @ b.abs())


def sigmoid_off(dt):
    """Of the sigmoid, relative to itself: in bf16 the exponent's rounding, in fp32 three units of the last place."""
    return 2.0 ** -17 if dt == torch.bfloat16 else 3 * 2.0 ** -23


def up(r, x, W1, W3):
    """{name: (value, bound)} of g, u, h."""
    out = {n: (r.zeros(r.f), r.zeros(r.f)) for n in ("g", "u", "h")}
    for e, i in enumerate(r.of):
        (g, eg), (u, eu) = product(x[i], W1[e]), product(x[i], W3[e])
        silu = g * torch.sigmoid(g)
        h = silu * u
        # (silu's slope is at most 1.0999; the products of the errors are covered by the doubled rounding steps)
        eh = 1.1 * eg * u.abs() + (silu.abs() + 1.1 * eg) * eu + h.abs() * (r.half + sigmoid_off(r.dt) + 4 * 2.0 ** -24)
        for n, v, o in (("g", g, eg + r.half * g.abs()), ("u", u, eu + r.half * u.abs()), ("h", h, eh)):
            out[n][0][i], out[n][1][i] = v, o * (1 + 2.0 ** -6)
    return out


def down(r, h, W2):
    y, off = r.zeros(r.d), r.zeros(r.d)
    for e, i in enumerate(r.of):
        v, o = product(h[i], W2[e])
        y[i], off[i] = v, (o + r.half * v.abs()) * (1 + 2.0 ** -6)
    return {"y": (y, off)}


def matrix_grad(r, a, b):
    out = torch.zeros(r.E, a.shape[1], b.shape[1], dtype=torch.float64)
    off = torch.zeros_like(out)
    for e, i in enumerate(r.of):
        v, o = product(a[i].t(), b[i])
        out[e], off[e] = v, (o + r.half * v.abs()) * (1 + 2.0 ** -6)
    return out, off


def down_backward(r, dy, W2, h, g, u):
    out = {n: (r.zeros(r.f), r.zeros(r.f)) for n in ("dh", "dg", "du")}
    for e, i in enumerate(r.of):
        dh, eh = product(dy[i], W2[e].t())
        G, U = g[i].double(), u[i].double()
        s = torch.sigmoid(G)
        slope = s * (1 + G * (1 - s))
        dg, du = dh * U * slope, dh * G * s
        # s moves by so much of itself, s (1 + g (1 - s)) by |1 + g - 2 g s| <= 1 + |g| times that, and four roundings
        es = (sigmoid_off(r.dt) + 4 * 2.0 ** -24) * s * (1 + G.abs())
        eg = eh * (U * slope).abs() + (dh.abs() + eh) * U.abs() * es + dg.abs() * (r.half + 4 * 2.0 ** -24)
        eu = eh * (G * s).abs() + du.abs() * (r.half + sigmoid_off(r.dt) + 4 * 2.0 ** -24)
        for n, v, o in (("dh", dh, eh + r.half * dh.abs()), ("dg", dg, eg), ("du", du, eu)):
            out[n][0][i], out[n][1][i] = v, o * (1 + 2.0 ** -6)
    if h is not None:
        out["dW2"] = matrix_grad(r, h, dy)
    return out


def up_backward(r, x, W1, W3, dg, du):
    dx, off = r.zeros(r.d), r.zeros(r.d)
    for e, i in enumerate(r.of):
        v, o = product(torch.cat([dg[i], du[i]], 1), torch.cat([W1[e], W3[e]], 1).t())
        dx[i], off[i] = v, (o + r.half * v.abs()) * (1 + 2.0 ** -6)
    return {"dx": (dx, off), "dW1": matrix_grad(r, x, dg), "dW3": matrix_grad(r, x, du)}


def check(name, got, want):
    value, off = want
    got = got.cpu().double()
    assert torch.isfinite(got).all(), f"{name}: not finite"
    # (numbers below the type's normal ones are rounded to its smallest step)
    far = (got - value).abs() > off + 2.0 ** -133
    assert not far.any(), f"{name}: {int(far.sum())} of {far.numel()} off, by {float(((got - value).abs() / (off + 1e-300)).max()):.3g} of the bound"

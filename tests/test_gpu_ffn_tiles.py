"""The experts' products over every tile, cut and order of tiles that they choose from, against the definitions in 64 bits; a training step of all
of them together."""
import pytest
import torch

from tests import ffn_forms as F
from tests.test_gpu_ffn import NAN, all_calls, ids, poisoned, workspace

pytestmark = pytest.mark.gpu

# (T, E, k, d, f, capacity, dtype).  Few rows and many steps cut the reduction of rows' products, many rows and few columns that of the weights'
# gradients; more tiles than there are workgroups, twice, are planned: over few experts and over dozens, ragged and padded.
SHAPES = [
    (6, 64, 1, 2080, 16, 1, "f32"), (30, 64, 1, 16, 2112, 1, "f32"), (40, 64, 2, 2000, 16, 0, "f32"), (79, 64, 1, 16, 2224, 0, "f32"),
    (3015, 8, 3, 64, 64, 0, "bf16"), (6, 64, 3, 64, 1984, 0, "bf16"), (11, 40, 2, 1600, 64, 1, "bf16"), (4127, 2, 2, 576, 16, 0, "f32"),
    (4999, 1, 1, 16, 1072, 9349, "f32"), (2, 5, 3, 2144, 1744, 0, "f32"), (1, 40, 3, 80, 784, 0, "f32"), (2, 40, 2, 960, 192, 1, "bf16"),
    (3161, 64, 2, 1568, 16, 0, "f32"), (1, 33, 3, 2112, 192, 1, "bf16"), (1, 8, 1, 2112, 1024, 0, "bf16"), (2, 8, 2, 2368, 896, 1, "bf16"),
    (2, 5, 1, 2208, 1568, 1, "f32"), (2403, 33, 3, 16, 2288, 0, "f32"), (1, 64, 1, 192, 1984, 0, "bf16"), (514, 40, 3, 16, 736, 29, "f32"),
    (1636, 64, 2, 64, 1856, 0, "bf16"), (6146, 5, 3, 1744, 16, 5632, "f32"), (1, 8, 1, 832, 1216, 0, "bf16"), (669, 64, 3, 1664, 64, 0, "bf16"),
    (951, 64, 2, 2112, 64, 28, "bf16"), (549, 64, 3, 64, 2496, 39, "bf16"), (5110, 64, 1, 960, 64, 0, "bf16"), (6, 8, 1, 2304, 960, 1, "bf16"),
    (1475, 33, 2, 16, 2368, 163, "f32"), (4705, 5, 1, 1632, 16, 0, "f32"), (7, 64, 1, 192, 1984, 1, "bf16"), (5565, 64, 3, 2160, 16, 0, "f32"),
    (5481, 5, 2, 64, 1984, 0, "bf16"), (6110, 5, 1, 1936, 16, 0, "f32"), (4187, 40, 1, 64, 704, 0, "bf16"), (100, 40, 1, 880, 768, 0, "f32"),
    (4470, 3, 2, 2496, 64, 5624, "bf16"), (1498, 8, 1, 1184, 864, 0, "f32"), (5678, 8, 3, 16, 1888, 0, "f32"), (4263, 8, 3, 80, 1152, 2932, "f32"),
]


@pytest.mark.parametrize("shape", SHAPES, ids=ids)
def test_all_calls(shape):
    """Every output of every call against its definition on that call's own inputs."""
    gen = torch.Generator().manual_seed(20)
    r = F.Rows(gen, *shape)
    run, out, _ = all_calls(r, gen)
    gen = torch.Generator().manual_seed(20)
    F.Rows(gen, *shape)
    x, dy, _ = r.draw(gen, r.d), r.draw(gen, r.d), r.draw(gen, 2 * r.f)
    W1, W3, W2 = r.weights(gen, r.d, r.f), r.weights(gen, r.d, r.f), r.weights(gen, r.f, r.d)
    run()
    got = {n: t.cpu() for n, t in out.items()}
    g, u, dg, du = got["gu"][:, :r.f], got["gu"][:, r.f:], got["dg"][:, :r.f], got["dg"][:, r.f:]
    for want, names in ((F.up(r, x, W1, W3), dict(g=g, u=u, h=got["h"])), (F.down(r, got["h"], W2), dict(y=got["y"])),
                        (F.down_backward(r, dy, W2, got["h"], g, u), dict(dg=dg, du=du, dW2=got["dW2"])),
                        (F.up_backward(r, x, W1, W3, dg, du), dict(dx=got["dx"], dW1=got["dW1"], dW3=got["dW3"]))):
        for name, value in names.items():
            F.check(name, value, want[name])


# reductions cut and joined; planned tiles over few experts and over dozens
MIXED = [(5, 4, 1, 2048, 1088, 0, "bf16"), (90, 2, 1, 1040, 528, 0, "f32"), (1636, 64, 2, 64, 1856, 0, "bf16"), (2403, 33, 3, 16, 2288, 0, "f32"),
         (2, 8, 2, 2368, 896, 1, "bf16")]


@pytest.mark.parametrize("shape", MIXED, ids=ids)
def test_captured_and_replayed(shape):
    gen = torch.Generator().manual_seed(21)
    r = F.Rows(gen, *shape)
    run, out, _ = all_calls(r, gen)
    run()
    want = {n: t.clone() for n, t in out.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        for t in out.values():
            t.fill_(NAN)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[n], want[n]) for n in out)
        run()  # (eagerly in between, with the workspace that the graph has)
        assert all(torch.equal(out[n], want[n]) for n in out)


@pytest.mark.parametrize("shape", MIXED, ids=ids)
def test_no_rows(shape):
    """No expert has any: every output is zeros, the rows' and the gradients'."""
    gen = torch.Generator().manual_seed(27)
    r = F.Rows(gen, *shape)
    run, out, n = all_calls(r, gen)
    n.zero_()
    run()
    assert all((t == 0).all() for t in out.values())


@pytest.mark.parametrize("shape", [(1100, 5, 1, 192, 320, 0, "bf16"), (3, 8, 2, 1984, 192, 0, "bf16"), (200, 3, 1, 80, 208, 90, "f32"), (1636, 64, 2, 64, 448, 0, "bf16")],
                         ids=ids)
def test_strides_and_nothing_around_is_touched(shape):
    """Rows and matrices further apart than they are long, 16 bytes behind a line's start: the results of dense ones, and what lies between is kept."""
    from paper_2605_00686_amd import binding as B
    gen = torch.Generator().manual_seed(28)
    r = F.Rows(gen, *shape)
    x, dy, W1, W3, W2 = r.draw(gen, r.d).cuda(), r.draw(gen, r.d).cuda(), r.weights(gen, r.d, r.f).cuda(), r.weights(gen, r.d, r.f).cuda(), r.weights(gen, r.f, r.d).cuda()
    p, n, ws = r.problem(), r.counts.cuda(), workspace(r.problem())
    piece = 16 // x.element_size()

    def wide(rows, cols):  # rows, and a row before and behind, with 3 pieces between
        whole = torch.full((rows + 2, cols + 3 * piece), 77.0, dtype=r.dt, device="cuda")
        return whole, whole[1:-1, piece:piece + cols]

    def matrices(t):
        whole, view = wide(r.E * t.shape[1], t.shape[2])
        view = view.unflatten(0, t.shape[:2])
        view.copy_(t)
        return whole, view

    def calls(g, u, dg, du, h, y, dW2, dx, dW1, dW3, w1, w3):
        B.moe_ffn_up(p, x, w1, w3, n, g, u, h, ws)
        B.moe_ffn_down(p, h, W2, n, y, ws)
        B.moe_ffn_down_backward(p, dy, W2, h, g, u, n, None, dg, du, dW2, ws)
        B.moe_ffn_up_backward(p, x, w1, w3, dg, du, n, dx, dW1, dW3, ws)
    dense = dict(g=(r.n, r.f), u=(r.n, r.f), dg=(r.n, r.f), du=(r.n, r.f), h=(r.n, r.f), y=(r.n, r.d), dW2=W2.shape, dx=(r.n, r.d), dW1=W1.shape, dW3=W1.shape)
    want = {name: poisoned(*s, dt=r.dt) for name, s in dense.items()}
    calls(**want, w1=W1, w3=W3)
    wholes, got = {}, {}
    for name, s in dense.items():
        if name in ("dW1", "dW3"):
            wholes[name], got[name] = matrices(poisoned(*s, dt=r.dt))
        elif name in ("g", "u", "dg", "du"):
            wholes[name], got[name] = wide(*s)
        else:  # dense ones, 16 bytes behind a line's start and with numbers on both sides
            size = torch.Size(s).numel()
            wholes[name] = torch.full((size + 2 * piece,), 77.0, dtype=r.dt, device="cuda")
            got[name] = wholes[name][piece:-piece].view(s)
    calls(**got, w1=matrices(W1)[1], w3=matrices(W3)[1])
    for name in dense:
        assert torch.equal(got[name], want[name]), name
        got[name].fill_(77.0)
        assert (wholes[name] == 77.0).all(), name


def test_calls_at_the_same_time():
    """Two streams, each with a workspace of its own."""
    gen = torch.Generator().manual_seed(22)
    sets = [all_calls(F.Rows(gen, *shape), gen) for shape in MIXED[:4]]
    wants = []
    for run, out, _ in sets:
        run()
        wants.append({n: t.clone() for n, t in out.items()})
    streams = [torch.cuda.Stream() for _ in sets]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for s, (run, _, _) in zip(streams, sets):
            with torch.cuda.stream(s):
                run()
    torch.cuda.synchronize()
    for (_, out, _), want in zip(sets, wants):
        assert all(torch.equal(out[n], want[n]) for n in out)


def test_long_sums_in_fp32():
    """16384 steps.  A rounding of a partial sum is at most 2^-24 of it, evenly spread and independent; partial sums of random terms grow as the root
    of their number, so N of them leave sqrt(N / 6) 2^-24 of the sum.  Sums of 512 steps have N = 192 (six products per 16 steps), 32 of those are
    added up: 4.8e-7.  Twice that; one sum of all steps has 1.9e-6."""
    from paper_2605_00686_amd import binding as B
    gen = torch.Generator().manual_seed(23)
    r = F.Rows(gen, 512, 4, 1, 256, 8192, 0, "f32")
    x, W1, W3, dgu = r.draw(gen, 256), r.weights(gen, 256, 8192), r.weights(gen, 256, 8192), r.draw(gen, 2 * 8192)
    dx = poisoned(r.n, 256, dt=r.dt)
    B.moe_ffn_up_backward(r.problem(), x.cuda(), W1.cuda(), W3.cuda(), dgu[:, :8192].contiguous().cuda(), dgu[:, 8192:].contiguous().cuda(),
                          r.counts.cuda(), dx, None, None, workspace(r.problem()))
    want = torch.cat([torch.cat([dgu[i, :8192].double() @ W1[e].double().t() + dgu[i, 8192:].double() @ W3[e].double().t()]) for e, i in enumerate(r.of)])
    rest = 2 * 2.0 ** -24 * ((192 / 6) ** 0.5 + (32 / 6) ** 0.5)
    assert float((dx.cpu().double() - want).norm() / want.norm()) < rest


@pytest.mark.parametrize("T", [70, 900])
def test_fp32_numbers_at_the_end_of_the_range(T):
    """Numbers that bf16 rounds to infinity, and products that only its numbers' leave the range with, give what fp32 gives."""
    from paper_2605_00686_amd import binding as B
    gen = torch.Generator().manual_seed(24)
    r = F.Rows(gen, T, 2, 1, 64, 80, 0, "f32")
    h, W2 = r.draw(gen, 80), r.weights(gen, 80, 64)
    a, b = int(r.of[0][5]), int(r.of[1][-1])
    h[a] = 0
    h[a, 3] = 3.4e38  # (times weights of 0.2 at most)
    near = 2.0 ** 64 * (1 - 2.0 ** -10)
    h[b] = 0
    h[b, 7], W2[1, 7, 11] = near, near
    h[r.of[1][:-1], 7] = 0
    y = poisoned(r.n, 64, dt=r.dt)
    B.moe_ffn_down(r.problem(), h.cuda(), W2.cuda(), r.counts.cuda(), y, workspace(r.problem()))
    F.check("y", y, F.down(r, h, W2)["y"])
    assert float(y[b, 11]) == near * near


def f32_step(gen, T=60, E=5, k=2, d=112, f=144):
    r = F.Rows(gen, T, E, k, d, f, 0, "f32")
    return r, r.draw(gen, d), r.draw(gen, d), r.weights(gen, d, f, 0.1), r.weights(gen, d, f, 0.1), r.weights(gen, f, d, 0.1)


def test_gradients_against_differences():
    """<y, dy> in 64 bits as a function of every input, by central differences: each of a chain of three products is off by (K + 1) 2^-23 of the sum
    of the magnitudes, which random terms hold to sqrt(K) times the sum: 3 * 145 * 12 * 2^-23 = 6e-4 of the gradient."""
    from paper_2605_00686_amd import binding as B
    gen = torch.Generator().manual_seed(25)
    r, x, dy, W1, W3, W2 = f32_step(gen)
    p, n, ws = r.problem(), r.counts.cuda(), workspace(r.problem())
    c = [t.cuda() for t in (x, W1, W3, W2, dy)]
    g, u, h, dg, du = (poisoned(r.n, r.f, dt=r.dt) for _ in range(5))
    grads = [torch.empty_like(t) for t in c[:4]]
    B.moe_ffn_up(p, c[0], c[1], c[2], n, g, u, h, ws)
    B.moe_ffn_down_backward(p, c[4], c[3], h, g, u, n, None, dg, du, grads[3], ws)
    B.moe_ffn_up_backward(p, c[0], c[1], c[2], dg, du, n, grads[0], grads[1], grads[2], ws)

    def loss(x, W1, W3, W2):
        total = 0.0
        for e, i in enumerate(r.of):
            gg = x[i] @ W1[e]
            total += float(((gg * torch.sigmoid(gg) * (x[i] @ W3[e])) @ W2[e] * dy[i].double()).sum())
        return total
    at = [t.double() for t in (x, W1, W3, W2)]
    for j, grad in enumerate(grads):
        grad = grad.cpu().double()
        for way in (grad / grad.norm(), torch.randn(grad.shape, generator=gen, dtype=torch.float64) / grad.numel() ** 0.5):
            step = 2.0 ** -14
            ends = [loss(*[t + s * step * way if i == j else t for i, t in enumerate(at)]) for s in (1, -1)]
            assert abs((ends[0] - ends[1]) / (2 * step) - float((grad * way).sum())) < 6e-4 * float(grad.norm())


@pytest.mark.parametrize("dtype,capacity", [("f32", 0), ("f32", 80), ("bf16", 0), ("bf16", 80)])
def test_a_training_step(dtype, capacity):
    """Tokens to their experts, the products, back to the tokens, the way back, the norm of all gradients and all of them clipped: eagerly and as a graph,
    against automatic differentiation in 64 bits.  fp32: as for the differences, 4 products in a chain of up to 193 steps, 4 * 193 * 14 * 2^-23 =
    1.3e-3.  bf16: a rounding is 2^-8 at most, evenly spread: 2^-8 / sqrt(3) of a tensor's norm; up to 8 are behind an output (g and u, h, y, dy, dg and
    du, dx's rows, its own), their squares add up to 6.4e-3; twice that, for what the activation's slope makes of them."""
    from paper_2605_00686_amd import binding as B
    gen = torch.Generator().manual_seed(26)
    T, E, k, d, f = 96, 6, 2, 128, 192
    dt = F.dtype_of(dtype)
    x, dout = torch.randn(T, d, generator=gen).to(dt), torch.randn(T, d, generator=gen).to(dt)
    W1, W3, W2 = ((torch.randn(E, *s, generator=gen) * 0.08).to(dt) for s in ((d, f), (d, f), (f, d)))
    idx = torch.stack([torch.randperm(E, generator=gen)[:k] for _ in range(T)]).int()
    idx[:40, 0], idx[:40, 1] = 2, 4
    w = torch.rand(T, k, generator=gen) + 0.1
    p = B.problem(T, d, E, k, f, 1, dt, capacity=capacity)
    c = {n: t.cuda() for n, t in dict(x=x, dout=dout, W1=W1, W3=W3, W2=W2, idx=idx, w=w).items()}
    rows = E * capacity if capacity else T * k
    b, ws, status = B.Buffers(p), workspace(p), torch.zeros(1, dtype=torch.int32, device="cuda")
    xp, y, dy, dxp = (poisoned(rows, d, dt=dt) for _ in range(4))
    g, u, h, dg, du = (poisoned(rows, f, dt=dt) for _ in range(5))
    out, dx, dw = poisoned(T, d, dt=dt), poisoned(T, d, dt=dt), poisoned(T, k, dt=torch.float32)
    dWs = [poisoned(*c[n].shape, dt=dt) for n in ("W1", "W3", "W2")]
    clipped = [torch.empty_like(t) for t in dWs]
    total, norm = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1, device="cuda")
    tensors = B.tensor_list(dWs, clipped)
    grad_ws = torch.empty(B.moe_grad_workspace_bytes(tensors), dtype=torch.uint8, device="cuda")

    def step():
        B.moe_dispatch(p, c["x"], c["idx"], b.counts, b.offsets, b.perm, b.inv_perm, xp, status, b.workspace)
        B.moe_ffn_up(p, xp, c["W1"], c["W3"], b.counts, g, u, h, ws)
        B.moe_ffn_down(p, h, c["W2"], b.counts, y, ws)
        B.moe_unsort(p, y, b.inv_perm, c["w"], None, out, status)
        B.moe_unsort_backward(p, c["dout"], y, b.inv_perm, c["w"], b.counts, dy, dw, status)
        B.moe_ffn_down_backward(p, dy, c["W2"], h, g, u, b.counts, None, dg, du, dWs[2], ws)
        B.moe_ffn_up_backward(p, xp, c["W1"], c["W3"], dg, du, b.counts, dxp, dWs[0], dWs[1], ws)
        B.moe_unsort(p, dxp, b.inv_perm, None, None, dx, status)
        B.moe_grad_norm(tensors, total, norm, grad_ws)
        B.moe_grad_clip(tensors, total, 0.5)
    step()
    outputs = dict(out=out, dx=dx, dw=dw, dW1=dWs[0], dW3=dWs[1], dW2=dWs[2], norm=norm, total=total, c1=clipped[0], c3=clipped[1], c2=clipped[2])
    got = {n: t.clone() for n, t in outputs.items()}
    assert int(status.item()) == 0

    leaves = [t.double().requires_grad_() for t in (x, w, W1, W3, W2)]
    X, Wt, V1, V3, V2 = leaves
    value = torch.zeros(T, d, dtype=torch.float64)
    for e in range(E):
        for j in range(k):
            t = torch.nonzero(idx[:, j] == e).flatten()
            a = X[t] @ V1[e]
            value = value.index_add(0, t, (a * torch.sigmoid(a) * (X[t] @ V3[e])) @ V2[e] * Wt[t, j, None])
    grads = torch.autograd.grad((value * dout.double()).sum(), leaves)
    rest = 1.3e-3 if dtype == "f32" else 1.28e-2
    for name, want in zip(("out", "dx", "dw", "dW1", "dW3", "dW2"), (value.detach(), *grads)):
        assert float((got[name].cpu().double() - want).norm()) <= rest * float(want.norm()), name
    want = float(torch.cat([v.flatten() for v in grads[2:]]).norm())
    assert want > 1 and abs(float(got["norm"]) - want) <= rest * want
    assert abs(float(torch.cat([got[n].cpu().double().flatten() for n in ("c1", "c3", "c2")]).norm()) - 0.5) <= rest * 0.5

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in outputs.values():
            t.fill_(NAN)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, got[n]) for n, t in outputs.items())

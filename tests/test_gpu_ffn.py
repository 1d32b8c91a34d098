"""The experts' products as calls of their own, against the definitions in 64 bits; bounds from the arithmetic."""
import pytest
import torch

from tests import ffn_forms as F

pytestmark = pytest.mark.gpu
NAN = float("nan")


def workspace(p):
    from paper_2605_00686_amd import binding as B
    return torch.full((B.moe_ffn_workspace_bytes(p),), 255, dtype=torch.uint8, device="cuda")


def poisoned(*shape, dt):
    return torch.full(shape, NAN, dtype=dt, device="cuda")


def ids(shape):
    return "T%d_E%d_k%d_d%d_f%d_C%d_%s" % shape


@pytest.mark.parametrize("shape", F.SHAPES, ids=ids)
@pytest.mark.parametrize("halves", [False, True])
def test_up(shape, halves):
    from paper_2605_00686_amd import binding as B
    gen = torch.Generator().manual_seed(1)
    r = F.Rows(gen, *shape)
    x, W1, W3 = r.draw(gen, r.d), r.weights(gen, r.d, r.f), r.weights(gen, r.d, r.f)
    p = r.problem()
    h = poisoned(r.n, r.f, dt=r.dt)
    if halves:  # two products side by side, forward and in the weights
        W13 = torch.cat([W1, W3], 2).cuda()
        w1, w3 = W13[:, :, :r.f], W13[:, :, r.f:]
        gu = poisoned(r.n, 2 * r.f, dt=r.dt)
        g, u = gu[:, :r.f], gu[:, r.f:]
    else:
        w1, w3, g, u = W1.cuda(), W3.cuda(), poisoned(r.n, r.f, dt=r.dt), poisoned(r.n, r.f, dt=r.dt)
    B.moe_ffn_up(p, x.cuda(), w1, w3, r.counts.cuda(), g, u, h, workspace(p))
    want = F.up(r, x, W1, W3)
    for name, got in (("g", g), ("u", u), ("h", h)):
        F.check(name, got, want[name])
    # each output without the others has the same bits
    alone = poisoned(r.n, r.f, dt=r.dt)
    B.moe_ffn_up(p, x.cuda(), w1, w3, r.counts.cuda(), None, None, alone, workspace(p))
    assert torch.equal(alone, h)
    B.moe_ffn_up(p, x.cuda(), w1, w3, r.counts.cuda(), alone, torch.empty_like(alone), None, workspace(p))
    assert torch.equal(alone, g)


@pytest.mark.parametrize("shape", F.SHAPES, ids=ids)
def test_down(shape):
    from paper_2605_00686_amd import binding as B
    gen = torch.Generator().manual_seed(2)
    r = F.Rows(gen, *shape)
    h, W2 = r.draw(gen, r.f), r.weights(gen, r.f, r.d)
    p = r.problem()
    y = poisoned(r.n, r.d, dt=r.dt)
    B.moe_ffn_down(p, h.cuda(), W2.cuda(), r.counts.cuda(), y, workspace(p))
    F.check("y", y, F.down(r, h, W2)["y"])


@pytest.mark.parametrize("shape", F.SHAPES, ids=ids)
@pytest.mark.parametrize("halves", [False, True])
def test_down_backward(shape, halves):
    from paper_2605_00686_amd import binding as B
    gen = torch.Generator().manual_seed(3)
    r = F.Rows(gen, *shape)
    dy, W2, h, gu = r.draw(gen, r.d), r.weights(gen, r.f, r.d), r.draw(gen, r.f), r.draw(gen, 2 * r.f, 2.0)
    p, n = r.problem(), r.counts.cuda()
    gud = gu.cuda()
    if halves:  # in place
        g, u = gud[:, :r.f], gud[:, r.f:]
        dg, du = g, u
    else:
        g, u = gud[:, :r.f].contiguous(), gud[:, r.f:].contiguous()
        dg, du = poisoned(r.n, r.f, dt=r.dt), poisoned(r.n, r.f, dt=r.dt)
    dh, dW2 = poisoned(r.n, r.f, dt=r.dt), poisoned(r.E, r.f, r.d, dt=r.dt)
    B.moe_ffn_down_backward(p, dy.cuda(), W2.cuda(), h.cuda(), g, u, n, dh, dg, du, dW2, workspace(p))
    want = F.down_backward(r, dy, W2, h, gu[:, :r.f], gu[:, r.f:])
    for name, got in (("dh", dh), ("dg", dg), ("du", du), ("dW2", dW2)):
        F.check(name, got, want[name])
    # one at a time: the same bits, and nothing else is needed
    one = poisoned(r.n, r.f, dt=r.dt)
    B.moe_ffn_down_backward(p, dy.cuda(), W2.cuda(), None, None, None, n, one, None, None, None, workspace(p))
    assert torch.equal(one, dh)
    one = poisoned(r.E, r.f, r.d, dt=r.dt)
    B.moe_ffn_down_backward(p, dy.cuda(), None, h.cuda(), None, None, n, None, None, None, one, workspace(p))
    assert torch.equal(one, dW2)


@pytest.mark.parametrize("shape", F.SHAPES, ids=ids)
@pytest.mark.parametrize("halves", [False, True])
def test_up_backward(shape, halves):
    from paper_2605_00686_amd import binding as B
    gen = torch.Generator().manual_seed(4)
    r = F.Rows(gen, *shape)
    x, W1, W3, dgu = r.draw(gen, r.d), r.weights(gen, r.d, r.f), r.weights(gen, r.d, r.f), r.draw(gen, 2 * r.f)
    p, n, xd = r.problem(), r.counts.cuda(), x.cuda()
    if halves:
        W13, dW13, dgud = torch.cat([W1, W3], 2).cuda(), poisoned(r.E, r.d, 2 * r.f, dt=r.dt), dgu.cuda()
        w1, w3, dW1, dW3, dg, du = W13[:, :, :r.f], W13[:, :, r.f:], dW13[:, :, :r.f], dW13[:, :, r.f:], dgud[:, :r.f], dgud[:, r.f:]
    else:
        w1, w3, dg, du = W1.cuda(), W3.cuda(), dgu[:, :r.f].contiguous().cuda(), dgu[:, r.f:].contiguous().cuda()
        dW1, dW3 = poisoned(r.E, r.d, r.f, dt=r.dt), poisoned(r.E, r.d, r.f, dt=r.dt)
    dx = poisoned(r.n, r.d, dt=r.dt)
    B.moe_ffn_up_backward(p, xd, w1, w3, dg, du, n, dx, dW1, dW3, workspace(p))
    want = F.up_backward(r, x, W1, W3, dgu[:, :r.f], dgu[:, r.f:])
    for name, got in (("dx", dx), ("dW1", dW1), ("dW3", dW3)):
        F.check(name, got, want[name])
    for name, whole in (("dx", dx), ("dW1", dW1), ("dW3", dW3)):
        one = torch.full_like(whole, NAN)
        out = {**dict(dx=None, dW1=None, dW3=None), name: one}
        if not one.is_contiguous():
            continue
        if name == "dx":
            B.moe_ffn_up_backward(p, None, w1, w3, dg, du, n, one, None, None, workspace(p))
        else:
            B.moe_ffn_up_backward(p, xd, None, None, dg if name == "dW1" else None, du if name == "dW3" else None, n, out["dx"], out["dW1"],
                                  out["dW3"], workspace(p))
        assert torch.equal(one, whole.contiguous()), name


def all_calls(r, gen):
    """Inputs on the GPU, a function that makes the four calls with them, and the outputs."""
    from paper_2605_00686_amd import binding as B
    x, dy, dgu = r.draw(gen, r.d).cuda(), r.draw(gen, r.d).cuda(), r.draw(gen, 2 * r.f).cuda()
    W1, W3, W2 = r.weights(gen, r.d, r.f).cuda(), r.weights(gen, r.d, r.f).cuda(), r.weights(gen, r.f, r.d).cuda()
    p, n, f = r.problem(), r.counts.cuda(), r.f
    ws = workspace(p)
    out = dict(gu=poisoned(r.n, 2 * f, dt=r.dt), h=poisoned(r.n, f, dt=r.dt), y=poisoned(r.n, r.d, dt=r.dt), dg=poisoned(r.n, 2 * f, dt=r.dt),
               dW2=poisoned(r.E, f, r.d, dt=r.dt), dx=poisoned(r.n, r.d, dt=r.dt), dW1=poisoned(r.E, r.d, f, dt=r.dt), dW3=poisoned(r.E, r.d, f, dt=r.dt))

    def run():
        gu, dg = out["gu"], out["dg"]
        B.moe_ffn_up(p, x, W1, W3, n, gu[:, :f], gu[:, f:], out["h"], ws)
        B.moe_ffn_down(p, out["h"], W2, n, out["y"], ws)
        B.moe_ffn_down_backward(p, dy, W2, out["h"], gu[:, :f], gu[:, f:], n, None, dg[:, :f], dg[:, f:], out["dW2"], ws)
        B.moe_ffn_up_backward(p, x, W1, W3, dg[:, :f], dg[:, f:], n, out["dx"], out["dW1"], out["dW3"], ws)
    return run, out, n


@pytest.mark.parametrize("shape", [(40, 8, 2, 192, 448, 0, "bf16"), (517, 4, 2, 192, 320, 0, "bf16"), (150, 6, 3, 80, 272, 72, "f32")], ids=ids)
def test_captured_and_on_another_stream(shape):
    gen = torch.Generator().manual_seed(5)
    r = F.Rows(gen, *shape)
    run, out, _ = all_calls(r, gen)
    run()
    want = {n: t.clone() for n, t in out.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for t in out.values():
            t.fill_(NAN)
        run()
    side.synchronize()
    assert all(torch.equal(out[n], want[n]) for n in out)
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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_rows_and_rows_of_nobody(dtype):
    """Counts that come to less than the rows, or to nothing: zeros behind the last expert's rows, gradients of zero for experts without."""
    gen = torch.Generator().manual_seed(6)
    r = F.Rows(gen, 300, 3, 2, 64, 128, 0, dtype, lost=70)
    assert int((~r.used).sum()) == 70
    run, out, n = all_calls(r, gen)
    run()
    for name in ("gu", "h", "y", "dg", "dx"):
        assert (out[name][~r.used.cuda()] == 0).all() and torch.isfinite(out[name]).all(), name
    n.zero_()
    for t in out.values():
        t.fill_(NAN)
    run()
    assert all((t == 0).all() for t in out.values())


def test_counts_that_cannot_be():
    """A count below zero is zero, one past the rows ends there."""
    from paper_2605_00686_amd import binding as B
    gen = torch.Generator().manual_seed(7)
    r = F.Rows(gen, 64, 4, 2, 64, 64, 0, "bf16")
    h, W2 = r.draw(gen, 64).cuda(), r.weights(gen, 64, 64).cuda()
    p, ws = r.problem(), workspace(r.problem())

    def call(counts):
        y = poisoned(r.n, 64, dt=r.dt)
        B.moe_ffn_down(p, h, W2, torch.tensor(counts, dtype=torch.int32).cuda(), y, ws)
        dW2 = poisoned(r.E, 64, 64, dt=r.dt)
        B.moe_ffn_down_backward(p, h, None, h, None, None, torch.tensor(counts, dtype=torch.int32).cuda(), None, None, None, dW2, ws)
        return y, dW2
    for bad, good in (([50, -7, 20, 1000], [50, 0, 20, 58]), ([2 ** 31 - 1] * 4, [128, 0, 0, 0])):
        for a, b in zip(call(bad), call(good)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_numbers_that_are_not_finite_stay_in_their_row_and_expert(dtype):
    from paper_2605_00686_amd import binding as B
    gen = torch.Generator().manual_seed(8)
    r = F.Rows(gen, 90, 3, 2, 64, 64, 0, dtype)
    h, W2, dy = r.draw(gen, 64), r.weights(gen, 64, 64), r.draw(gen, 64)
    row = int(r.of[1][3])
    h[row, 5] = float("inf")
    p, ws = r.problem(), workspace(r.problem())
    y, dW2 = poisoned(r.n, 64, dt=r.dt), poisoned(3, 64, 64, dt=r.dt)
    B.moe_ffn_down(p, h.cuda(), W2.cuda(), r.counts.cuda(), y, ws)
    B.moe_ffn_down_backward(p, dy.cuda(), None, h.cuda(), None, None, r.counts.cuda(), None, None, None, dW2, ws)
    others = torch.arange(r.n) != row
    assert torch.isinf(y[row]).all() and torch.isfinite(y.cpu()[others]).all()
    assert torch.isinf(dW2[1, 5]).all() and torch.isfinite(dW2[0]).all() and torch.isfinite(dW2[2]).all()
    assert torch.isfinite(dW2[1, :5]).all() and torch.isfinite(dW2[1, 6:]).all()


def test_offsets_past_32_bits():
    """More than 2^31 elements in the rows of g and u, and more than 2^31 in the weights: the last rows and the last expert."""
    from paper_2605_00686_amd import binding as B
    gen = torch.Generator(device="cuda").manual_seed(9)
    bf = torch.bfloat16

    def normal(*shape, std=1.0):
        return torch.empty(shape, dtype=bf, device="cuda").normal_(0.0, std, generator=gen)
    # rows
    T, f = 264192, 4160
    p = B.problem(T, 64, 2, 1, f, 1, bf)
    n = torch.tensor([T - 300, 300], dtype=torch.int32).cuda()
    x, W1, W3 = normal(T, 64), normal(2, 64, f, std=0.1), normal(2, 64, f, std=0.1)
    gu = torch.full((T, 2 * f), NAN, dtype=bf, device="cuda")
    assert gu.numel() > 2 ** 31
    ws = workspace(p)
    B.moe_ffn_up(p, x, W1, W3, n, gu[:, :f], gu[:, f:], None, ws)
    g, u = x[-300:].double() @ W1[1].double(), x[-300:].double() @ W3[1].double()
    assert float((gu[-300:, :f].double() - g).norm() / g.norm()) < 2.0 ** -8 and float((gu[-300:, f:].double() - u).norm() / u.norm()) < 2.0 ** -8
    dx, dW1 = torch.full((T, 64), NAN, dtype=bf, device="cuda"), torch.full((2, 64, f), NAN, dtype=bf, device="cuda")
    B.moe_ffn_up_backward(p, x, W1, W3, gu[:, :f], gu[:, f:], n, dx, dW1, None, ws)
    want = gu[-300:, :f].double() @ W1[1].double().t() + gu[-300:, f:].double() @ W3[1].double().t()
    assert float((dx[-300:].double() - want).norm() / want.norm()) < 2.0 ** -8
    want = x[-300:].double().t() @ gu[-300:, :f].double()
    assert float((dW1[1].double() - want).norm() / want.norm()) < 2.0 ** -8
    del gu, x, dx
    # weights
    E, d, f = 41, 7168, 7424
    p = B.problem(50, d, E, 1, f, 1, bf)
    n = torch.zeros(E, dtype=torch.int32).cuda()
    n[0], n[E - 1] = 20, 30
    W2, h, dy = normal(E, f, d, std=0.02), normal(50, f), normal(50, d)
    assert W2.numel() > 2 ** 31
    ws = workspace(p)
    y, dh, dW2 = torch.full((50, d), NAN, dtype=bf, device="cuda"), torch.full((50, f), NAN, dtype=bf, device="cuda"), torch.full_like(W2, NAN)
    B.moe_ffn_down(p, h, W2, n, y, ws)
    B.moe_ffn_down_backward(p, dy, W2, h, None, None, n, dh, None, None, dW2, ws)
    last = W2[E - 1].double()
    for got, want in ((y[20:], h[20:].double() @ last), (dh[20:], dy[20:].double() @ last.t()), (dW2[E - 1], h[20:].double().t() @ dy[20:].double())):
        assert float((got.double() - want).norm() / want.norm()) < 2.0 ** -8
    assert not dW2[1:E - 1].any()

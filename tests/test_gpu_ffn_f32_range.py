"""fp32 numbers of every size in the experts' products, subnormal ones too, and those that are worst to cut, against 64 bits."""
import pytest
import torch

from tests import ffn_forms as F
from tests.test_gpu_ffn import poisoned, workspace

pytestmark = pytest.mark.gpu

# (T, E, k, d, f, capacity): row blocks of 64 and 128 rows; reductions that are cut; padded rows
SHAPES = [(300, 3, 1, 144, 208, 0), (2000, 2, 1, 64, 336, 0), (5, 3, 2, 2208, 1568, 0), (150, 6, 3, 80, 272, 72)]


def near(got, want, smallest):
    value, off = want
    assert torch.isfinite(got).all()
    got = got.cpu().double()
    # (a result below the normal numbers is rounded twice, to half a step of the smallest each time, and so is each of the parts that it is made of)
    far = (got - value).abs() > off + smallest * 2.0 ** -149
    assert not far.any(), f"{int(far.sum())} of {far.numel()} off, by {float(((got - value).abs() / (off + 2.0 ** -149)).max()):.3g} of the bound"


# standard deviations of the two operands: subnormal numbers that come out as ordinary ones; small ones; sums that are subnormal; either end at once
@pytest.mark.parametrize("a,b", [(-146, 98), (98, -146), (-135, 60), (-120, 100), (-112, 0), (-70, -70), (-60, -66), (-146, 120), (120, -146), (50, 40)])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "T%d_E%d_k%d_d%d_f%d_C%d" % s)
def test_products_of_numbers_of_any_size(shape, a, b):
    from paper_2605_00686_amd import binding as B
    gen = torch.Generator().manual_seed(51)
    r = F.Rows(gen, *shape, "f32")
    p, n, ws = r.problem(), r.counts.cuda(), workspace(r.problem())

    def rows(cols, power):  # (scaled in 64 bits, rounded once)
        return (r.draw(gen, cols).double() * 2.0 ** power).float()

    def matrices(*shape, power):
        return (torch.randn(r.E, *shape, generator=gen).double() * 2.0 ** power).float()
    h, W2, dy = rows(r.f, a), matrices(r.f, r.d, power=b), rows(r.d, b)
    x, W1, W3, dg, du = rows(r.d, b), matrices(r.d, r.f, power=b), matrices(r.d, r.f, power=b), rows(r.f, a), rows(r.f, a)
    y, dW2, dx, dW1, dW3 = poisoned(r.n, r.d, dt=r.dt), poisoned(*W2.shape, dt=r.dt), poisoned(r.n, r.d, dt=r.dt), poisoned(*W1.shape, dt=r.dt), poisoned(*W1.shape, dt=r.dt)
    c = {name: t.cuda() for name, t in dict(h=h, W2=W2, dy=dy, x=x, W1=W1, W3=W3, dg=dg, du=du).items()}
    B.moe_ffn_down(p, c["h"], c["W2"], n, y, ws)
    B.moe_ffn_down_backward(p, c["dy"], None, c["h"], None, None, n, None, None, None, dW2, ws)
    B.moe_ffn_up_backward(p, c["x"], c["W1"], c["W3"], c["dg"], c["du"], n, dx, dW1, dW3, ws)
    parts = 32  # (of a reduction that is cut, at most)
    near(y, F.down(r, h, W2)["y"], parts)
    near(dW2, F.matrix_grad(r, h, dy), parts)
    for name, value in F.up_backward(r, x, W1, W3, dg, du).items():
        near(dict(dx=dx, dW1=dW1, dW3=dW3)[name], value, parts)
    # dh and g, u with the operands' sizes the other way round too
    dh, g, u = (poisoned(r.n, r.f, dt=r.dt) for _ in range(3))
    dy, W2, x, W1, W3 = rows(r.d, a), matrices(r.f, r.d, power=b), rows(r.d, a), matrices(r.d, r.f, power=b), matrices(r.d, r.f, power=b)
    B.moe_ffn_down_backward(p, dy.cuda(), W2.cuda(), None, None, None, n, dh, None, None, None, ws)
    B.moe_ffn_up(p, x.cuda(), W1.cuda(), W3.cuda(), n, g, u, None, ws)
    zero = torch.zeros(r.n, r.f)
    near(dh, F.down_backward(r, dy, W2, None, zero, zero)["dh"], parts)
    want = F.up(r, x, W1, W3)
    near(g, want["g"], parts)
    near(u, want["u"], parts)


def test_numbers_that_a_cut_loses_most_of():
    """The bits behind the first eight nearly half a step, and those behind the next eight again: the products that are left out come to nearly 2^-24 of each, all with one sign.  A sum of 16 such products is added up in
    six steps, each off by a unit in the last place at most."""
    from paper_2605_00686_amd import binding as B
    worst = float.fromhex("0x1.00ff8p0")
    for T in (3, 300):
        p = B.problem(T, 16, 1, 1, 16, 1, torch.float32)
        h, W2, y = torch.full((T, 16), worst, device="cuda"), torch.full((1, 16, 16), worst, device="cuda"), torch.empty(T, 16, device="cuda")
        B.moe_ffn_down(p, h, W2, torch.tensor([T], dtype=torch.int32).cuda(), y, workspace(p))
        want = 16 * worst * worst
        assert float((y.double() - want).abs().max()) <= (2.0 ** -24 + 6 * 2.0 ** -23) * want

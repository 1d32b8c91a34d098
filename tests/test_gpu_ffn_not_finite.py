"""Numbers that are not finite, or that a scaled fp32 number leaves the range with, in reductions that are cut, in planned tiles and in padded rows: they
have their effect on their row (and their expert's gradients) and no other, eagerly and in a graph."""
import pytest
import torch

from tests import ffn_forms as F
from tests.test_gpu_ffn import NAN, ids, poisoned, workspace
from tests.test_gpu_ffn_tiles import MIXED

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [float("inf"), NAN, 2.0 ** 120])
@pytest.mark.parametrize("shape", MIXED, ids=ids)
def test_one_number(shape, bad):
    from paper_2605_00686_amd import binding as B
    gen = torch.Generator().manual_seed(61)
    r = F.Rows(gen, *shape)
    h, W2, dy = r.draw(gen, r.f), r.weights(gen, r.f, r.d), r.draw(gen, r.d)
    e = max(range(r.E), key=lambda e: len(r.of[e]))
    row, step = int(r.of[e][-1]), 5
    clean = h.clone()
    clean[row] = 0  # (what the others are compared with: the bad row's own results are looked at apart)
    h[row, step] = bad
    p, n, ws = r.problem(), r.counts.cuda(), workspace(r.problem())
    y, dW2, dh = poisoned(r.n, r.d, dt=r.dt), poisoned(*W2.shape, dt=r.dt), poisoned(r.n, r.f, dt=r.dt)
    hd, Wd, dyd = h.cuda(), W2.cuda(), dy.cuda()
    broken = dy.clone()
    broken[row, 3] = bad
    bd = broken.cuda()

    def calls():
        B.moe_ffn_down(p, hd, Wd, n, y, ws)
        B.moe_ffn_down_backward(p, dyd, None, hd, None, None, n, None, None, None, dW2, ws)
        B.moe_ffn_down_backward(p, bd, Wd, None, None, None, n, dh, None, None, None, ws)
    calls()
    others = torch.arange(r.n) != row
    want = F.down(r, clean, W2)["y"]
    F.check("y", y.cpu()[others], (want[0][others], want[1][others]))
    clean_dy = dy.clone()
    clean_dy[row] = 0
    zero = torch.zeros(r.n, r.f)
    want = F.down_backward(r, clean_dy, W2, None, zero, zero)["dh"]
    F.check("dh", dh.cpu()[others], (want[0][others], want[1][others]))
    clean[row] = h[row]
    clean[row, step] = 0
    value, off = F.matrix_grad(r, clean, dy)
    rest = torch.ones(r.f, dtype=torch.bool)
    rest[step] = False
    for x in range(r.E):
        keep = rest if x == e else torch.ones_like(rest)
        F.check("dW2", dW2[x].cpu()[keep], (value[x][keep], off[x][keep]))
    if bad == 2.0 ** 120:  # finite: its products are those of any other number
        clean[row, step] = bad
        want = F.down(r, clean, W2)["y"]
        F.check("y", y[row], (want[0][row], want[1][row]))
        value, off = F.matrix_grad(r, clean, dy)
        F.check("dW2", dW2[e, step], (value[e, step], off[e, step]))
    else:
        for got in (y[row], dh[row], dW2[e, step]):
            assert not torch.isfinite(got).any()
    before = [t.clone() for t in (y, dW2, dh)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(2):
        for t in (y, dW2, dh):
            t.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a.nan_to_num(1.5), b.nan_to_num(1.5)) for a, b in zip((y, dW2, dh), before))

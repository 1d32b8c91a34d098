"""GPU tests of moe_route_backward with infinite weight gradients: every infinity and NaN is the one of the definition."""
import pytest
import torch

from tests.test_gpu_gate_grad import call, expected, make

pytestmark = pytest.mark.gpu


def definition(idx, w, dw, x, Wg):
    """The gradients in 64 bits, slot by slot: an expert that a token did not choose sees nothing of it."""
    T, k = idx.shape
    w, dw, x, Wg = w.double(), dw.double(), x.double(), Wg.double()
    dl = w * (dw - (w * dw).sum(1, keepdim=True))
    dx, dWg, db = torch.zeros_like(x), torch.zeros(Wg.shape[1], Wg.shape[0], dtype=torch.float64), torch.zeros(Wg.shape[1], dtype=torch.float64)
    for j in range(k):
        e = idx[:, j].long()
        dx += dl[:, j, None] * Wg.t()[e]
        dWg.index_add_(0, e, dl[:, j, None] * x)
        db.index_add_(0, e, dl[:, j])
    return dx, dWg.t(), db


# both shapes of a task, two groups of experts, more than 8 and 16 choices, several parts of the tokens
@pytest.mark.parametrize("case", [(300, 192, 12, 3, "bf16"), (200, 80, 140, 4, "f32"), (70, 320, 70, 2, "bf16"), (500, 128, 200, 2, "bf16"),
                                  (64, 64, 48, 11, "f32"), (900, 80, 20, 17, "f32"), (2500, 144, 131, 3, "f32"), (2500, 192, 40, 9, "bf16"),
                                  (2, 64, 2, 2, "f32")],
                         ids=lambda c: "T%d_d%d_E%d_k%d_%s" % c)
def test_infinite_weight_gradients(case):
    print(f"case infinite {case}", flush=True)
    B, p, gen, dt, idx, w, dw, x, Wg = make(*case)
    T, d, E, k, _ = case
    hit = sorted({0, T // 2, T - 1})
    for i, t in enumerate(hit):
        dw[t, i % k] = float("-inf") if i % 2 else float("inf")
    x[hit[0], 3] = 0.0  # an infinity times nothing
    x[hit[-1], 5], x[hit[0], 7] = float("inf"), float("nan")
    x[(T // 2 + 1) % T, 9] = 1.0 / 3.0
    got = [g.cpu() for g in call(B, p, x, Wg, idx, w, dw)]
    want = definition(idx, w, dw, x, Wg)
    assert bool(torch.isinf(want[1]).any())
    for g, ref in zip(got, want):
        for what in (torch.isnan, torch.isposinf, torch.isneginf):
            assert torch.equal(what(g), what(ref)), what.__name__
    # the rest, as if those tokens were not there
    rest = torch.ones(T, dtype=torch.bool)
    rest[hit] = False
    if not bool(rest.any()):
        return
    for g, ref, (clean, bound) in zip(got, want, expected(idx[rest], w[rest], dw[rest], x[rest], Wg, dt)):
        g = g[rest] if g.shape == (T, d) and g.shape == ref.shape and clean.shape != g.shape else g
        at = torch.isfinite(g)
        assert bool(((g.double() - clean).abs() <= bound)[at].all())
    # each gradient alone: the same bits
    for i, one in enumerate("xwb"):
        alone = call(B, p, x, Wg, idx, w, dw, one)[i].cpu()
        assert torch.equal(torch.nan_to_num(alone, nan=7.0), torch.nan_to_num(got[i], nan=7.0))


def test_a_finite_difference_past_the_range_is_infinite():
    # dw apart by more than fp32 holds: dl is infinite without an infinity among the inputs
    B, p, gen, dt, idx, w, dw, x, Wg = make(100, 64, 8, 2, "f32")
    w[50], dw[50] = torch.tensor([0.9, 0.1]), torch.tensor([3e38, -3e38])
    dx, dWg, db = (t.cpu() for t in call(B, p, x, Wg, idx, w, dw))
    # choice 1: 0.1 (-3e38 - 2.4e38), past the range before the product; choice 0: 0.9 (3e38 - 2.4e38)
    e = int(idx[50, 1])
    assert float(db[e]) == float("-inf")
    assert torch.equal(dWg[:, e], torch.where(x[50] > 0, float("-inf"), float("inf")))
    others = [i for i in range(8) if i != e]
    assert bool(torch.isfinite(dWg[:, others]).all()) and bool(torch.isfinite(db[others]).all())

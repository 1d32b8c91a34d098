"""GPU tests of moe_route_backward against the definitions in 64 bits, and together with moe_route against differences."""
import pytest
import torch

from tests.train_forms import HALF_STEP, dtype_of, routing, weights

pytestmark = pytest.mark.gpu

# T, d, E, k, dtype: one token, rows from 64 bytes, odd numbers of pieces, experts nobody chose, all experts chosen, tokens around multiples of 64 and 256
CASES = [(1, 64, 2, 2, "bf16"), (1, 2048, 128, 8, "bf16"), (2, 16, 3, 2, "f32"), (5, 7168, 256, 8, "bf16"), (31, 192, 33, 32, "bf16"),
         (63, 528, 17, 5, "f32"), (64, 512, 8, 2, "f32"), (65, 320, 64, 6, "bf16"), (128, 448, 250, 11, "bf16"), (255, 4112, 9, 3, "f32"),
         (257, 960, 256, 32, "bf16"), (511, 64, 31, 4, "bf16"), (513, 2112, 48, 8, "bf16"), (1000, 1088, 128, 7, "bf16"), (1300, 256, 200, 1, "f32"),
         (2500, 640, 16, 16, "bf16"), (4099, 128, 5, 2, "f32"), (6000, 192, 256, 8, "bf16")]
IDS = ["T%d_d%d_E%d_k%d_%s" % c for c in CASES]


def make(T, d, E, k, dtype):
    from paper_2605_00686_amd import binding as B
    dt = dtype_of(dtype)
    gen = torch.Generator().manual_seed(7 * T + d + E + k)
    p = B.problem(T, d, E, k, 64, 1, dt)
    idx, _, _ = routing(gen, T, E, k)
    w, dw = weights(gen, T, k), torch.randn(T, k, generator=gen)
    x, Wg = torch.randn(T, d, generator=gen).to(dt), (0.02 * torch.randn(d, E, generator=gen)).to(dt)
    return B, p, gen, dt, idx, w, dw, x, Wg


def workspace(B, p):
    # what the call finds there is not its own
    return torch.full((max(256, B.moe_backward_workspace_bytes(p)),), 255, dtype=torch.uint8, device="cuda")


def call(B, p, x, Wg, idx, w, dw, want="xwb", status=None, stream=None):
    T, d, E = p.T, p.d, p.E
    dx = torch.full((T, d), float("nan"), dtype=x.dtype, device="cuda") if "x" in want else None
    dWg = torch.full((d, E), float("nan"), device="cuda") if "w" in want else None
    db = torch.full((E,), float("nan"), device="cuda") if "b" in want else None
    ws = workspace(B, p) if "w" in want or "b" in want else None
    B.moe_route_backward(p, x.cuda() if "w" in want else None, Wg.cuda() if "x" in want else None, idx.cuda(), w.cuda(), dw.cuda(), dx, dWg, db,
                         status, ws, stream)
    torch.cuda.synchronize()
    return dx, dWg, db


def expected(idx, w, dw, x, Wg, dt):
    """The gradients in 64 bits and how far fp32 sums may be off."""
    T, k = idx.shape
    E, d = Wg.shape[1], Wg.shape[0]
    ok = (idx >= 0) & (idx < E)
    w, dw = w.double(), dw.double()
    mean = (w * dw).sum(1, keepdim=True)
    dl = torch.where(ok, w * (dw - mean), 0.0)
    # mean: k products and sums; the difference and the product: two more roundings
    off = torch.where(ok, w * (2 * k * 2.0 ** -24 * (w * dw).abs().sum(1, keepdim=True) + 2.0 ** -24 * (dw - mean).abs()) + 2.0 ** -24 * dl.abs(), 0.0)
    dense, dense_off = torch.zeros(T, E, dtype=torch.float64), torch.zeros(T, E, dtype=torch.float64)
    at = torch.where(ok, idx, 0).long()
    dense.scatter_add_(1, at, dl)
    dense_off.scatter_add_(1, at, off)
    n = (dense != 0).sum(0).max().item()
    size_x, size_w = dense.abs() @ Wg.double().abs().t(), x.double().abs().t() @ dense.abs()
    dx, dWg, db = dense @ Wg.double().t(), x.double().t() @ dense, dense.sum(0)
    # k (one expert's n) products and sums in fp32, in any order, then dx one rounding to dtype
    bx = dense_off @ Wg.double().abs().t() + 2 * k * 2.0 ** -24 * size_x + HALF_STEP[dt] * 1.01 * dx.abs()
    bw = x.double().abs().t() @ dense_off + 2 * (n + 1) * 2.0 ** -24 * size_w
    bb = dense_off.sum(0) + 2 * (n + 1) * 2.0 ** -24 * dense.abs().sum(0)
    return [(v, b * 1.01 + 1e-37) for v, b in ((dx, bx), (dWg, bw), (db, bb))]


def check(got, want):
    for g, (ref, bound) in zip(got, want):
        assert bool(((g.cpu().double() - ref).abs() <= bound).all())


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_route_backward(case):
    print(f"case route_backward {case}", flush=True)
    B, p, gen, dt, idx, w, dw, x, Wg = make(*case)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = call(B, p, x, Wg, idx, w, dw, status=status)
    assert int(status.item()) == 0
    check(got, expected(idx, w, dw, x, Wg, dt))
    # each gradient alone, and once more: the same bits
    for i, one in enumerate("xwb"):
        assert torch.equal(call(B, p, x, Wg, idx, w, dw, one)[i], got[i]), one
    assert all(torch.equal(a, b) for a, b in zip(call(B, p, x, Wg, idx, w, dw), got))


def test_every_token_chooses_the_same_experts():
    # one expert has all rows, the others of 256 none
    B, p, gen, dt, idx, w, dw, x, Wg = make(900, 192, 256, 2, "bf16")
    idx[:, 0], idx[:, 1] = 7, 255
    got = call(B, p, x, Wg, idx, w, dw)
    check(got, expected(idx, w, dw, x, Wg, dt))
    rest = [e for e in range(256) if e not in (7, 255)]
    assert bool((got[1].cpu()[:, rest] == 0).all()) and bool((got[2].cpu()[rest] == 0).all())


def test_ids_that_are_no_expert_are_reported_and_left_out():
    B, p, gen, dt, idx, w, dw, x, Wg = make(300, 256, 16, 4, "bf16")
    idx[5, 1], idx[64, 0], idx[299, 3], idx[200, 2] = -1, 16, 2 ** 31 - 1, -2 ** 31
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    check(call(B, p, x, Wg, idx, w, dw, status=status), expected(idx, w, dw, x, Wg, dt))
    assert int(status.item()) == B.MOE_ERR_BAD_ROUTING
    for want in "xwb":
        status.zero_()
        call(B, p, x, Wg, idx, w, dw, want, status)
        assert int(status.item()) == B.MOE_ERR_BAD_ROUTING
    call(B, p, x, Wg, idx, w, dw)


def test_not_finite_gradients_reach_their_own_token_and_experts_only():
    B, p, gen, dt, idx, w, dw, x, Wg = make(400, 128, 12, 3, "bf16")
    dw[100, 1] = float("nan")
    dx, dWg, db = call(B, p, x, Wg, idx, w, dw)
    bad_t = torch.isnan(dx.cpu()).any(1)
    assert bad_t.nonzero().flatten().tolist() == [100]
    hit = sorted(idx[100].tolist())
    assert torch.isnan(db.cpu()).nonzero().flatten().tolist() == hit
    assert torch.isnan(dWg.cpu()).any(0).nonzero().flatten().tolist() == hit


@pytest.mark.parametrize("T,d,E,k", [(4, 64, 6, 3), (3, 128, 16, 8)])
def test_gate_gradient_agrees_with_differences(T, d, E, k):
    from paper_2605_00686_amd import binding as B
    gen = torch.Generator().manual_seed(T)
    p = B.problem(T, d, E, k, 64, 1, "f32")
    x, Wg, bias = torch.randn(T, d, generator=gen), 0.1 * torch.randn(d, E, generator=gen), torch.randn(E, generator=gen)
    idx = torch.empty((T, k), dtype=torch.int32, device="cuda")
    w = torch.empty((T, k), device="cuda")
    B.moe_route(p, x.cuda(), Wg.cuda(), bias.cuda(), idx, w)
    dw = torch.randn(T, k, generator=gen)
    dx, dWg, db = call(B, p, x, Wg, idx, w, dw)
    chosen = idx.cpu().long()

    def loss(x, Wg, bias):
        return (torch.softmax(torch.gather(x @ Wg + bias, 1, chosen), 1) * dw.double()).sum()
    base, step = [x.double(), Wg.double(), bias.double()], 1e-4
    for at, grad in enumerate((dx, dWg, db)):
        flat = grad.cpu().double().reshape(-1)
        for i in torch.randperm(flat.numel(), generator=gen)[:24].tolist():
            pair = []
            for sign in (1, -1):
                moved = [b.clone() for b in base]
                moved[at].reshape(-1)[i] += sign * step
                pair.append(loss(*moved))
            diff = float(pair[0] - pair[1]) / (2 * step)
            # differences: step^2 / 6 of a third derivative (at most the sum of |dw| times |x|^3 or |Wg|^3, under 300 here) and roundings; the
            # kernel: fp32 weights (2^-22 each) and sums of order ten
            assert abs(diff - float(flat[i])) <= 300 * step ** 2 + 1e-9 + 100 * 2.0 ** -23


def test_tokens_past_32_bit_offsets():
    # 2.2e9 elements of x and dx
    from paper_2605_00686_amd import binding as B
    T, d, E, k = 300_032, 7168, 4, 2
    p = B.problem(T, d, E, k, 64, 1, "bf16")
    gen = torch.Generator(device="cuda").manual_seed(6)
    x = torch.empty((T, d), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    Wg = torch.empty((d, E), dtype=torch.bfloat16, device="cuda").normal_(0.0, 0.02, generator=gen)
    idx = torch.topk(torch.rand((T, E), generator=gen, device="cuda"), k, dim=1).indices.to(torch.int32)
    w = torch.softmax(torch.randn((T, k), generator=gen, device="cuda"), 1)
    dw = torch.zeros((T, k), device="cuda")
    dw[-5:] = torch.randn((5, k), generator=gen, device="cuda")  # the last tokens alone have a gradient
    dx, dWg, db = torch.empty_like(x), torch.empty((d, E), device="cuda"), torch.empty(E, device="cuda")
    B.moe_route_backward(p, x, Wg, idx, w, dw, dx, dWg, db, None, workspace(B, p))
    torch.cuda.synchronize()
    want = expected(idx[-5:].cpu(), w[-5:].cpu(), dw[-5:].cpu(), x[-5:].cpu(), Wg.cpu(), torch.bfloat16)
    check((dx[-5:], dWg, db), want)
    assert float(dx[:-5].abs().max()) == 0.0


def test_other_stream_and_captured_graph():
    B, p, gen, dt, idx, w, dw, x, Wg = make(700, 512, 32, 4, "bf16")
    idx, w, dw, x, Wg = (t.cuda() for t in (idx, w, dw, x, Wg))
    outs = [torch.empty_like(x), torch.empty((512, 32), device="cuda"), torch.empty(32, device="cuda")]
    ws = workspace(B, p)

    def go(stream=None):
        B.moe_route_backward(p, x, Wg, idx, w, dw, *outs, None, ws, stream)
    go()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    for t in outs:
        t.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    go(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for _ in range(4):
        for t in outs:
            t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs))
        go()
        torch.cuda.synchronize()


@pytest.mark.parametrize("T,d,E,k,dtype", [(300, 192, 12, 3, "bf16"), (200, 80, 140, 4, "f32"), (70, 320, 70, 2, "bf16"), (500, 128, 200, 2, "bf16")])
def test_not_finite_inputs_reach_the_chosen_experts_and_tokens_only(T, d, E, k, dtype):
    B, p, gen, dt, idx, w, dw, x, Wg = make(T, d, E, k, dtype)
    odd = [(3, 5, float("inf")), (3, 6, float("nan")), (T - 1, d - 1, float("-inf")), (T // 2, 5, float("nan"))]
    clean = x.clone()
    for t, c, v in odd:
        x[t, c], clean[t, c] = v, 0.0
    odd_e = int(idx[1, 0])
    Wg[7, odd_e] = float("inf")
    dx, dWg, db = (t.cpu() for t in call(B, p, x, Wg, idx, w, dw))
    # dx: column 7 of the tokens that chose the expert
    bad = torch.zeros(T, d, dtype=torch.bool)
    bad[(idx == odd_e).any(1), 7] = True
    assert torch.equal(~torch.isfinite(dx), bad)
    # dWg: the columns of x at hand, of the token's experts; everything else as if those numbers were zero
    bad = torch.zeros(d, E, dtype=torch.bool)
    for t, c, v in odd:
        bad[c, idx[t].long()] = True
    assert torch.equal(~torch.isfinite(dWg), bad)
    (_, _), (ref, bound), (ref_b, bound_b) = expected(idx, w, dw, clean, torch.zeros_like(Wg), dt)
    assert bool(((dWg.double() - ref).abs() <= bound)[~bad].all())
    assert bool(((db.double() - ref_b).abs() <= bound_b).all())


# several parts of the tokens together with two groups of experts, whose number is odd or a multiple of 4 and not of 8, and chunks of columns cut short
@pytest.mark.parametrize("case", [(2500, 144, 131, 3, "f32"), (2100, 192, 129, 9, "bf16"), (3001, 64, 244, 2, "bf16"), (1900, 448, 65, 5, "bf16"),
                                  (1700, 80, 68, 12, "f32"), (5000, 64, 64, 1, "bf16"), (1111, 704, 256, 17, "f32")],
                         ids=lambda c: "T%d_d%d_E%d_k%d_%s" % c)
def test_parts_and_groups(case):
    print(f"case parts and groups {case}", flush=True)
    B, p, gen, dt, idx, w, dw, x, Wg = make(*case)
    got = call(B, p, x, Wg, idx, w, dw)
    check(got, expected(idx, w, dw, x, Wg, dt))
    assert torch.equal(call(B, p, x, Wg, idx, w, dw, "w")[1], got[1])
    assert torch.equal(call(B, p, x, Wg, idx, w, dw, "b")[2], got[2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_expert(dtype):
    # a weight of exactly one has no gradient; any other is treated as given
    B, p, gen, dt, idx, w, dw, x, Wg = make(130, 128, 1, 1, dtype)
    assert all(float(g.abs().max()) == 0.0 for g in call(B, p, x, Wg, idx, w, dw))
    w = torch.rand(130, 1, generator=gen)
    check(call(B, p, x, Wg, idx, w, dw), expected(idx, w, dw, x, Wg, dt))

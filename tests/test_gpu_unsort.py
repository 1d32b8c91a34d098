"""GPU tests of moe_unsort and moe_unsort_backward against sums in 64 bits."""
import pytest
import torch

from tests.train_forms import HALF_STEP, dtype_of, routing, used_rows, weights

pytestmark = pytest.mark.gpu

# T, d, E, k, capacity (0 = ragged), dtype: one token and many, rows from 64 bytes (fewer pieces than lanes) to past 28 KB, odd
# numbers of pieces, k from 1 to 32, experts without rows, experts beyond their capacity
CASES = [(1, 2048, 128, 8, 0, "bf16"), (1, 64, 1, 1, 0, "bf16"), (1, 16, 2, 2, 0, "f32"), (2, 7168, 9, 3, 0, "bf16"), (3, 192, 256, 32, 0, "bf16"),
         (5, 14400, 7, 6, 0, "bf16"), (7, 7216, 5, 4, 0, "f32"), (63, 1040, 17, 9, 0, "f32"), (64, 512, 8, 2, 16, "bf16"),
         (129, 320, 12, 5, 64, "f32"), (255, 960, 256, 8, 8, "bf16"), (257, 2112, 48, 17, 0, "bf16"), (700, 1088, 33, 7, 150, "bf16"),
         (1025, 64, 4, 1, 0, "bf16"), (1500, 448, 16, 16, 0, "bf16"), (2049, 1024, 8, 2, 512, "f32"), (4100, 256, 64, 8, 0, "bf16"),
         (16390, 64, 32, 3, 0, "bf16"), (333, 4096, 16, 12, 0, "bf16"), (40, 128, 40, 31, 1, "bf16")]
IDS = ["T%d_d%d_E%d_k%d_C%d_%s" % c for c in CASES]


def make(T, d, E, k, C, dtype):
    from paper_2605_00686_amd import binding as B
    dt = dtype_of(dtype)
    gen = torch.Generator().manual_seed(T * 31 + d + k)
    idx, inv, counts = routing(gen, T, E, k, C)
    n = E * C if C else T * k
    rows = torch.randn(n, d, generator=gen).to(dt)
    if C:
        rows[~used_rows(counts, C)] = float("nan")  # nobody may look at these
    w = weights(gen, T, k)
    w[inv.reshape(T, k) < 0] = float("nan")  # nor at the weight of a slot without a row
    return B, B.problem(T, d, E, k, 64, 1, dt, capacity=C), gen, dt, inv, counts, rows, w


def gathered(inv, rows, T, k):
    got = rows.double()[inv.long().clamp(min=0)]
    return torch.where((inv >= 0)[:, None], got, 0.0).reshape(T, k, -1)


@pytest.mark.parametrize("case", CASES, ids=IDS)
@pytest.mark.parametrize("weighted,added", [(True, False), (False, True), (True, True)])
def test_unsort(case, weighted, added):
    T, d, E, k, C, dtype = case
    print(f"case unsort {case} weighted={weighted} added={added}", flush=True)
    B, p, gen, dt, inv, counts, rows, w = make(*case)
    addend = torch.randn(T, d, generator=gen).to(dt)
    out = torch.full((T, d), float("nan"), dtype=dt, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.moe_unsort(p, rows.cuda(), inv.cuda(), w.cuda() if weighted else None, addend.cuda() if added else None, out, status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    terms = gathered(inv, rows, T, k)
    if weighted:
        terms = terms * torch.where(inv.reshape(T, k) >= 0, w.double(), 0.0)[:, :, None]
    if added:
        terms = torch.cat([terms, addend.double()[:, None]], 1)
    ref = terms.sum(1)
    # k + 1 fp32 roundings of partial sums (and k of products, where they are not fused), each 2^-24 of at most the sum of magnitudes; one to dtype
    bound = 2 * (k + 1) * 2.0 ** -24 * terms.abs().sum(1) + HALF_STEP[dt] * (1 + 2.0 ** -10) * ref.abs() + 1e-37
    assert bool(((out.cpu().double() - ref).abs() <= bound).all())


@pytest.mark.parametrize("case", CASES, ids=IDS)
@pytest.mark.parametrize("weighted", [True, False])
def test_unsort_backward(case, weighted):
    T, d, E, k, C, dtype = case
    print(f"case unsort_backward {case} weighted={weighted}", flush=True)
    B, p, gen, dt, inv, counts, rows, w = make(*case)
    dout = torch.randn(T, d, generator=gen).to(dt)
    drows = torch.full(rows.shape, 7.0, dtype=dt, device="cuda")
    dw = torch.full((T, k), float("nan"), device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = (dout.cuda(), rows.cuda(), inv.cuda(), w.cuda() if weighted else None, counts.cuda() if C else None)
    B.moe_unsort_backward(p, *args, drows, dw, status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    has = (inv >= 0)
    factor = torch.where(has, w.reshape(-1).double() if weighted else torch.ones(T * k, dtype=torch.float64), 0.0)
    ref = torch.zeros(rows.shape, dtype=torch.float64)
    ref[inv[has].long()] = (factor[:, None] * dout.double().repeat_interleave(k, 0))[has]
    # one fp32 rounding of the product, one to dtype; unused rows exactly zero
    half = HALF_STEP[dt]
    assert bool(((drows.cpu().double() - ref).abs() <= (half + 2.0 ** -24) * (1 + 2.0 ** -8) * ref.abs() + 1e-37).all())
    if C:
        assert bool((drows.cpu()[~used_rows(counts, C)] == 0).all())
    terms = gathered(inv, rows, T, k) * dout.double()[:, None]
    # d products and sums in fp32, in any order
    bound = 2 * d * 2.0 ** -24 * terms.abs().sum(-1) + 1e-37
    assert bool(((dw.cpu().double() - terms.sum(-1)).abs() <= bound).all())
    assert bool((dw.cpu()[inv.reshape(T, k) < 0] == 0).all())
    # the outputs one at a time, and the rows' gradient in place of the rows: the same bits
    only = torch.full_like(drows, 7.0)
    B.moe_unsort_backward(p, args[0], None, args[2], args[3], args[4], only, None, status)
    assert torch.equal(only, drows)
    only_w = torch.empty_like(dw)
    B.moe_unsort_backward(p, *args, None, only_w, status)
    assert torch.equal(only_w, dw)
    same = args[1].clone()
    B.moe_unsort_backward(p, args[0], same, *args[2:], same, only_w, status)
    torch.cuda.synchronize()
    assert torch.equal(same, drows) and torch.equal(only_w, dw) and int(status.item()) == 0


def test_unsort_gradient_agrees_with_differences():
    T, d, E, k = 6, 64, 8, 3
    B, p, gen, dt, inv, counts, rows, w = make(T, d, E, k, 0, "f32")
    dout = torch.randn(T, d, generator=gen)
    drows, dw = torch.empty(T * k, d, device="cuda"), torch.empty(T, k, device="cuda")
    B.moe_unsort_backward(p, dout.cuda(), rows.cuda(), inv.cuda(), w.cuda(), None, drows, dw, None)

    def loss(rows, w):
        return ((rows[inv.long()].reshape(T, k, d) * w[:, :, None]).sum(1) * dout.double()).sum()
    step = 1e-3  # (the loss is linear in each: differences are exact but for 64-bit roundings)
    for grad, at, n in ((drows, 0, 12), (dw, 1, T * k)):
        base = [rows.double(), w.double()]
        flat = grad.cpu().double().reshape(-1)
        for i in torch.randperm(flat.numel(), generator=gen)[:n].tolist():
            up, down = base[at].clone(), base[at].clone()
            up.reshape(-1)[i] += step
            down.reshape(-1)[i] -= step
            pair = [loss(*(v if at == 0 else base[0], v if at == 1 else base[1])) for v in (up, down)]
            diff = float(pair[0] - pair[1]) / (2 * step)
            # fp32 roundings of the kernel (as above, d products of order one), and 1e-13 / step of the difference
            assert abs(diff - float(flat[i])) <= 2 * d * 2.0 ** -24 * 8 + 1e-8


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_not_finite_numbers_stay_where_they_are(dtype):
    T, d, E, k = 5, 128, 8, 2
    B, p, gen, dt, inv, counts, rows, w = make(T, d, E, k, 0, dtype)
    slot = 2 * k + 1
    rows[inv[slot].long(), 5], rows[inv[slot].long(), 9] = float("inf"), float("nan")
    out = torch.empty((T, d), dtype=dt, device="cuda")
    B.moe_unsort(p, rows.cuda(), inv.cuda(), w.cuda(), None, out, None)
    got = out.cpu()
    assert torch.isnan(got[2, 9]) and got[2, 5] == float("inf")
    got[2, 9], got[2, 5] = 0, 0
    assert bool(torch.isfinite(got).all())
    dout = torch.randn(T, d, generator=gen).to(dt)
    drows, dw = torch.empty((T * k, d), dtype=dt, device="cuda"), torch.empty((T, k), device="cuda")
    B.moe_unsort_backward(p, dout.cuda(), rows.cuda(), inv.cuda(), w.cuda(), None, drows, dw, None)
    bad = torch.isnan(dw.cpu())
    assert bool(bad[2, 1]) and int(bad.sum()) == 1 and bool(torch.isfinite(drows.cpu()).all())


def test_rows_that_do_not_exist_are_reported_and_left_out():
    T, d, E, k = 70, 256, 8, 2
    B, p, gen, dt, inv, counts, rows, w = make(T, d, E, k, 0, "bf16")
    bad = inv.clone()
    bad[3], bad[10], bad[70], bad[139] = T * k, -2, 2 ** 31 - 1, -2 ** 31
    dropped = torch.where((bad >= 0) & (bad < T * k), bad, -1)
    outs = []
    for which in (bad, dropped):
        out = torch.zeros((T, d), dtype=dt, device="cuda")
        drows, dw = torch.zeros((T * k, d), dtype=dt, device="cuda"), torch.empty((T, k), device="cuda")
        status = torch.zeros(2, dtype=torch.int32, device="cuda")
        B.moe_unsort(p, rows.cuda(), which.cuda(), w.cuda(), None, out, status[:1])
        B.moe_unsort_backward(p, rows.cuda()[:T], rows.cuda(), which.cuda(), w.cuda(), None, drows, dw, status[1:])
        outs.append((out, drows, dw))
        want = B.MOE_ERR_BAD_ROUTING if which is bad else 0
        assert status.tolist() == [want, want]
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    B.moe_unsort(p, rows.cuda(), bad.cuda(), w.cuda(), None, out, None)  # nobody asks for the status
    assert torch.equal(out, outs[0][0])


def test_addend_in_place_and_counts_past_the_capacity():
    T, d, E, k, C = 90, 320, 4, 2, 16
    B, p, gen, dt, inv, counts, rows, w = make(T, d, E, k, C, "bf16")
    assert int(counts.max()) > C
    addend = torch.randn(T, d, generator=gen).to(dt).cuda()
    out = torch.empty_like(addend)
    B.moe_unsort(p, rows.cuda(), inv.cuda(), w.cuda(), addend, out, None)
    B.moe_unsort(p, rows.cuda(), inv.cuda(), w.cuda(), addend, addend, None)
    assert torch.equal(out, addend)


def test_rows_past_32_bit_offsets():
    # 2.2e9 elements, 4.4 GB: the last rows lie past 2^32 bytes and 2^31 elements
    from paper_2605_00686_amd import binding as B
    T, d, E, k = 38400, 7168, 16, 8
    p = B.problem(T, d, E, k, 64, 1, "bf16")
    gen = torch.Generator(device="cuda").manual_seed(5)
    inv = torch.randperm(T * k, generator=gen, device="cuda").to(torch.int32)
    rows = torch.empty((T * k, d), dtype=torch.bfloat16, device="cuda")
    rows.normal_(generator=gen)
    w = torch.rand((T, k), generator=gen, device="cuda")
    out = torch.empty((T, d), dtype=torch.bfloat16, device="cuda")
    dout = torch.empty_like(out).normal_(generator=gen)
    dw = torch.empty((T, k), device="cuda")
    B.moe_unsort(p, rows, inv, w, None, out, None)
    some = torch.cat([(inv == T * k - 1).nonzero()[:, 0] // k, torch.tensor([0, 1, T // 2, T - 1], device="cuda")])
    terms = rows[inv.reshape(T, k)[some].long()].double() * w[some].double()[:, :, None]
    bound = 2 * k * 2.0 ** -24 * terms.abs().sum(1) + 2.0 ** -8 * 1.001 * terms.sum(1).abs()
    assert bool(((out[some].double() - terms.sum(1)).abs() <= bound).all())
    want = (rows[inv.reshape(T, k)[some].long()].double() * dout[some].double()[:, None])
    B.moe_unsort_backward(p, dout, rows, inv, w, None, rows, dw, None)
    assert bool(((dw[some].double() - want.sum(-1)).abs() <= 2 * d * 2.0 ** -24 * want.abs().sum(-1)).all())
    got = rows[inv.reshape(T, k)[some].long()].double()
    ref = w[some].double()[:, :, None] * dout[some].double()[:, None]
    assert bool(((got - ref).abs() <= (2.0 ** -8 + 2.0 ** -24) * 1.01 * ref.abs()).all())


def test_other_stream_and_captured_graph():
    T, d, E, k, C = 300, 512, 8, 2, 64
    B, p, gen, dt, inv, counts, rows, w = make(T, d, E, k, C, "bf16")
    dout = torch.randn(T, d, generator=gen).to(dt).cuda()
    rows, inv, w, counts = rows.cuda(), inv.cuda(), w.cuda(), counts.cuda()
    out, drows, dw = torch.empty_like(dout), torch.empty_like(rows), torch.empty((T, k), device="cuda")

    def both(stream=None):
        B.moe_unsort(p, rows, inv, w, None, out, None, stream)
        B.moe_unsort_backward(p, dout, rows, inv, w, counts, drows, dw, None, stream)
    both()
    torch.cuda.synchronize()
    want = [t.clone() for t in (out, drows, dw)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for t in (out, drows, dw):
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    both(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (out, drows, dw)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(4):
        for t in (out, drows, dw):
            t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (out, drows, dw)))
        both()
        torch.cuda.synchronize()


# where the gradient's workgroups change: slots of a token apart below 512 tokens, workgroups of 1024 threads for long rows up to 32 tokens
@pytest.mark.parametrize("case", [(32, 2368, 9, 9, 0, "f32"), (33, 2368, 9, 9, 0, "f32"), (32, 2112, 40, 17, 12, "bf16"), (7, 16448, 33, 32, 0, "bf16"),
                                  (511, 1024, 24, 24, 0, "bf16"), (512, 1024, 24, 24, 0, "bf16"), (511, 64, 20, 20, 400, "bf16"), (31, 8192, 8, 1, 5, "f32")],
                         ids=lambda c: "T%d_d%d_E%d_k%d_C%d_%s" % c)
def test_few_tokens(case):
    test_unsort_backward(case, True)
    test_unsort_backward(case, False)

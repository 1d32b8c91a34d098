"""GPU tests of the training calls on more rows than the caches hold, which they read past them: every instance of those forms."""
import pytest
import torch

from tests.train_forms import HALF_STEP, dtype_of, routing, used_rows, weights

pytestmark = pytest.mark.gpu

STREAM = 96 << 20  # bytes of rows from which on they are read past the caches

# T, d, E, k, capacity, dtype: 2, 4 and 8 rows in flight; 1, 2 and 4 pieces per lane; 64, 128, 256 and 1024 lanes per token in the gradient
CASES = [(52_000, 512, 16, 2, 0, "bf16"), (26_000, 1024, 16, 2, 0, "bf16"), (13_000, 2112, 8, 2, 0, "bf16"), (30_000, 448, 16, 4, 0, "bf16"),
         (12_000, 1472, 16, 3, 0, "bf16"), (16_000, 448, 48, 8, 0, "bf16"), (8000, 960, 32, 7, 0, "bf16"), (26_000, 528, 4, 2, 0, "f32"),
         (13_000, 1040, 8, 2, 0, "f32"), (30_000, 240, 9, 4, 0, "f32"), (9000, 720, 24, 11, 0, "f32"), (4000, 1040, 16, 6, 2000, "f32"),
         (5000, 2112, 16, 5, 1600, "bf16"), (50_000, 320, 64, 1, 3000, "bf16"), (32, 50_176, 33, 32, 0, "bf16"), (20, 316_416, 8, 4, 0, "f32"),
         (32, 400_000, 3, 2, 0, "f32")]


def make(T, d, E, k, C, dtype):
    from paper_2605_00686_amd import binding as B
    dt = dtype_of(dtype)
    gen = torch.Generator().manual_seed(T + d + k)
    idx, inv, counts = routing(gen, T, E, k, C, skew=0.5)
    n = E * C if C else T * k
    assert n * d * dt.itemsize > STREAM
    w = weights(gen, T, k) if k > 1 else torch.rand(T, 1, generator=gen)
    w[inv.reshape(T, k) < 0] = float("nan")
    dev = torch.Generator(device="cuda").manual_seed(T)

    def normal(*shape):
        return torch.empty(shape, dtype=dt, device="cuda").normal_(generator=dev)
    rows = normal(n, d)
    used = used_rows(counts, C).cuda() if C else None
    if C:
        rows[~used] = float("nan")
    return B, B.problem(T, d, E, k, 64, 1, dt, capacity=C), dt, inv.cuda(), counts.cuda(), used, rows, w.cuda(), normal


def tokens_at_a_time(T, d, k):
    step = max(1, (1 << 25) // (d * k))
    return [slice(t, min(T, t + step)) for t in range(0, T, step)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "T%d_d%d_E%d_k%d_C%d_%s" % c)
def test_unsort_and_its_gradient(case):
    T, d, E, k, C, dtype = case
    print(f"case stream {case}", flush=True)
    B, p, dt, inv, counts, used, rows, w, normal = make(*case)
    addend, dout, status = normal(T, d), normal(T, d), torch.zeros(1, dtype=torch.int32, device="cuda")
    has, at = (inv >= 0).reshape(T, k), inv.reshape(T, k).long().clamp(min=0)
    half = HALF_STEP[dt]
    for weighted in (True, False):
        factor = torch.where(has, w.double() if weighted else 1.0, 0.0)
        out = torch.full_like(addend, float("nan"))
        B.moe_unsort(p, rows, inv, w if weighted else None, None if weighted else addend, out, status)
        drows, dw = torch.full_like(rows, 7.0), torch.full((T, k), float("nan"), device="cuda")
        B.moe_unsort_backward(p, dout, rows, inv, w if weighted else None, counts if C else None, drows, dw, status)
        for ts in tokens_at_a_time(T, d, k):
            mine = torch.where(has[ts][:, :, None], rows[at[ts]].double(), 0.0)
            terms = mine * factor[ts][:, :, None]
            if not weighted:
                terms = torch.cat([terms, addend[ts].double()[:, None]], 1)
            ref = terms.sum(1)
            # (as in the tests of smaller calls) k + 1 fp32 roundings of sums and k of products, and one to dtype
            bound = 2 * (k + 1) * 2.0 ** -24 * terms.abs().sum(1) + half * (1 + 2.0 ** -10) * ref.abs() + 1e-37
            assert bool(((out[ts].double() - ref).abs() <= bound).all())
            g = dout[ts].double()[:, None]
            terms = mine * g
            assert bool(((dw[ts].double() - terms.sum(-1)).abs() <= 2 * d * 2.0 ** -24 * terms.abs().sum(-1) + 1e-37).all())
            ref = factor[ts][:, :, None] * g
            got = torch.where(has[ts][:, :, None], drows[at[ts]].double(), 0.0)
            assert bool(((got - ref).abs() <= (half + 2.0 ** -24) * (1 + 2.0 ** -8) * ref.abs() + 1e-37).all())
        if C:
            assert bool((drows[~used] == 0).all())
        if weighted:  # the gradient in place of the rows: the same bits
            same, dw2 = rows.clone(), torch.empty_like(dw)
            B.moe_unsort_backward(p, dout, same, inv, w, counts if C else None, same, dw2, status)
            assert torch.equal(same, drows) and torch.equal(dw2, dw)
    assert int(status.item()) == 0


# T, k, E, f, capacity, dtype
SWIGLU = [(13_000, 2, 4, 1088, 0, "bf16"), (9000, 2, 4, 1040, 0, "f32"), (4000, 2, 8, 1088, 3400, "bf16"), (9000, 1, 8, 720, 3100, "f32"), (3600, 1, 4, 7232, 0, "bf16")]


@pytest.mark.parametrize("joint", [False, True])
@pytest.mark.parametrize("case", SWIGLU, ids=lambda c: "T%d_k%d_E%d_f%d_C%d_%s" % c)
def test_swiglu_and_its_gradient(case, joint):
    """The same bits as of calls on a quarter or an eighth of the rows, which the caches hold."""
    from paper_2605_00686_amd import binding as B
    T, k, E, f, C, dtype = case
    print(f"case stream swiglu {case} joint={joint}", flush=True)
    dt = dtype_of(dtype)
    n, blocks, parts = E * C if C else T * k, -(-f // 32), E if C else 4
    assert n * f * 2 * dt.itemsize > STREAM and n * f * (2 + dt.itemsize) > STREAM and n // parts * f * 2 * dt.itemsize < STREAM
    gen = torch.Generator(device="cuda").manual_seed(f)

    def normal(*shape):
        return torch.empty(shape, dtype=dt, device="cuda").normal_(generator=gen)

    def halves():
        both = normal(n, 2 * f) * torch.exp(normal(2 * f))
        return (both[:, :f], both[:, f:]) if joint else (both[:, :f].contiguous(), both[:, f:].contiguous())

    def outputs(rows):
        return (torch.full((rows, f), 7.0, dtype=dt, device="cuda"), torch.full((rows, 2, f), 99, dtype=torch.uint8, device="cuda"),
                torch.full((rows, 2, blocks), 99, dtype=torch.uint8, device="cuda"))
    g, u = halves()
    counts = torch.tensor([(i * 997) % (C + 300) for i in range(E)], dtype=torch.int32, device="cuda") if C else None
    dh = normal(n, f)
    if C:
        unused = ~used_rows(counts.cpu().clamp(max=C), C).cuda()
        g[unused], u[unused], dh[unused] = float("nan"), float("nan"), float("nan")
    p = B.problem(T, 64, E, k, f, 1, dt, capacity=C)
    h, codes, scales = outputs(n)
    B.moe_swiglu(p, g, u, counts, h, codes, scales)
    dg, du = halves()
    h2 = torch.full_like(h, 7.0)
    B.moe_swiglu_backward(p, dh, codes, scales, counts, dg, du, h2)
    small = B.problem(1 if C else T // parts, 64, 1 if C else E, 1 if C else k, f, 1, dt, capacity=C)
    rows = n // parts
    for i in range(parts):
        at, cnt = slice(i * rows, (i + 1) * rows), counts[i:i + 1].clone() if C else None
        a, b, c = outputs(rows)
        B.moe_swiglu(small, g[at], u[at], cnt, a, b, c)
        assert torch.equal(a, h[at]) and torch.equal(b, codes[at]) and torch.equal(c, scales[at])
        dg1, du1 = torch.full_like(a, 7.0), torch.full_like(a, 7.0)
        B.moe_swiglu_backward(small, dh[at], b, c, cnt, dg1, du1, a)
        assert torch.equal(dg1, dg[at]) and torch.equal(du1, du[at]) and torch.equal(a, h2[at])

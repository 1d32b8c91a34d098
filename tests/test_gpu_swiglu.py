"""GPU tests of moe_swiglu (8-bit codes bit for bit) and moe_swiglu_backward against the definitions in 64 bits."""
import pytest
import torch

from tests.train_forms import HALF_STEP, code_values, decode, dtype_of, encode, used_rows

pytestmark = pytest.mark.gpu

# T, k, E, f, capacity, dtype: rows of one block and of half a one, odd numbers of blocks, rows of more than a workgroup
CASES = [(1, 1, 1, 64, 0, "bf16"), (1, 8, 128, 768, 0, "bf16"), (3, 1, 4, 16, 0, "f32"), (5, 2, 8, 48, 0, "f32"), (7, 3, 5, 80, 4, "f32"),
         (37, 2, 8, 1408, 0, "bf16"), (64, 4, 16, 320, 24, "bf16"), (130, 1, 3, 2112, 64, "bf16"), (9, 2, 4, 14336, 0, "bf16"),
         (33, 5, 48, 1040, 0, "f32"), (1000, 1, 8, 64, 0, "bf16"), (700, 3, 9, 192, 250, "bf16"), (257, 1, 2, 4112, 0, "f32")]
IDS = ["T%d_k%d_E%d_f%d_C%d_%s" % c for c in CASES]


def make(T, k, E, f, C, dtype, joint):
    from paper_2605_00686_amd import binding as B
    dt = dtype_of(dtype)
    p = B.problem(T, 64, E, k, f, 1, dt, capacity=C)
    gen = torch.Generator().manual_seed(T + f + k)
    n = E * C if C else T * k
    counts = torch.randint(0, 2 * C + 1, (E,), generator=gen).to(torch.int32) if C else None  # (some past the capacity, some zero)
    if C:
        counts[0] = 0
    # columns of different size, some blocks far below and above the others
    gu = torch.randn(n, 2 * f, generator=gen) * torch.exp(2 * torch.randn(2 * f, generator=gen))
    gu[:, :16] *= 2.0 ** -20
    gu = gu.to(dt)
    used = used_rows(counts.clamp(max=C), C) if C else torch.ones(n, dtype=torch.bool)
    gu[~used] = float("nan")
    dev = gu.cuda()
    if joint:
        g, u = dev[:, :f], dev[:, f:]
    else:
        g, u = dev[:, :f].contiguous(), dev[:, f:].contiguous()
    return B, p, gen, dt, n, counts, used, gu, g, u


def h_bound(g, u, dt):
    """silu(g) u: exp(-g) with its argument rounded (|g| log2 e 2^-24 in the exponent) and two units of the hardware's, the sum, the
    reciprocal (1 ulp) and two products, one rounding to dtype; below 2^-126 hardware may return zero."""
    s = torch.sigmoid(g)
    rel = (1 - s) * (g.abs() + 4) * 2.0 ** -23 + 6 * 2.0 ** -23
    h = g * s * u
    return h, (rel + HALF_STEP[dt] * (1 + 2.0 ** -8)) * h.abs() + 2.0 ** -118 * (1 + u.abs()) * (1 + g.abs())


@pytest.mark.parametrize("case", CASES, ids=IDS)
@pytest.mark.parametrize("joint", [False, True])
def test_swiglu(case, joint):
    T, k, E, f, C, dtype = case
    print(f"case swiglu {case} joint={joint}", flush=True)
    B, p, gen, dt, n, counts, used, gu, g, u = make(*case, joint)
    blocks = -(-f // 32)
    h = torch.full((n, f), float("nan"), dtype=dt, device="cuda")
    codes = torch.full((n, 2, f), 99, dtype=torch.uint8, device="cuda")
    scales = torch.full((n, 2, blocks), 99, dtype=torch.uint8, device="cuda")
    cnt = counts.cuda() if C else None
    B.moe_swiglu(p, g, u, cnt, h, codes, scales)
    torch.cuda.synchronize()
    x = torch.where(used[:, None], gu.double(), 0.0)
    want, bound = h_bound(x[:, :f], x[:, f:], dt)
    assert bool(((h.cpu().double() - want).abs() <= bound).all())
    values, byte = encode(x.reshape(n * 2, f))
    assert torch.equal(scales.cpu().long(), byte.reshape(n, 2, blocks))
    assert torch.equal(code_values(codes.cpu()), values.reshape(n, 2, f))
    assert bool((h.cpu()[~used] == 0).all()) and bool((codes.cpu()[~used] == 0).all())
    # without codes (a forward pass that keeps nothing) and without h: the same
    alone = torch.full_like(h, float("nan"))
    B.moe_swiglu(p, g, u, cnt, alone, None, None)
    codes_alone, scales_alone = torch.zeros_like(codes), torch.zeros_like(scales)
    B.moe_swiglu(p, g, u, cnt, None, codes_alone, scales_alone)
    assert torch.equal(alone, h) and torch.equal(codes_alone, codes) and torch.equal(scales_alone, scales)


def grad_bounds(g, u, dh, dt):
    s = torch.sigmoid(g)
    silu, slope = g * s, s * (1 + g * (1 - s))
    # as in h_bound for s (relative error r); 1 - s is then off by s r and a rounding, the bracket by |g| times that and two more
    r = (1 - s) * (g.abs() + 4) * 2.0 ** -23 + 3 * 2.0 ** -23
    tiny = 2.0 ** -118 * (1 + g.abs()) ** 2
    off = s * (r * (1 + g.abs() * (1 - s)) + g.abs() * (s * r + 2.0 ** -23) + 4 * 2.0 ** -23 * (1 + g.abs() * (1 - s))) + tiny
    half = HALF_STEP[dt] * (1 + 2.0 ** -8)
    du, dg = dh * silu, dh * u * slope
    return (dg, (dh * u).abs() * (off * (1 + half) + half * slope.abs() + 2.0 ** -22 * slope.abs()) + tiny,
            du, dh.abs() * silu.abs() * (r + half + 3 * 2.0 ** -23) + dh.abs() * tiny + tiny)


@pytest.mark.parametrize("case", CASES, ids=IDS)
@pytest.mark.parametrize("joint", [False, True])
def test_swiglu_backward(case, joint):
    T, k, E, f, C, dtype = case
    print(f"case swiglu_backward {case} joint={joint}", flush=True)
    B, p, gen, dt, n, counts, used, gu, g, u = make(*case, joint)
    blocks = -(-f // 32)
    # every code but the NaNs, and scales that make values from 2^-40 to 2^6 of them
    codes = torch.randint(0, 256, (n, 2, f), generator=gen, dtype=torch.uint8)
    codes[(codes & 127) == 127] = 1
    scales = torch.randint(96, 125, (n, 2, blocks), generator=gen, dtype=torch.uint8)
    codes[~used], scales[~used] = 127, 255
    dh = torch.randn(n, f, generator=gen).to(dt)
    dh[~used] = float("nan")
    cnt = counts.cuda() if C else None
    h = torch.full((n, f), float("nan"), dtype=dt, device="cuda")
    dgu = torch.full((n, 2 * f), float("nan"), dtype=dt, device="cuda")
    dg, du = (dgu[:, :f], dgu[:, f:]) if joint else (dgu.reshape(2, n, f)[0], dgu.reshape(2, n, f)[1])
    B.moe_swiglu_backward(p, dh.cuda(), codes.cuda(), scales.cuda(), cnt, dg, du, h)
    torch.cuda.synchronize()
    codes[~used], scales[~used], dh[~used] = 0, 0, 0.0
    gd, ud = decode(codes, scales)
    want, bound = h_bound(gd, ud, dt)
    assert bool(((h.cpu().double() - want).abs() <= bound).all())
    want_g, bound_g, want_u, bound_u = grad_bounds(gd, ud, dh.double(), dt)
    assert bool(((dg.cpu().double() - want_g).abs() <= bound_g).all())
    assert bool(((du.cpu().double() - want_u).abs() <= bound_u).all())
    if C:
        assert bool((torch.cat([dg, du, h], 1).cpu()[~used] == 0).all())
    again = torch.full_like(dgu, float("nan"))
    ag, au = (again[:, :f], again[:, f:]) if joint else (again.reshape(2, n, f)[0], again.reshape(2, n, f)[1])
    B.moe_swiglu_backward(p, dh.cuda(), codes.cuda(), scales.cuda(), cnt, ag, au, None)  # without h
    assert torch.equal(again, dgu)


def test_codes_hold_every_exponent_and_the_ends_of_the_range():
    from paper_2605_00686_amd import binding as B
    gen = torch.Generator().manual_seed(3)
    rows = []
    for e in range(-149, 128):  # the block's largest: 2^e and 1.75 2^e (the last that fits the exponent), its neighbours
        for m in (1.0, 1.75, 1.7499999, 1.7500001, 1.9999999):
            row = (torch.rand(64, generator=gen, dtype=torch.float64) * 2 - 1) * 2.0 ** e
            row[int(torch.randint(0, 32, (1,), generator=gen))] = m * 2.0 ** e
            row[32:] = 0.0 if e % 2 else -row[:32]
            rows.append(row)
    # halves between two codes, at every step of a block whose scale is one: they go to the even code
    grid = torch.tensor([v for v in range(127)], dtype=torch.uint8)
    values = code_values(grid)
    halves = torch.cat([(values[1:] + values[:-1]) / 2, torch.tensor([448.0] * 2, dtype=torch.float64)]).reshape(4, 32)
    halves[:, 0] = 448.0
    rows += list(torch.cat([halves, -halves], 1))
    g = torch.stack(rows).to(torch.float32)
    n = g.shape[0]
    p = B.problem(n, 64, 1, 1, 64, 1, "f32")
    codes = torch.empty((n, 2, 64), dtype=torch.uint8, device="cuda")
    scales = torch.empty((n, 2, 2), dtype=torch.uint8, device="cuda")
    B.moe_swiglu(p, g.cuda(), g.flip(1).contiguous().cuda(), None, None, codes, scales)
    values, byte = encode(torch.cat([g, g.flip(1)], 1).double().reshape(n * 2, 64))
    assert torch.equal(scales.cpu().long(), byte.reshape(n, 2, 2))
    got = code_values(codes.cpu())
    assert torch.equal(got, values.reshape(n, 2, 64))
    # what is kept is within half a step of e4m3 of what was: 2^-4 of a value, or half of 2^-9 of the scale
    dec_g, _ = decode(codes.cpu(), scales.cpu())
    low = torch.exp2(scales[:, 0].cpu().double() - 127.0 - 10.0).repeat_interleave(32, 1)
    assert bool(((dec_g - g.double()).abs() <= torch.maximum(2.0 ** -4 * g.double().abs(), low)).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_not_finite_numbers_keep_to_themselves(dtype):
    from paper_2605_00686_amd import binding as B
    dt = dtype_of(dtype)
    gen = torch.Generator().manual_seed(11)
    n, f = 4, 64
    p = B.problem(n, 64, 1, 1, f, 1, dt)
    g, u = torch.randn(n, f, generator=gen).to(dt), torch.randn(n, f, generator=gen).to(dt)
    g[1, 3], g[1, 4], g[2, 40], u[2, 41], u[3, :32] = float("inf"), float("-inf"), float("nan"), float("nan"), float("inf")
    h = torch.empty((n, f), dtype=dt, device="cuda")
    codes, scales = torch.empty((n, 2, f), dtype=torch.uint8, device="cuda"), torch.empty((n, 2, 2), dtype=torch.uint8, device="cuda")
    B.moe_swiglu(p, g.cuda(), u.cuda(), None, h, codes, scales)
    values, byte = encode(torch.stack([g, u], 1).double().reshape(n * 2, f))
    got = code_values(codes.cpu()).reshape(n * 2, f)
    assert torch.equal(torch.isnan(got), torch.isnan(values))
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(values)) and torch.equal(scales.cpu().long().reshape(n * 2, 2), byte)
    want = g.double() * torch.sigmoid(g.double()) * u.double()
    assert torch.equal(torch.isnan(h.cpu()), torch.isnan(want)) and torch.equal(torch.isinf(h.cpu()), torch.isinf(want))
    dh = torch.ones((n, f), dtype=dt, device="cuda")
    dg, du = torch.empty_like(dh), torch.empty_like(dh)
    B.moe_swiglu_backward(p, dh, codes, scales, None, dg, du, h)
    bad = torch.isnan(values).reshape(n, 2, f).any(1)
    assert torch.equal(torch.isnan(dg.cpu()), bad) and torch.equal(torch.isnan(h.cpu()), bad)
    assert torch.equal(torch.isnan(du.cpu()), torch.isnan(values).reshape(n, 2, f)[:, 0])


def test_gradient_agrees_with_differences():
    from paper_2605_00686_amd import binding as B
    gen = torch.Generator().manual_seed(2)
    n, f = 8, 64
    p = B.problem(n, 64, 1, 1, f, 1, "f32")
    codes = torch.randint(0, 256, (n, 2, f), generator=gen, dtype=torch.uint8)
    codes[(codes & 127) == 127] = 1
    scales = torch.full((n, 2, 2), 127 - 6, dtype=torch.uint8)  # values up to 7
    dh = torch.randn(n, f, generator=gen)
    dg, du = torch.empty((n, f), device="cuda"), torch.empty((n, f), device="cuda")
    B.moe_swiglu_backward(p, dh.cuda(), codes.cuda(), scales.cuda(), None, dg, du, None)
    g, u = decode(codes, scales)

    def loss(g, u):
        return g / (1 + torch.exp(-g)) * u * dh.double()
    step = 1e-4
    num_g = (loss(g + step, u) - loss(g - step, u)) / (2 * step)
    num_u = (loss(g, u + step) - loss(g, u - step)) / (2 * step)
    # differences: step^2 / 6 of the third derivative (below 1 for silu) and 64-bit roundings / step; the kernel: as in grad_bounds, for |g| up to 7
    scale = (dh.double() * u).abs() + 1
    assert bool(((dg.cpu().double() - num_g).abs() <= scale * (step ** 2 + 1e-10 + 80 * 2.0 ** -23)).all())
    assert bool(((du.cpu().double() - num_u).abs() <= (dh.double().abs() * (1 + g.abs()) + 1) * (1e-10 + 20 * 2.0 ** -23)).all())


def test_rows_past_32_bit_offsets():
    from paper_2605_00686_amd import binding as B
    T, k, f = 38400, 2, 14336  # g and u side by side: 2.2e9 elements
    p = B.problem(T, 64, 8, k, f, 1, "bf16")
    n = T * k
    gen = torch.Generator(device="cuda").manual_seed(4)
    gu = torch.empty((n, 2 * f), dtype=torch.bfloat16, device="cuda")
    gu.normal_(generator=gen)
    h = torch.empty((n, f), dtype=torch.bfloat16, device="cuda")
    codes = torch.empty((n, 2, f), dtype=torch.uint8, device="cuda")
    scales = torch.empty((n, 2, f // 32), dtype=torch.uint8, device="cuda")
    B.moe_swiglu(p, gu[:, :f], gu[:, f:], None, h, codes, scales)
    some = torch.tensor([0, 1, n // 2, n - 2, n - 1], device="cuda")
    x = gu[some].cpu().double()
    want, bound = h_bound(x[:, :f], x[:, f:], torch.bfloat16)
    assert bool(((h[some].cpu().double() - want).abs() <= bound).all())
    values, byte = encode(x.reshape(-1, f))
    assert torch.equal(code_values(codes[some].cpu()).reshape(-1, f), values)
    assert torch.equal(scales[some].cpu().long().reshape(byte.shape), byte)
    dh = h.clone()
    B.moe_swiglu_backward(p, dh, codes, scales, None, gu[:, :f], gu[:, f:], h)
    g, u = decode(codes[some].cpu(), scales[some].cpu())
    want_g, bound_g, want_u, bound_u = grad_bounds(g, u, dh[some].cpu().double(), torch.bfloat16)
    got = gu[some].cpu().double()
    assert bool(((got[:, :f] - want_g).abs() <= bound_g).all()) and bool(((got[:, f:] - want_u).abs() <= bound_u).all())


def test_other_stream_and_captured_graph():
    case = (64, 4, 16, 320, 24, "bf16")
    B, p, gen, dt, n, counts, used, gu, g, u = make(*case, True)
    f = case[3]
    cnt = counts.cuda()
    dh = torch.randn(n, f, generator=gen).to(dt).cuda()
    outs = [torch.empty((n, f), dtype=dt, device="cuda"), torch.empty((n, 2, f), dtype=torch.uint8, device="cuda"),
            torch.empty((n, 2, f // 32), dtype=torch.uint8, device="cuda"), torch.empty((n, f), dtype=dt, device="cuda"),
            torch.empty((n, f), dtype=dt, device="cuda")]

    def both(stream=None):
        B.moe_swiglu(p, g, u, cnt, outs[0], outs[1], outs[2], stream)
        B.moe_swiglu_backward(p, dh, outs[1], outs[2], cnt, outs[3], outs[4], outs[0], stream)
    both()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    for t in outs:
        t.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    both(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(4):
        for t in outs:
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs))
        both()
        torch.cuda.synchronize()

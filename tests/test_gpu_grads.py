"""The norm of many gradients and their clipping, against 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
BF, F32 = torch.bfloat16, torch.float32


def draw(gen, sizes, std=1.0):
    """Tensors of (size, type), each a piece of a buffer of its type: most start where 16 bytes do not."""
    flat = {dt: (torch.randn(sum(n for n, t in sizes if t == dt) + 3, generator=gen) * std).to(dt).cuda() for dt in (BF, F32)}
    at, out = {BF: 1, F32: 1}, []
    for n, dt in sizes:
        out.append(flat[dt][at[dt]:at[dt] + n])
        at[dt] += n
    return out


def norm_of(B, tensors):
    total, norm = torch.full((1,), float("nan"), dtype=torch.float64, device="cuda"), torch.full((1,), float("nan"), device="cuda")
    ws = torch.full((B.moe_grad_workspace_bytes(tensors),), 255, dtype=torch.uint8, device="cuda")
    B.moe_grad_norm(tensors, total, norm, ws)
    return total, norm


def want_sum(grads):
    return math.fsum(float(v) ** 2 for g in grads for v in g.double().cpu().tolist())


LISTS = {
    "one_number": [(1, F32)], "few": [(7, BF), (0, F32), (2047, F32), (8, BF), (1, BF)],
    "chunk_ends": [(8191, F32), (8192, F32), (8193, F32), (16383, BF), (16384, BF), (16385, BF)],
    "many": [(3 + 17 * (i % 13), BF if i % 3 else F32) for i in range(300)],
    "long": [(1 << 20, BF), (5, F32), ((1 << 20) + 77, F32)],
}


@pytest.mark.parametrize("name", LISTS)
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("limit", [0.0, 0.37, 1.5])
def test_norm_and_clip(name, in_place, limit):
    from paper_2605_00686_amd import binding as B
    gen = torch.Generator().manual_seed(len(name))
    grads = draw(gen, LISTS[name])
    before = [g.clone() for g in grads]
    outs = grads if in_place else [torch.full_like(g, float("nan")) for g in grads]
    tensors = B.tensor_list(grads, None if in_place else outs)
    total, norm = norm_of(B, tensors)
    want = want_sum(before)
    n = sum(s for s, _ in LISTS[name])
    # squares are exact or rounded once in 64 bits, and n sums are: each by 2^-53 of what it has
    assert abs(float(total) - want) <= (n + 2) * 2.0 ** -53 * want
    assert abs(float(norm) - math.sqrt(want)) <= (2.0 ** -24 + 2.0 ** -30) * math.sqrt(want)
    most = limit * math.sqrt(want)
    B.moe_grad_clip(tensors, total, most)
    factor = min(1.0, torch.tensor(most, dtype=F32).double().item() / math.sqrt(float(total)))
    for g, o in zip(before, outs):
        ref = g.double() * factor
        # fp32: the product in 64 bits, rounded once; bf16: factor, product and output are rounded, the first two to 2^-24
        off = HALF_STEP[g.dtype] * (1 + 2.0 ** -14) * ref.abs() + 2.0 ** -134
        assert ((o.double() - ref).abs() <= off).all()
        if limit > 1:
            assert torch.equal(o, g)


def test_no_tensors():
    from paper_2605_00686_amd import binding as B
    tensors = B.tensor_list([])
    total, norm = norm_of(B, tensors)
    assert float(total) == 0.0 and float(norm) == 0.0
    B.moe_grad_clip(tensors, total, 1.0)


def test_numbers_whose_squares_leave_the_range_of_fp32():
    from paper_2605_00686_amd import binding as B
    grads = [torch.tensor([3e38, -3e38, 1.0], device="cuda"), torch.tensor([2.0 ** -140], device="cuda")]
    tensors = B.tensor_list(grads)
    total, norm = norm_of(B, tensors)
    assert abs(float(total) - 2 * float(grads[0][0].double()) ** 2) < 1e-15 * float(total)
    assert math.isinf(float(norm))  # (past fp32; the sum is not)
    B.moe_grad_clip(tensors, total, 1.0)
    assert abs(float(grads[0][0]) - math.sqrt(0.5)) < 1e-6 and abs(float(grads[0][1]) + math.sqrt(0.5)) < 1e-6
    small = [torch.full((1000,), 2.0 ** -130, device="cuda")]
    total, norm = norm_of(B, B.tensor_list(small))
    assert float(total) == 1000 * 2.0 ** -260


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_norm_that_is_not_finite_scales_nothing(bad, dtype):
    from paper_2605_00686_amd import binding as B
    g = torch.ones(5000, dtype=dtype, device="cuda")
    g[4999] = bad
    out = torch.zeros_like(g)
    tensors = B.tensor_list([g], [out])
    total, norm = norm_of(B, tensors)
    assert not math.isfinite(float(total)) and not math.isfinite(float(norm))
    B.moe_grad_clip(tensors, total, 1.0)
    assert torch.equal(out[:4999], g[:4999]) and (math.isnan(bad) and math.isnan(float(out[4999])) or float(out[4999]) == bad)


def test_captured_and_on_another_stream_and_nothing_around_is_touched():
    from paper_2605_00686_amd import binding as B
    gen = torch.Generator().manual_seed(11)
    sizes = [(9, BF), (70000, BF), (1, F32), (33333, F32), (100, BF)]
    grads = draw(gen, sizes)
    # outputs as pieces of buffers with guards between them, at starts of their own
    guard = {dt: torch.full((sum(n + 5 for n, t in sizes if t == dt) + 7,), 77.0, dtype=dt, device="cuda") for dt in (BF, F32)}
    at, outs, spans = {BF: 3, F32: 2}, [], []
    for n, dt in sizes:
        outs.append(guard[dt][at[dt]:at[dt] + n])
        spans.append((dt, at[dt], at[dt] + n))
        at[dt] += n + 5
    tensors = B.tensor_list(grads, outs)
    total, norm = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1, device="cuda")
    ws = torch.empty(B.moe_grad_workspace_bytes(tensors), dtype=torch.uint8, device="cuda")

    def run():
        B.moe_grad_norm(tensors, total, norm, ws)
        B.moe_grad_clip(tensors, total, 2.0)
    run()
    want, wanted = [o.clone() for o in outs], float(total)
    for dt in guard:
        rest = torch.ones(guard[dt].numel(), dtype=torch.bool)
        for t, a, b in spans:
            if t == dt:
                rest[a:b] = False
        assert (guard[dt].cpu()[rest] == 77.0).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for o in outs:
            o.zero_()
        run()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want)) and float(total) == wanted
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        for o in outs:
            o.zero_()
        total.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)) and float(total) == wanted


def test_more_numbers_than_32_bits_count():
    from paper_2605_00686_amd import binding as B
    n = (1 << 31) + 12345
    g = torch.ones(n, dtype=BF, device="cuda")
    g[n - 1] = 3.0
    tensors = B.tensor_list([g])
    total, _ = norm_of(B, tensors)
    assert float(total) == n + 8
    B.moe_grad_clip(tensors, total, math.sqrt(n + 8) / 2)
    assert float(g[n - 1]) == 1.5 and float(g[0]) == 0.5 and float(g[n - 2]) == 0.5

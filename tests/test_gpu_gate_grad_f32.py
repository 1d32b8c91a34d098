"""GPU tests of dWg in fp32: a product is as good as fp32's, whatever the bits of its factors."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def mantissas(shape, kind, gen):
    """Numbers of 2^-3 to 2^4 with the bits that a cut into shorter numbers loses most of, or random ones; of one sign, or both."""
    if kind == "random":
        return torch.randn(shape, generator=gen)
    power = torch.exp2(torch.randint(-3, 4, shape, generator=gen).float())
    low = {"ones": 0x00ffff, "ones_behind_a_zero": 0x00ff7f, "halves": 0x008080}[kind]
    v = (torch.full(shape, 0x3f800000 | low, dtype=torch.int32) ^ torch.randint(0, 4, shape, generator=gen).to(torch.int32)).view(torch.float32)
    return power * v


# E: both shapes of a task, and two groups of experts; per: tokens that choose an expert
@pytest.mark.parametrize("E,d,per", [(8, 80, 1), (8, 128, 2), (64, 16, 1), (128, 144, 1), (128, 64, 2), (200, 80, 1), (256, 128, 2)])
@pytest.mark.parametrize("kind", ["ones", "ones_behind_a_zero", "halves", "random"])
def test_products_of_few_tokens(E, d, per, kind):
    from paper_2605_00686_amd import binding as B
    gen = torch.Generator().manual_seed(E + d + per)
    T = E * per
    p = B.problem(T, d, E, 1, 64, 1, "f32")
    x, dl = mantissas((T, d), kind, gen), mantissas((T, 1), kind, gen)
    idx = (torch.randperm(T, generator=gen) % E).to(torch.int32)[:, None].contiguous()
    # one choice with a weight of a half: dl = 1/2 (4 dl - 1/2 4 dl), without a rounding
    w, dw = torch.full((T, 1), 0.5), 4.0 * dl
    dWg = torch.empty((d, E), device="cuda")
    ws = torch.empty(max(256, B.moe_backward_workspace_bytes(p)), dtype=torch.uint8, device="cuda")
    B.moe_route_backward(p, x.cuda(), None, idx.cuda(), w.cuda(), dw.cuda(), None, dWg, None, None, ws)
    dense = torch.zeros(T, E, dtype=torch.float64).scatter_(1, idx.long(), dl.double())
    want, size = x.double().t() @ dense, x.double().abs().t() @ dense.abs()
    # a rounding of each product and of each sum, 2^-24 each, twice over
    assert bool(((dWg.cpu().double() - want).abs() <= 2 * (per + 1) * 2.0 ** -24 * size).all())


def test_numbers_at_the_end_of_the_range():
    # the largest numbers of fp32 lie past the largest of bf16
    from paper_2605_00686_amd import binding as B
    T = E = 4
    p = B.problem(T, 16, E, 1, 64, 1, "f32")
    bits = torch.tensor([0x7f7fffff, 0x7f7f8000, 0x7f7f7fff, 0x7f7f8001], dtype=torch.int32)
    x = bits.view(torch.float32)[:, None].repeat(1, 16) * torch.tensor([1.0, -1.0]).repeat(8)
    idx = torch.arange(T, dtype=torch.int32)[:, None].contiguous()
    dWg = torch.empty((16, E), device="cuda")
    ws = torch.empty(max(256, B.moe_backward_workspace_bytes(p)), dtype=torch.uint8, device="cuda")
    B.moe_route_backward(p, x.cuda(), None, idx.cuda(), torch.full((T, 1), 0.5).cuda(), torch.full((T, 1), 1.0).cuda(), None, dWg, None, None, ws)
    want = x.double().t() / 4
    assert bool(((dWg.cpu().double() - want).abs() <= 4 * 2.0 ** -24 * want.abs()).all())

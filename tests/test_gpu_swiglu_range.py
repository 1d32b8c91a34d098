"""GPU tests of moe_swiglu and moe_swiglu_backward over the whole range of their inputs: fp32 to a few units of its last place, and
no number that the definition keeps finite and not zero becomes anything else."""
import pytest
import torch

pytestmark = pytest.mark.gpu

# 1 / (1 + exp(-g)) in units of 2^-24 of itself: the exponential's argument to 2^-25 and the exponential to one place (both count 1 - s
# times: 2.5), the sum 1, the reciprocal one place (2)
def sigmoid_units(s):
    return 2.5 * (1 - s) + 3


def rows_of(values, f=64):
    n = -(-values.numel() // f)
    out = torch.zeros(n * f, dtype=values.dtype)
    out[:values.numel()] = values
    return out.reshape(n, f)


def forward(g, u, dtype):
    from paper_2605_00686_amd import binding as B
    n, f = g.shape
    p = B.problem(n, 64, 1, 1, f, 1, dtype)
    h = torch.full((n, f), 7.0, dtype=dtype, device="cuda")
    B.moe_swiglu(p, g.cuda(), u.cuda(), None, h, None, None)
    return h.cpu().double()


# powers of two that u multiplies silu with: h stays in the range
@pytest.mark.parametrize("power", [0, 40, 100])
def test_fp32_forward(power):
    gen = torch.Generator().manual_seed(power)
    g = rows_of(torch.cat([torch.linspace(-110.0, 110.0, 20_001), torch.randn(20_000, generator=gen), torch.tensor([-87.3, -87.4, -88.0, -88.7, -88.8, -92.0])]))
    u = torch.randn(g.shape, generator=gen) * 2.0 ** power
    got = forward(g, u, torch.float32)
    gd, ud = g.double(), u.double()
    s = torch.sigmoid(gd)
    want = gd * s * ud
    # two products more; below 2^-126 s and h are multiples of 2^-149
    bound = (sigmoid_units(s) + 2) * 2.0 ** -24 * 1.001 * want.abs() + 2.0 ** -149 * (1 + (gd * ud).abs())
    assert bool(((got - want).abs() <= bound).all())


def test_bf16_forward_keeps_small_numbers():
    g = rows_of(torch.cat([torch.linspace(-92.0, -60.0, 2000), torch.tensor([-87.5, -88.0, -88.5, -89.0, -90.0, -91.0])]).to(torch.bfloat16))
    for power in (0, 100):
        u = torch.full_like(g, 2.0 ** power)
        got = forward(g, u, torch.bfloat16)
        gd = g.double()
        want = gd * torch.sigmoid(gd) * 2.0 ** power
        # the rounding to bf16, a 64th of it for what comes before; s is a multiple of 2^-149 below 2^-126, h of 2^-133
        assert bool(((got - want).abs() <= 2.0 ** -8 * (1 + 2.0 ** -6) * want.abs() + 2.0 ** -149 * gd.abs() * 2.0 ** power + 2.0 ** -134).all())

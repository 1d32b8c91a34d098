"""GPU tests of moe_swiglu and moe_swiglu_backward over the whole range of their inputs: fp32 to a few units of its last place, and
no number that the definition keeps finite and not zero becomes anything else."""
import pytest
import torch

from tests.train_forms import decode

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


def backward(codes, scales, dh, dtype):
    from paper_2605_00686_amd import binding as B
    n, f = dh.shape
    p = B.problem(n, 64, 1, 1, f, 1, dtype)
    dg, du, h = (torch.full((n, f), 7.0, dtype=dtype, device="cuda") for _ in range(3))
    B.moe_swiglu_backward(p, dh.cuda(), codes.cuda(), scales.cuda(), None, dg, du, h)
    return [t.cpu().double() for t in (dg, du, h)]


def every_code(byte, f=64):
    """codes and scales of rows in which g takes every code but the NaNs, with blocks' exponents `byte` and one below, and u is one."""
    values = torch.tensor([c for c in range(256) if c & 127 != 127], dtype=torch.uint8)
    g = rows_of(values.repeat(2), f)
    codes = torch.stack([g, torch.full_like(g, 0x38)], 1).contiguous()
    scales = torch.full((g.shape[0], 2, f // 32), 127, dtype=torch.uint8)
    scales[:, 0, 0::2], scales[:, 0, 1::2] = byte, byte - 1
    return codes, scales


@pytest.mark.parametrize("byte", [127, 126, 125, 124, 122, 118])
def test_fp32_backward(byte):
    codes, scales = every_code(byte)
    gen = torch.Generator().manual_seed(byte)
    dh = torch.randn(codes.shape[0], 64, generator=gen)
    dg, du, h = backward(codes, scales, dh, torch.float32)
    g, u = decode(codes, scales)
    d, unit, low = dh.double(), 2.0 ** -24 * 1.001, 2.0 ** -149
    s = torch.sigmoid(g)
    silu, b = g * s, 1 + g * (1 - s)
    units = sigmoid_units(s)
    assert bool(((h - silu * u).abs() <= (units + 2) * unit * (silu * u).abs() + low * (1 + g.abs())).all())
    assert bool(((du - d * silu).abs() <= (units + 2) * unit * (d * silu).abs() + low * (1 + d.abs() * (1 + g.abs()))).all())
    # 1 - s is off by s's error and a rounding, the bracket by |g| times that and two roundings of its own; then three products
    off = s * (g.abs() * (s * units + 2 * (1 - s)) + b.abs() * (units + 5)) * unit
    assert bool(((dg - d * u * s * b).abs() <= (d * u).abs() * (off + low * (1 + g.abs())) + low).all())


# dh u past the range, dg within it: silu's slope is small there
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_large_gradients_of_closed_gates(dtype):
    codes, scales = every_code(125)
    codes[:, 0] |= 0x80  # g from -112 to 0
    scales[:, 0], scales[:, 1] = 125, 127 + 90
    g, u = decode(codes, scales)
    dh = torch.full(g.shape, 2.0 ** 60)
    keep = g < -60.0  # dh u = 2^150, the slope below 2^-80
    dg, du, h = backward(codes, scales, torch.where(keep, dh, 1.0).to(dtype), dtype)
    s = torch.sigmoid(g)
    want = dh.double() * u * s * (1 + g * (1 - s))
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -19  # (fp32: far more than its roundings come to)
    bound = half * (1 + 2.0 ** -6) * want.abs() + 2.0 ** 150 * 2.0 ** -149 * (1 + g.abs())
    assert bool(keep.any()) and bool(((dg - want).abs() <= bound)[keep].all())
    assert bool(torch.isfinite(dg).all()) and bool(torch.isfinite(du).all()) and bool(torch.isfinite(h).all())

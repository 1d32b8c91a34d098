"""Clipping by factors that fp32 has no, or no whole, number for, against 64 bits."""
import math

import pytest
import torch

from tests.test_gpu_grads import BF, F32, HALF_STEP, draw, norm_of

pytestmark = pytest.mark.gpu

SIZES = [(9, BF), (40000, BF), (1, F32), (3333, F32), (100, BF)]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("limit", [3e-2, 1e-3, 1e-5, 1e-7, 1e-20, 1e-36, 1e-40, 1e-44, 0.0])
def test_factors_below_the_normal_numbers(limit, in_place):
    """Gradients of 2^120 clipped to ordinary norms and to the smallest ones: bf16's and fp32's results have their type's one rounding."""
    from paper_2605_00686_amd import binding as B
    gen = torch.Generator().manual_seed(41)
    grads = draw(gen, SIZES, std=2.0 ** 120)
    before = [g.clone() for g in grads]
    outs = grads if in_place else [torch.full_like(g, float("nan")) for g in grads]
    tensors = B.tensor_list(grads, None if in_place else outs)
    total, norm = norm_of(B, tensors)
    B.moe_grad_clip(tensors, total, limit)
    most = torch.tensor(limit, dtype=F32).double().item()
    factor = most / math.sqrt(float(total))
    assert factor < 2.0 ** -126
    for g, o in zip(before, outs):
        ref = g.double() * factor
        # (fp32's rounding in front of bf16's is 2^-24; below the normal numbers a rounding is half a step of the smallest: 2^-134 of bf16, 2^-150 of fp32)
        off = HALF_STEP[g.dtype] * (1 + 2.0 ** -14) * ref.abs() + 2.0 ** (-133.9 if g.dtype == BF else -150)
        assert ((o.double() - ref).abs() <= off).all()
    if limit >= 1e-20:
        whole = math.sqrt(sum(float(o.double().square().sum()) for o in outs))
        assert abs(whole - most) <= 2.0 ** -8 * (1 + 2.0 ** -14) * most


def test_one_number_at_the_end_of_the_range():
    """The whole norm is one bf16 number's: it comes out as max_norm, rounded."""
    from paper_2605_00686_amd import binding as B
    for limit in (1e-5, 1e-7, 1.0):
        g = torch.tensor([3e38, 0.0, -0.0], dtype=BF, device="cuda")
        tensors = B.tensor_list([g])
        total, _ = norm_of(B, tensors)
        B.moe_grad_clip(tensors, total, limit)
        assert abs(float(g[0]) - limit) <= 2.0 ** -8 * limit * (1 + 2.0 ** -14) and float(g[1]) == 0 and float(g[2]) == 0

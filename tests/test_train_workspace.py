"""Host-only checks of what moe_route_backward asks for."""
import pytest

from paper_2605_00686_amd import binding as B


def ask(T, d, E, k, dtype="bf16"):
    return B.moe_backward_workspace_bytes(B.problem(T, d, E, k, 64, 1, dtype))


@pytest.mark.parametrize("case", [(2048, 7168, 256, 8), (1, 2048, 128, 8), (64, 512, 8, 2), (64, 4096, 256, 8, "f32")])
def test_tokens_in_one_part_need_no_sums(case):
    # their sums are the gradients: next to nothing, and not nothing, which says that the problem is invalid
    assert ask(*case) == 256


@pytest.mark.parametrize("case", [(4096, 2048, 128, 8), (9683, 720, 3, 3, "f32"), (16384, 64, 32, 4)])
def test_parts_have_sums_of_their_own(case):
    T, d, E, k = case[:4]
    parts = ask(*case) // (4 * ((d * E + E + 63) // 64 * 64))
    assert parts > 1 and ask(*case) == parts * 4 * ((d * E + E + 63) // 64 * 64)

"""Problems that pass the general checks and have more tiles than a launch of the experts' products counts; the workspace of long lists of gradients."""
import pytest

from paper_2605_00686_amd import binding as B
from tests.test_ffn_abi import down, down_backward, tensors, up, up_backward

CAPACITY, WIDE = 1 << 27, 1 << 16  # 8 experts' padded rows: 2^22 row blocks of 256 rows at least, of 2^8 columns of tiles
MATRIX = 1 << 19                   # 2^22 tiles of 256 x 256 for each of 256 experts


@pytest.mark.parametrize("call,problem,other", [
    (up, dict(f=WIDE), dict(ld=WIDE, ldw=WIDE)),
    (up, dict(f=WIDE), dict(g=None, u=None, ldw=WIDE)),
    (down, dict(d=WIDE), {}),
    (down_backward, dict(f=WIDE), dict(ld=WIDE, dW2=None)),
    (down_backward, dict(f=WIDE), dict(ld=WIDE, dg=None, du=None, dW2=None)),
    (down_backward, dict(k=1, E=256, capacity=0, d=MATRIX, f=MATRIX), dict(dh=None, dg=None, du=None)),
    (up_backward, dict(d=WIDE), dict(ld=64, ldw=64, dW1=None, dW3=None)),
    (up_backward, dict(k=1, E=256, capacity=0, d=MATRIX, f=MATRIX), dict(ld=MATRIX, ldw=MATRIX, dx=None)),
    (up_backward, dict(k=1, E=256, capacity=0, d=MATRIX, f=2 * MATRIX), dict(ld=2 * MATRIX, ldw=2 * MATRIX, dx=None, dW3=None)),
], ids=lambda v: "_".join(f"{n}{x}" for n, x in v.items()) if isinstance(v, dict) else None)
def test_too_many_tiles(call, problem, other):
    p = B.problem(**{**dict(T=1, d=64, E=8, k=8, f=64, R=1, dtype="bf16", capacity=CAPACITY), **problem})
    assert B.moe_ffn_workspace_bytes(p) > 0
    assert call(p, **other) == B.MOE_ERR_UNSUPPORTED


def test_a_long_list_takes_as_many_sums_as_workgroups():
    t, n = tensors(*[(0x10000, 0x20000, 1 << 30, 1)] * 200)  # 140 and 60 of 65536 chunks: 4096 workgroups each
    assert B._lib.moe_grad_workspace_bytes(t, n) == 2 * 4096 * 8

"""What the experts' products ask for as workspace, on the host: enough for the largest batch is enough for a smaller one; a shorter one is refused."""
import itertools

import pytest
import torch

from paper_2605_00686_amd import binding as B

TOKENS = [1, 2, 3, 7, 16, 33, 64, 100, 128, 256, 500, 512, 1000, 1024, 2048, 4096, 10000, 16384, 65536, 1 << 20]
LAYERS = [(512, 8, 2, 1024, "f32"), (4096, 8, 2, 14336, "bf16"), (2048, 128, 8, 768, "bf16"), (64, 2, 1, 14336, "bf16"), (1040, 48, 6, 368, "f32"),
          (64, 1, 1, 64, "bf16"), (16, 2, 2, 16, "f32"), (7168, 256, 8, 2048, "bf16"), (2112, 3, 3, 64, "bf16"), (256, 2, 1, 256, "bf16")]


def ask(T, d, E, k, f, dtype, capacity=0):
    n = B.moe_ffn_workspace_bytes(B.problem(T, d, E, k, f, 1, dtype, capacity=capacity))
    assert n >= 256 and n % 256 == 0
    return n


@pytest.mark.parametrize("layer", LAYERS)
def test_fewer_rows_need_no_more(layer):
    d, E, k, f, dtype = layer
    sizes = [ask(T, *layer) for T in TOKENS]
    assert sizes == sorted(sizes), sizes
    for T in TOKENS:
        by_choices = [ask(T, d, E, j, f, dtype) for j in range(1, k + 1)]
        assert by_choices == sorted(by_choices)
    if E * TOKENS[-1] <= 1 << 30:
        for T, C in itertools.product(TOKENS, TOKENS):
            assert ask(T, *layer, capacity=C) <= ask(TOKENS[-1], *layer, capacity=TOKENS[-1])
        for T in (1, 100, 4096):
            by_capacity = [ask(T, *layer, capacity=C) for C in TOKENS]
            assert by_capacity == sorted(by_capacity)


def test_no_more_than_the_sums_of_two_products():
    assert max(ask(T, *layer) for layer in LAYERS for T in TOKENS) <= (2 << 25) + (1 << 16)


class Buffer:  # a device tensor as far as the binding looks at a workspace
    is_cuda = True

    def __init__(self, nbytes):
        self.nbytes = nbytes

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x10000


def test_a_workspace_that_is_too_short_is_refused(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    p = B.problem(256, 512, 8, 2, 1024, 1, "f32")
    need = B.moe_ffn_workspace_bytes(p)
    assert B._ffn_workspace(p, Buffer(need)) == 0x10000 and B._ffn_workspace(p, None) is None
    short = Buffer(need - 1)
    short.get_device = lambda: 0
    for call, others in ((B.moe_ffn_up, 7), (B.moe_ffn_down, 4), (B.moe_ffn_down_backward, 10), (B.moe_ffn_up_backward, 9)):
        with pytest.raises(AssertionError, match="workspace"):
            call(p, *[None] * others, short, object())


def test_a_workspace_of_the_norm_that_is_too_short_is_refused(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    tensors = B.tensor_list([])
    assert B.moe_grad_workspace_bytes(tensors) == 256
    short = Buffer(255)
    short.get_device = lambda: 0
    with pytest.raises(AssertionError, match="workspace"):
        B.moe_grad_norm(tensors, None, None, short, object())

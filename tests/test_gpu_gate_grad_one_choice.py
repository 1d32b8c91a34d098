"""GPU tests of moe_route_backward with one choice per token, whose weight is taken as given: a weight of one has no gradient."""
import pytest
import torch

from tests.test_gpu_gate_grad import call, check, expected, make

pytestmark = pytest.mark.gpu


# up to 64 experts, up to 128 and two groups, with the tokens in one part and in several
@pytest.mark.parametrize("case", [(5000, 64, 64, 1, "bf16"), (1300, 256, 200, 1, "f32"), (4000, 192, 33, 1, "bf16"), (6000, 128, 130, 1, "bf16"),
                                  (3000, 64, 8, 1, "f32"), (700, 1040, 100, 1, "f32"), (100, 7168, 256, 1, "bf16")],
                         ids=lambda c: "T%d_d%d_E%d_k%d_%s" % c)
def test_one_choice_with_a_weight(case):
    print(f"case one choice {case}", flush=True)
    B, p, gen, dt, idx, w, dw, x, Wg = make(*case)
    w = torch.rand(w.shape, generator=gen)
    want = expected(idx, w, dw, x, Wg, dt)
    assert all(float(ref.abs().max()) > 0.0 for ref, _ in want)
    got = call(B, p, x, Wg, idx, w, dw)
    check(got, want)
    for i, one in enumerate("xwb"):
        assert torch.equal(call(B, p, x, Wg, idx, w, dw, one)[i], got[i]), one

"""Gradients of the experts' weights over more than 2^29 rows."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_weight_gradients_of_more_than_2_29_rows():
    """Zeros but for 4096 rows of small whole numbers, the first and last of every expert among them: sums that every order has exactly."""
    from paper_2605_00686_amd import binding as B
    T, d, f = (1 << 29) + 10 ** 6, 16, 16
    counts = [1000, T - 4000, 3000]
    p = B.problem(T, d, 3, 1, f, 1, torch.float32)
    gen = torch.Generator(device="cuda").manual_seed(31)
    ends = torch.tensor(counts).cumsum(0)
    at = torch.cat([torch.tensor([0, 999, 1000, T - 3001, T - 3000, T - 1]), torch.randint(0, T, (4090,), generator=torch.Generator().manual_seed(32))]).unique()
    h, dy = torch.zeros(T, f, device="cuda"), torch.zeros(T, d, device="cuda")
    few = [torch.randint(-4, 5, (len(at), 16), generator=gen, device="cuda").float() for _ in range(2)]
    h[at.cuda()], dy[at.cuda()] = few[0], few[1]
    dW2 = torch.full((3, f, d), float("nan"), device="cuda")
    ws = torch.empty(B.moe_ffn_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    B.moe_ffn_down_backward(p, dy, None, h, None, None, torch.tensor(counts, dtype=torch.int32).cuda(), None, None, None, dW2, ws)
    expert = torch.bucketize(at, ends, right=True)
    for e in range(3):
        i = (expert == e).nonzero()[:, 0].cuda()
        want = few[0][i].double().t() @ few[1][i].double()
        assert i.numel() >= 2 and torch.equal(dW2[e].double(), want), e

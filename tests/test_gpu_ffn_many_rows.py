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


# (E, k, d, f, capacity, dtype), tokens of the smaller batches: reductions that only they cut
@pytest.mark.parametrize("layer", [(8, 2, 512, 1024, 0, "f32"), (4, 1, 2048, 1088, 0, "bf16"), (5, 3, 144, 2144, 300, "f32"), (40, 2, 960, 192, 0, "bf16")])
def test_the_largest_batch_s_workspace(layer):
    """Smaller batches in the workspace of 4096 tokens: the results that they have with their own, and nothing behind it is touched."""
    from paper_2605_00686_amd import binding as B
    from tests import ffn_forms as F
    E, k, d, f, capacity, dtype = layer
    most = F.Rows(torch.Generator().manual_seed(33), 4096, E, k, d, f, capacity, dtype)
    need = B.moe_ffn_workspace_bytes(most.problem())
    guard = 80 << 20
    shared = torch.full((need + guard,), 171, dtype=torch.uint8, device="cuda")
    for T in (1, 2, 17, 64, 256, 1000, 4096):
        gen = torch.Generator().manual_seed(34)
        r = F.Rows(gen, T, E, k, d, f, capacity, dtype)
        x, dy, gu = r.draw(gen, d).cuda(), r.draw(gen, d).cuda(), r.draw(gen, 2 * f).cuda()
        W1, W3, W2 = r.weights(gen, d, f).cuda(), r.weights(gen, d, f).cuda(), r.weights(gen, f, d).cuda()
        p, n, g, u = r.problem(), r.counts.cuda(), gu[:, :f], gu[:, f:]

        def calls(ws):
            h, y, dgu, dW2, dx, dW1, dW3 = (torch.full(s, float("nan"), dtype=r.dt, device="cuda")
                                            for s in ((r.n, f), (r.n, d), (r.n, 2 * f), W2.shape, (r.n, d), W1.shape, W1.shape))
            B.moe_ffn_up(p, x, W1, W3, n, None, None, h, ws)
            B.moe_ffn_down(p, h, W2, n, y, ws)
            B.moe_ffn_down_backward(p, dy, W2, h, g, u, n, None, dgu[:, :f], dgu[:, f:], dW2, ws)
            B.moe_ffn_up_backward(p, x, W1, W3, g, u, n, dx, dW1, dW3, ws)
            return h, y, dgu, dW2, dx, dW1, dW3
        own = calls(torch.empty(B.moe_ffn_workspace_bytes(p), dtype=torch.uint8, device="cuda"))
        assert all(torch.equal(a, b) for a, b in zip(own, calls(shared[:need]))), T
        assert (shared[need:] == 171).all(), T

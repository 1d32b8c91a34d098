"""The training example: its gradients against autograd in 64 bits, and that it learns."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def reference(layer, x, dout):
    """Gradients of the layer in 64 bits on the CPU, with the layer's own routing."""
    par = [t.detach().cpu().double().requires_grad_() for t in (x, layer.Wg, layer.bias, layer.W13, layer.W2)]
    xx, Wg, bias, W13, W2 = par
    idx = layer.idx.cpu().long()
    w = torch.softmax(torch.gather(xx @ Wg + bias, 1, idx), 1)
    out = xx.clone()
    for e in range(layer.E):
        t, j = (idx == e).nonzero(as_tuple=True)
        if t.numel():
            gu = xx[t] @ W13[e]
            y = (torch.nn.functional.silu(gu[:, :layer.f]) * gu[:, layer.f:]) @ W2[e]
            out = out.index_add(0, t, w[t, j, None] * y)
    out.backward(dout.cpu().double())
    return out.detach(), [p.grad for p in par]


def off(got, ref):
    return float((got.cpu().double() - ref).norm() / ref.norm())


def test_gradients_of_the_layer():
    from examples.train_layer import Layer
    layer = Layer(200, 96, 12, 3, 80, torch.float32, seed=3)
    gen = torch.Generator().manual_seed(4)
    x, dout = torch.randn(200, 96, generator=gen).cuda(), torch.randn(200, 96, generator=gen).cuda()
    out = layer.forward(x).clone()
    dx = layer.backward(dout)
    layer.check()
    ref_out, (rx, rWg, rb, rW13, rW2) = reference(layer, x, dout)
    # fp32 sums of up to 96 and 80 terms in a row; the gate's gradient has no 8-bit numbers in it
    assert off(out, ref_out) <= 1e-5
    assert off(layer.dWg, rWg) <= 1e-4 and off(layer.dbias, rb) <= 1e-4
    # g and u are kept to 2^-4 each at worst; h and the gradients of g and u are products of a function of either, whose relative
    # slopes are about one for g of order one: 2 * 2^-4, and an eighth more for what is beyond first order
    for got, ref in ((dx, rx), (layer.dW13, rW13), (layer.dW2, rW2)):
        assert off(got, ref) <= 2 * 2.0 ** -4 * 1.125


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_layer_learns(dtype):
    from examples.train_layer import train
    losses = train(T=512, d=128, E=8, k=2, f=256, dtype=dtype, steps=60)
    assert all(v == v for v in losses)
    assert sum(losses[-5:]) < 0.9 * sum(losses[:5])

"""The training example with this package's products: its gradients against autograd in 64 bits, clipped ones, and that its step can be captured."""
import pytest
import torch

from tests.test_gpu_train_layer import off, reference

pytestmark = pytest.mark.gpu


def make(dtype, T=200, d=128, E=12, k=3, f=192):
    from examples.train_layer import Layer
    layer = Layer(T, d, E, k, f, dtype, seed=5, products="own")
    gen = torch.Generator().manual_seed(6)
    return layer, torch.randn(T, d, generator=gen).to(dtype).cuda(), torch.randn(T, d, generator=gen).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_of_the_layer(dtype):
    layer, x, dout = make(dtype)
    out = layer.forward(x).clone()
    dx = layer.backward(dout).clone()
    layer.check()
    ref_out, (rx, rWg, rb, rW13, rW2) = reference(layer, x, dout)
    # fp32: 4 products in a chain of up to 384 steps, each off by (K + 1) 2^-23 of the sum of the magnitudes, which random terms hold to sqrt(K) times
    # the sum: 4 * 385 * 20 * 2^-23.  bf16: up to 9 roundings behind an output, 2^-8 / sqrt(3) of a tensor's norm each and evenly spread: their squares
    # add up to 6.8e-3; twice that, for what the slopes of the activation and of the softmax make of them.
    rest = 3.7e-3 if dtype == torch.float32 else 1.36e-2
    for got, ref in ((out, ref_out), (dx, rx), (layer.dWg, rWg), (layer.dbias, rb), (layer.dW13, rW13), (layer.dW2, rW2)):
        assert off(got, ref) <= rest
    grads = [layer.dWg, layer.dbias, layer.dW13, layer.dW2]
    before = [g.clone() for g in grads]
    whole = float(torch.cat([g.double().flatten() for g in grads]).norm())
    layer.clip(2 * whole)
    assert all(torch.equal(a, b) for a, b in zip(grads, before))
    layer.clip(whole / 4)
    assert abs(float(layer.norm) - whole) <= 2.0 ** -22 * whole
    for a, b in zip(grads, before):  # (half a step, and half a one of fp32 for max_norm)
        assert ((a.double() - b.double() / 4).abs() <= (b.double() / 4).abs() * torch.finfo(a.dtype).eps * 1.01 + 2.0 ** -133).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_step_captured_and_replayed(dtype):
    layer, x, dout = make(dtype)

    def step():
        layer.forward(x)
        layer.backward(dout)
        layer.clip(0.5)
    outputs = lambda: [layer.out, layer.dx, layer.dWg, layer.dbias, layer.dW13, layer.dW2, layer.norm]
    step()
    want = [t.clone() for t in outputs()]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in outputs():
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outputs(), want))
    layer.check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_example_runs(dtype):
    from examples.train_layer import train
    losses = train(T=256, d=64, E=8, k=2, f=128, dtype=dtype, steps=4, products="own", clip=0.01)
    assert len(losses) == 4 and all(v == v for v in losses)

"""Tensors of other types or sizes than the experts' products and the norm take are refused by the binding: the C calls see addresses only."""
import pytest
import torch

from paper_2605_00686_amd import binding as B

T, E, k, d, f = 6, 4, 2, 64, 128
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def host_tensors(monkeypatch):
    """Tensors of this host pass for the current device's, up to where addresses are taken."""
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)


def tensors(rows, dt):
    e = lambda *shape, dtype=dt: torch.empty(shape, dtype=dtype)
    return {"up": dict(x_perm=e(rows, d), W1=e(E, d, f), W3=e(E, d, f), counts=e(E, dtype=torch.int32), g=e(rows, f), u=e(rows, f), h=e(rows, f)),
            "down": dict(h=e(rows, f), W2=e(E, f, d), counts=e(E, dtype=torch.int32), y=e(rows, d)),
            "down_backward": dict(dy=e(rows, d), W2=e(E, f, d), h=e(rows, f), g=e(rows, f), u=e(rows, f), counts=e(E, dtype=torch.int32), dh=e(rows, f),
                                  dg=e(rows, f), du=e(rows, f), dW2=e(E, f, d)),
            "up_backward": dict(x_perm=e(rows, d), W1=e(E, d, f), W3=e(E, d, f), dg=e(rows, f), du=e(rows, f), counts=e(E, dtype=torch.int32),
                                dx=e(rows, d), dW1=e(E, d, f), dW3=e(E, d, f))}


CALLS = {"up": B.moe_ffn_up, "down": B.moe_ffn_down, "down_backward": B.moe_ffn_down_backward, "up_backward": B.moe_ffn_up_backward}


def call(name, capacity=0, dt=BF, **other):
    given = {**tensors(E * capacity if capacity else T * k, dt)[name], **other}
    ws = torch.empty(1 << 20, dtype=torch.uint8)
    CALLS[name](B.problem(T, d, E, k, f, 1, dt, capacity=capacity), *given.values(), ws, object())


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("capacity", [0, 5])
@pytest.mark.parametrize("dt", [BF, F32])
def test_types_and_sizes(name, capacity, dt):
    rows = E * capacity if capacity else T * k
    good = tensors(rows, dt)[name]
    with pytest.raises(AssertionError, match="device tensors"):  # (nothing but where they lie is wrong)
        call(name, capacity, dt)
    for which, t in good.items():
        if which == "counts":
            for bad in (t.long(), t[:-1]):
                with pytest.raises(AssertionError, match="counts: int32"):
                    call(name, capacity, dt, counts=bad)
            continue
        for bad in (t.to(F32 if dt == BF else BF), t.to(torch.float16), t[:-1]):
            with pytest.raises(AssertionError, match="type and size"):
                call(name, capacity, dt, **{which: bad})


@pytest.mark.parametrize("name", ["up", "down_backward", "up_backward"])
def test_views_of_other_widths(name):
    good = tensors(T * k, BF)[name]
    for which, t in good.items():
        if which in ("g", "u", "dg", "du"):
            bad = torch.empty(4 * t.shape[0], 4 * f, dtype=BF)[:, :f // 2]
        elif which in ("W1", "W3", "dW1", "dW3"):
            bad = torch.empty(E, f, d, dtype=BF)
        else:
            continue
        with pytest.raises(AssertionError, match="type and size"):
            call(name, **{which: bad})


@pytest.mark.parametrize("name", CALLS)
def test_longer_ones_are_taken(name):
    """What a program keeps for its largest batch."""
    longer = tensors(T * k + 9, BF)[name]
    longer["counts"] = torch.empty(E + 3, dtype=torch.int32)
    with pytest.raises(AssertionError, match="device tensors"):
        call(name, **longer)


def test_the_norm():
    some, total, norm, ws = B.tensor_list([]), torch.empty(1, dtype=torch.float64), torch.empty(1), torch.empty(256, dtype=torch.uint8)
    for t, n in ((total.float(), norm), (total[:0], norm), (total, norm.double()), (total, norm[:0])):
        with pytest.raises(AssertionError, match="float"):
            B.moe_grad_norm(some, t, n, ws, object())
    for t in (total.float(), total.long(), total[:0]):
        with pytest.raises(AssertionError, match="float64"):
            B.moe_grad_clip(some, t, 1.0, object())

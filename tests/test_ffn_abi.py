"""Host-only checks of the experts' products and of clipping: what is refused before anything is launched."""
import ctypes

import pytest
import torch

from paper_2605_00686_amd import binding as B

A = ctypes.c_void_p(0x10000)  # never followed: every call here is refused
ODD = ctypes.c_void_p(0x10008)


def problem(**kw):
    base = dict(T=256, d=512, E=8, k=2, f=1024, R=2, dtype="bf16")
    base.update(kw)
    return B.problem(**base)


def caller(function, **defaults):
    def call(p, **kw):
        return function(ctypes.byref(p), *{**defaults, **kw}.values(), None)
    return call


up = caller(B._lib.moe_ffn_up, x=A, W1=A, W3=A, ldw=1024, counts=A, g=A, u=A, ld=1024, h=A, ws=A)
down = caller(B._lib.moe_ffn_down, h=A, W2=A, counts=A, y=A, ws=A)
down_backward = caller(B._lib.moe_ffn_down_backward, dy=A, W2=A, h=A, g=A, u=A, counts=A, dh=A, dg=A, du=A, ld=1024, dW2=A, ws=A)
up_backward = caller(B._lib.moe_ffn_up_backward, x=A, W1=A, W3=A, ldw=1024, dg=A, du=A, ld=1024, counts=A, dx=A, dW1=A, dW3=A, ws=A)
CALLS = [up, down, down_backward, up_backward]


@pytest.mark.parametrize("call", CALLS)
def test_bad_problems(call):
    assert call(problem(k=9)) == B.MOE_ERR_INVALID_ARG
    assert call(problem(T=0)) == B.MOE_ERR_INVALID_ARG
    assert call(problem(d=100)) == B.MOE_ERR_UNSUPPORTED
    assert call(problem(f=8, dtype="f32")) == B.MOE_ERR_UNSUPPORTED
    assert call(problem(E=300)) == B.MOE_ERR_UNSUPPORTED


@pytest.mark.parametrize("call,kw", [
    (up, dict(x=None)), (up, dict(W1=None)), (up, dict(W3=None)), (up, dict(counts=None)), (up, dict(g=None)), (up, dict(u=None)),
    (up, dict(g=None, u=None, h=None)), (up, dict(ldw=1016)), (up, dict(ldw=1028)), (up, dict(ld=1016)), (up, dict(ld=1028)),
    *((up, {n: ODD}) for n in ("x", "W1", "W3", "g", "u", "h")),
    (down, dict(h=None)), (down, dict(W2=None)), (down, dict(counts=None)), (down, dict(y=None)), *((down, {n: ODD}) for n in ("h", "W2", "y")),
    (down_backward, dict(dy=None)), (down_backward, dict(counts=None)), (down_backward, dict(dg=None)), (down_backward, dict(du=None)),
    (down_backward, dict(dh=None, dg=None, du=None, dW2=None)), (down_backward, dict(W2=None)), (down_backward, dict(g=None)),
    (down_backward, dict(u=None)), (down_backward, dict(h=None)), (down_backward, dict(ld=0)), (down_backward, dict(ld=1028)),
    *((down_backward, {n: ODD}) for n in ("dy", "W2", "h", "g", "u", "dh", "dg", "du", "dW2")),
    (up_backward, dict(counts=None)), (up_backward, dict(dx=None, dW1=None, dW3=None)), (up_backward, dict(W1=None)), (up_backward, dict(W3=None)),
    (up_backward, dict(dg=None)), (up_backward, dict(du=None)), (up_backward, dict(x=None)), (up_backward, dict(ld=1016)), (up_backward, dict(ldw=1028)),
    *((up_backward, {n: ODD}) for n in ("x", "W1", "W3", "dg", "du", "dx", "dW1", "dW3"))])
def test_bad_pointers_and_strides(call, kw):
    assert call(problem(), **kw) == B.MOE_ERR_INVALID_ARG


@pytest.mark.parametrize("call", CALLS)
def test_workspace(call):
    p = problem()
    assert B.moe_ffn_workspace_bytes(p) >= 256 and B.moe_ffn_workspace_bytes(p) % 256 == 0
    assert B.moe_ffn_workspace_bytes(problem(k=9)) == 0
    assert call(p, ws=None) == B.MOE_ERR_WORKSPACE
    assert call(p, ws=ODD) == B.MOE_ERR_WORKSPACE


@pytest.mark.parametrize("call", CALLS)
def test_a_grid_that_cannot_be_launched(call):
    assert call(problem(T=1 << 25, k=8, f=1 << 24, d=1 << 24, R=1), ld=1 << 24, ldw=1 << 24) == B.MOE_ERR_UNSUPPORTED if call in (up, up_backward) else True


class Rows:  # a device tensor as far as the binding looks
    is_cuda = True

    def __init__(self, shape, strides):
        self.shape, self._s = shape, strides

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        return self._s if i is None else self._s[i]

    def data_ptr(self):
        return 0x10000


def test_views_that_are_not_alike_are_refused():
    ok = Rows((4, 64), (128, 1))
    assert B._like_rows(ok, None, ok) == [128, 0x10000, None, 0x10000]
    assert B._like_rows(None, None) == [0, None, None]
    for bad in (Rows((4, 64), (64, 1)), Rows((4, 64), (128, 4)), Rows((4, 32), (128, 1))):
        with pytest.raises(AssertionError):
            B._like_rows(ok, bad)
    whole, half = Rows((3, 4, 64), (256, 64, 1)), Rows((3, 4, 64), (512, 128, 1))
    assert B._like_matrices(whole, None) == [64, 0x10000, None] and B._like_matrices(None, half) == [128, None, 0x10000]
    for bad in (Rows((3, 4, 64), (512, 64, 1)), Rows((3, 4, 64), (256, 64, 2)), half):
        with pytest.raises(AssertionError):
            B._like_matrices(whole, bad)


def tensors(*given):
    return (B.MoeTensor * max(1, len(given)))(*(B.MoeTensor(*t, 0) for t in given)), len(given)


def norm(t, n, total=A, out=A, ws=A):
    return B._lib.moe_grad_norm(t, n, total, out, ws, None)


def clip(t, n, total=A, most=1.0):
    return B._lib.moe_grad_clip(t, n, total, most, None)


GOOD = (0x10000, 0x20000, 5, B.MOE_DT_F32)


@pytest.mark.parametrize("bad", [(None, 0x20000, 5, 0), (0x10002, 0x20000, 5, 0), (0x10001, 0x20000, 5, 1), (0x10000, 0x20000, -1, 0),
                                 (0x10000, 0x20000, 5, 2)])
def test_bad_tensors(bad):
    t, n = tensors(GOOD, bad)
    assert norm(t, n) == clip(t, n) == B.MOE_ERR_INVALID_ARG
    assert B._lib.moe_grad_workspace_bytes(t, n) == 0


def test_bad_calls_of_the_norm_and_of_clipping():
    t, n = tensors(GOOD)
    assert norm(t, -1) == clip(t, -1) == norm(None, 1) == clip(None, 1) == B.MOE_ERR_INVALID_ARG
    assert norm(t, n, total=None) == norm(t, n, total=ctypes.c_void_p(0x10004)) == B.MOE_ERR_INVALID_ARG
    assert clip(t, n, total=None) == clip(t, n, total=ctypes.c_void_p(0x10004)) == B.MOE_ERR_INVALID_ARG
    assert clip(t, n, most=-1.0) == clip(t, n, most=float("nan")) == B.MOE_ERR_INVALID_ARG
    assert norm(t, n, ws=None) == norm(t, n, ws=ODD) == B.MOE_ERR_WORKSPACE
    for bad in ((0x10000, None, 5, 0), (0x10000, 0x20002, 5, 0), (0x10000, 0x20001, 5, 1)):
        t, n = tensors(bad)
        assert clip(t, n) == B.MOE_ERR_INVALID_ARG
    t, n = tensors((0x10000, 0x20000, 1 << 44, 0))
    assert norm(t, n) == clip(t, n) == B.MOE_ERR_UNSUPPORTED


def test_workspace_of_the_norm():
    assert B._lib.moe_grad_workspace_bytes(None, 0) == 256
    t, n = tensors((None, None, 0, 0))
    assert B._lib.moe_grad_workspace_bytes(t, n) == 256
    t, n = tensors(*[(0x10000, 0x20000, 1 << 30, 1)] * 200)
    assert B._lib.moe_grad_workspace_bytes(t, n) >= 3 * 2048 * 8


class Numbers:  # a device tensor as far as a list of tensors looks
    is_cuda, dtype, device = True, torch.float32, "cuda:0"

    def __init__(self, at, n, where=0):
        self.at, self.n, self.where = at, n, where

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.at

    def numel(self):
        return self.n

    def element_size(self):
        return 4

    def get_device(self):
        return self.where


def test_lists_of_tensors_that_overlap_or_lie_on_two_devices_are_refused():
    a, b, empty = Numbers(0x1000, 64), Numbers(0x1100, 64), Numbers(0x1010, 0)
    assert B.tensor_list([a, b, empty]).n == 3 and B.tensor_list([a], [b]).n == 1 and B.tensor_list([]).n == 0
    for ins, outs in (([a, a], None), ([a, Numbers(0x10fc, 4)], None), ([a], [Numbers(0x1004, 64)]), ([a, b], [b, Numbers(0x2000, 64)]),
                      ([a, Numbers(0x9000, 4, where=1)], None)):
        with pytest.raises(AssertionError):
            B.tensor_list(ins, outs)


def test_tensors_of_another_device_are_refused(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
    here, there = Numbers(0x1000, 64, where=1), Numbers(0x1000, 64)
    B._here(here, None, here)
    with pytest.raises(AssertionError):
        B._here(here, None, there)
    for call in (lambda: B.moe_ffn_down(problem(), there, here, here, here, here), lambda: B.moe_grad_norm(B.tensor_list([there]), here, here, here),
                 lambda: B.moe_grad_clip(B.tensor_list([there]), here, 1.0), lambda: B.moe_grad_clip(B.tensor_list([here]), there, 1.0)):
        with pytest.raises(AssertionError):
            call()

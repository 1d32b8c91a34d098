"""Host-only checks of the training calls: what they refuse before anything is launched."""
import ctypes

import pytest

from paper_2605_00686_amd import binding as B

A = ctypes.c_void_p(0x10000)  # never followed: every call here is refused
ODD = ctypes.c_void_p(0x10008)
PADDED = dict(capacity=64)


def problem(**kw):
    base = dict(T=256, d=512, E=8, k=2, f=1024, R=2, dtype="bf16")
    base.update(kw)
    return B.problem(**base)


def unsort(p, **kw):
    a = {**dict(rows=A, inv=A, w=A, addend=A, out=A, status=None), **kw}
    return B._lib.moe_unsort(ctypes.byref(p), *(a[n] for n in ("rows", "inv", "w", "addend", "out", "status")), None)


def unsort_backward(p, **kw):
    a = {**dict(dout=A, rows=A, inv=A, w=A, counts=A, drows=A, dw=A, status=None), **kw}
    return B._lib.moe_unsort_backward(ctypes.byref(p), *(a[n] for n in ("dout", "rows", "inv", "w", "counts", "drows", "dw", "status")), None)


def route_backward(p, **kw):
    a = {**dict(x=A, Wg=A, idx=A, w=A, dw=A, dx=A, dWg=A, db=A, status=None, ws=A), **kw}
    return B._lib.moe_route_backward(ctypes.byref(p), *(a[n] for n in ("x", "Wg", "idx", "w", "dw", "dx", "dWg", "db", "status", "ws")), None)


def swiglu(p, **kw):
    a = {**dict(g=A, u=A, ld=1024, counts=A, h=A, codes=A, scales=A), **kw}
    return B._lib.moe_swiglu(ctypes.byref(p), *(a[n] for n in ("g", "u", "ld", "counts", "h", "codes", "scales")), None)


def swiglu_backward(p, **kw):
    a = {**dict(dh=A, codes=A, scales=A, counts=A, dg=A, du=A, ld=1024, h=A), **kw}
    return B._lib.moe_swiglu_backward(ctypes.byref(p), *(a[n] for n in ("dh", "codes", "scales", "counts", "dg", "du", "ld", "h")), None)


CALLS = [unsort, unsort_backward, route_backward, swiglu, swiglu_backward]


@pytest.mark.parametrize("call", CALLS)
def test_bad_problems(call):
    assert call(problem(k=9)) == B.MOE_ERR_INVALID_ARG
    assert call(problem(T=0)) == B.MOE_ERR_INVALID_ARG
    assert call(problem(d=100)) == B.MOE_ERR_UNSUPPORTED
    assert call(problem(f=8, dtype="f32")) == B.MOE_ERR_UNSUPPORTED
    assert call(problem(E=300)) == B.MOE_ERR_UNSUPPORTED


@pytest.mark.parametrize("call,kw", [
    (unsort, dict(rows=None)), (unsort, dict(inv=None)), (unsort, dict(out=None)), (unsort, dict(rows=ODD)), (unsort, dict(addend=ODD)),
    (unsort, dict(out=ODD)),
    (unsort_backward, dict(dout=None)), (unsort_backward, dict(inv=None)), (unsort_backward, dict(drows=None, dw=None)),
    (unsort_backward, dict(rows=None)), (unsort_backward, dict(dout=ODD)), (unsort_backward, dict(rows=ODD)), (unsort_backward, dict(drows=ODD)),
    (route_backward, dict(idx=None)), (route_backward, dict(w=None)), (route_backward, dict(dw=None)), (route_backward, dict(Wg=None)),
    (route_backward, dict(x=None)), (route_backward, dict(dx=None, dWg=None, db=None)), (route_backward, dict(x=ODD)),
    (route_backward, dict(Wg=ODD)), (route_backward, dict(dx=ODD)), (route_backward, dict(dWg=ODD)),
    (swiglu, dict(g=None)), (swiglu, dict(u=None)), (swiglu, dict(h=None, codes=None, scales=None)), (swiglu, dict(codes=None)),
    (swiglu, dict(scales=None)), (swiglu, dict(ld=1016)), (swiglu, dict(ld=1028)), (swiglu, dict(ld=-1024)), (swiglu, dict(g=ODD)),
    (swiglu, dict(u=ODD)), (swiglu, dict(h=ODD)), (swiglu, dict(codes=ODD)),
    (swiglu_backward, dict(dh=None)), (swiglu_backward, dict(codes=None)), (swiglu_backward, dict(scales=None)), (swiglu_backward, dict(dg=None)),
    (swiglu_backward, dict(du=None)), (swiglu_backward, dict(ld=0)), (swiglu_backward, dict(ld=1028)), (swiglu_backward, dict(dh=ODD)),
    (swiglu_backward, dict(dg=ODD)), (swiglu_backward, dict(du=ODD)), (swiglu_backward, dict(h=ODD)), (swiglu_backward, dict(codes=ODD))])
def test_bad_pointers_and_strides(call, kw):
    assert call(problem(), **kw) == B.MOE_ERR_INVALID_ARG


@pytest.mark.parametrize("call", [unsort_backward, swiglu, swiglu_backward])
def test_padded_rows_need_counts(call):
    assert call(problem(**PADDED), counts=None) == B.MOE_ERR_INVALID_ARG


def test_workspace_of_the_gate_gradient():
    p = problem()
    assert B.moe_backward_workspace_bytes(p) > 0
    assert B.moe_backward_workspace_bytes(problem(k=9)) == 0
    assert route_backward(p, ws=None) == B.MOE_ERR_WORKSPACE
    assert route_backward(p, ws=ODD) == B.MOE_ERR_WORKSPACE
    assert route_backward(p, ws=None, dWg=None) == B.MOE_ERR_WORKSPACE


def test_row_views_that_are_not_alike_are_refused():
    class Rows:  # a device tensor as far as the binding looks
        is_cuda = True

        def __init__(self, shape, strides):
            self.shape, self._s = shape, strides

        def stride(self, i):
            return self._s[i]

        def data_ptr(self):
            return 0x10000
    ok = Rows((4, 64), (128, 1))
    assert B._row_ptrs(ok, ok)[2] == 128
    assert B._row_ptrs(Rows((1, 64), (1, 1)), Rows((1, 64), (64, 1)))[2] == 64  # (one row: its stride says nothing)
    for bad in (Rows((4, 64), (64, 1)), Rows((4, 64), (1, 4))):
        with pytest.raises(AssertionError):
            B._row_ptrs(ok, bad)

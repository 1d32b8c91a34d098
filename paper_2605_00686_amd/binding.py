"""Thin ctypes binding of the C ABI in include/moe.h: same names, argument
marshalling only.  Torch supplies device memory and streams; every step of the
path runs in the HIP library.  There is no fallback: if libmoe_hip.so is
missing the import of this module fails."""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmoe_hip.so")

MOE_OK = 0
MOE_ERR_INVALID_ARG, MOE_ERR_UNSUPPORTED, MOE_ERR_WORKSPACE = -1, -2, -3
MOE_ERR_NOT_READY, MOE_ERR_HIP, MOE_ERR_TIMEOUT, MOE_ERR_BAD_ROUTING, MOE_ERR_CAPACITY = -4, -5, -6, -7, -8
MOE_DT_F32, MOE_DT_BF16 = 0, 1
MOE_SIGNAL_PER_TILE, MOE_SIGNAL_PER_DEST = 0, 1
MOE_SCOPE_AGENT, MOE_SCOPE_SYSTEM = 0, 1
MOE_SCHED_STATIC, MOE_SCHED_READY_QUEUE = 0, 1
MOE_NUM_STATS = 20

EXPORTS = ("moe_workspace_bytes", "moe_num_flags", "moe_status_string", "moe_workspace_init", "moe_route",
           "moe_dispatch", "moe_dispatch_noalloc", "moe_megakernel_forward", "moe_combine", "moe_probe_mfma",
           "moe_probe_stream", "moe_unsort", "moe_unsort_backward", "moe_backward_workspace_bytes", "moe_route_backward",
           "moe_swiglu", "moe_swiglu_backward", "moe_ffn_workspace_bytes", "moe_ffn_up", "moe_ffn_down", "moe_ffn_down_backward",
           "moe_ffn_up_backward", "moe_grad_workspace_bytes", "moe_grad_norm", "moe_grad_clip")


class MoeProblem(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("T", "d", "E", "k", "f", "R", "dtype", "tile_m", "tile_n",
                                              "signal_mode", "fence_scope")] + [("epoch", ctypes.c_uint32),
                                                                                 ("group_size", ctypes.c_int32),
                                                                                 ("scheduler", ctypes.c_int32),
                                                                                 ("capacity", ctypes.c_int32),
                                                                                 ("wait_ticks", ctypes.c_uint32),
                                                                                 ("fuse_ffn", ctypes.c_int32)]


class MoeTensor(ctypes.Structure):
    _fields_ = [("inp", ctypes.c_void_p), ("out", ctypes.c_void_p), ("count", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("unused", ctypes.c_int32)]


class MoeError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is not built: run `python -c 'import __graft_entry__ as g; g.build()'`")
_lib = ctypes.CDLL(LIB_PATH)
_vp, _pp = ctypes.c_void_p, ctypes.POINTER(MoeProblem)
_lib.moe_workspace_bytes.restype = ctypes.c_size_t
_lib.moe_workspace_bytes.argtypes = [_pp]
_lib.moe_num_flags.restype = ctypes.c_size_t
_lib.moe_num_flags.argtypes = [_pp]
_lib.moe_status_string.restype = ctypes.c_char_p
_lib.moe_status_string.argtypes = [ctypes.c_int]
_lib.moe_workspace_init.argtypes = [_pp, _vp, _vp]
_lib.moe_route.argtypes = [_pp] + [_vp] * 6
_lib.moe_dispatch.argtypes = [_pp] + [_vp] * 10
_lib.moe_dispatch_noalloc.argtypes = [_pp] + [_vp] * 9
_lib.moe_megakernel_forward.argtypes = [_pp] + [_vp] * 19
_lib.moe_combine.argtypes = [_pp] + [_vp] * 7
_lib.moe_probe_mfma.argtypes = [_vp, ctypes.c_int32, ctypes.c_int32, _vp, _vp]
_lib.moe_probe_stream.argtypes = [_vp, ctypes.c_size_t, ctypes.c_size_t, ctypes.c_size_t, ctypes.c_int32, ctypes.c_int32,
                                  ctypes.c_int32, _vp, _vp]
_lib.moe_unsort.argtypes = [_pp] + [_vp] * 7
_lib.moe_unsort_backward.argtypes = [_pp] + [_vp] * 9
_lib.moe_backward_workspace_bytes.restype = ctypes.c_size_t
_lib.moe_backward_workspace_bytes.argtypes = [_pp]
_lib.moe_route_backward.argtypes = [_pp] + [_vp] * 11
_lib.moe_swiglu.argtypes = [_pp, _vp, _vp, ctypes.c_int64] + [_vp] * 5
_lib.moe_swiglu_backward.argtypes = [_pp] + [_vp] * 6 + [ctypes.c_int64, _vp, _vp]
_lib.moe_ffn_workspace_bytes.restype = ctypes.c_size_t
_lib.moe_ffn_workspace_bytes.argtypes = [_pp]
_lib.moe_ffn_up.argtypes = [_pp, _vp, _vp, _vp, ctypes.c_int64, _vp, _vp, _vp, ctypes.c_int64, _vp, _vp, _vp]
_lib.moe_ffn_down.argtypes = [_pp] + [_vp] * 6
_lib.moe_ffn_down_backward.argtypes = [_pp] + [_vp] * 9 + [ctypes.c_int64] + [_vp] * 3
_lib.moe_ffn_up_backward.argtypes = [_pp, _vp, _vp, _vp, ctypes.c_int64, _vp, _vp, ctypes.c_int64] + [_vp] * 6
_tp = ctypes.POINTER(MoeTensor)
_lib.moe_grad_workspace_bytes.restype = ctypes.c_size_t
_lib.moe_grad_workspace_bytes.argtypes = [_tp, ctypes.c_int32]
_lib.moe_grad_norm.argtypes = [_tp, ctypes.c_int32] + [_vp] * 4
_lib.moe_grad_clip.argtypes = [_tp, ctypes.c_int32, _vp, ctypes.c_float, _vp]
for _n in ("moe_workspace_init", "moe_route", "moe_dispatch", "moe_dispatch_noalloc", "moe_megakernel_forward",
           "moe_combine", "moe_probe_mfma", "moe_probe_stream", "moe_unsort", "moe_unsort_backward", "moe_route_backward",
           "moe_swiglu", "moe_swiglu_backward", "moe_ffn_up", "moe_ffn_down", "moe_ffn_down_backward", "moe_ffn_up_backward",
           "moe_grad_norm", "moe_grad_clip"):
    getattr(_lib, _n).restype = ctypes.c_int


def problem(T, d, E, k, f, R, dtype, tile_m=0, tile_n=0, signal_mode=MOE_SIGNAL_PER_DEST,
            fence_scope=MOE_SCOPE_AGENT, epoch=1, group_size=0, scheduler=0, capacity=0, wait_ticks=0,
            fuse_ffn=0) -> MoeProblem:
    if isinstance(dtype, torch.dtype):
        dtype = MOE_DT_F32 if dtype == torch.float32 else MOE_DT_BF16
    elif isinstance(dtype, str):
        dtype = MOE_DT_F32 if dtype == "f32" else MOE_DT_BF16
    return MoeProblem(T, d, E, k, f, R, dtype, tile_m, tile_n, signal_mode, fence_scope, epoch, group_size, scheduler,
                      capacity, wait_ticks, fuse_ffn)


def _ptr(t):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device tensors, contiguous"
    return t.data_ptr()


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    # torch.cuda.current_stream() makes an object first: 2.9 us, more than a launch
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _check(rc, where):
    if rc != MOE_OK:
        raise MoeError(rc, where)


def status_string(status: int) -> str:
    return _lib.moe_status_string(int(status)).decode()


def moe_workspace_bytes(p: MoeProblem) -> int:
    return int(_lib.moe_workspace_bytes(ctypes.byref(p)))


def moe_num_flags(p: MoeProblem) -> int:
    return int(_lib.moe_num_flags(ctypes.byref(p)))


def moe_workspace_init(p, workspace, stream=None):
    _check(_lib.moe_workspace_init(ctypes.byref(p), _ptr(workspace), _stream(stream)), "moe_workspace_init")


def moe_route(p, x, Wg, gate_bias, topk_idx, topk_w, stream=None):
    _check(_lib.moe_route(ctypes.byref(p), _ptr(x), _ptr(Wg), _ptr(gate_bias), _ptr(topk_idx), _ptr(topk_w),
                          _stream(stream)), "moe_route")


def moe_dispatch(p, x, topk_idx, counts, offsets, perm, inv_perm, x_perm, status_dev, workspace, stream=None):
    _check(_lib.moe_dispatch(ctypes.byref(p), _ptr(x), _ptr(topk_idx), _ptr(counts), _ptr(offsets), _ptr(perm),
                             _ptr(inv_perm), _ptr(x_perm), _ptr(status_dev), _ptr(workspace), _stream(stream)),
           "moe_dispatch")


def moe_dispatch_noalloc(p, x, topk_idx, counts, offsets, perm, inv_perm, x_perm, status_dev, stream=None):
    _check(_lib.moe_dispatch_noalloc(ctypes.byref(p), _ptr(x), _ptr(topk_idx), _ptr(counts), _ptr(offsets), _ptr(perm),
                                     _ptr(inv_perm), _ptr(x_perm), _ptr(status_dev), _stream(stream)),
           "moe_dispatch_noalloc")


def moe_megakernel_forward(p, x, Wg, gate_bias, W1, W3, W2, topk_idx, topk_w, counts, offsets, perm, inv_perm,
                           slot_flag, staging, flags, out, stats, workspace, stream=None):
    _check(_lib.moe_megakernel_forward(ctypes.byref(p), _ptr(x), _ptr(Wg), _ptr(gate_bias), _ptr(W1), _ptr(W3),
                                       _ptr(W2), _ptr(topk_idx), _ptr(topk_w), _ptr(counts), _ptr(offsets),
                                       _ptr(perm), _ptr(inv_perm), _ptr(slot_flag), _ptr(staging), _ptr(flags),
                                       _ptr(out), _ptr(stats), _ptr(workspace), _stream(stream)),
           "moe_megakernel_forward")


def moe_combine(p, staging, flags, slot_flag, topk_w, out, status_dev, stream=None):
    _check(_lib.moe_combine(ctypes.byref(p), _ptr(staging), _ptr(flags), _ptr(slot_flag), _ptr(topk_w), _ptr(out),
                            _ptr(status_dev), _stream(stream)), "moe_combine")


def moe_unsort(p, rows, inv_perm, topk_w, addend, out, status_dev, stream=None):
    _check(_lib.moe_unsort(ctypes.byref(p), _ptr(rows), _ptr(inv_perm), _ptr(topk_w), _ptr(addend), _ptr(out),
                           _ptr(status_dev), _stream(stream)), "moe_unsort")


def moe_unsort_backward(p, dout, rows, inv_perm, topk_w, counts, drows, dtopk_w, status_dev, stream=None):
    _check(_lib.moe_unsort_backward(ctypes.byref(p), _ptr(dout), _ptr(rows), _ptr(inv_perm), _ptr(topk_w), _ptr(counts),
                                    _ptr(drows), _ptr(dtopk_w), _ptr(status_dev), _stream(stream)), "moe_unsort_backward")


def moe_backward_workspace_bytes(p: MoeProblem) -> int:
    return int(_lib.moe_backward_workspace_bytes(ctypes.byref(p)))


def moe_route_backward(p, x, Wg, topk_idx, topk_w, dtopk_w, dx, dWg, dgate_bias, status_dev, workspace, stream=None):
    _check(_lib.moe_route_backward(ctypes.byref(p), _ptr(x), _ptr(Wg), _ptr(topk_idx), _ptr(topk_w), _ptr(dtopk_w), _ptr(dx),
                                   _ptr(dWg), _ptr(dgate_bias), _ptr(status_dev), _ptr(workspace), _stream(stream)),
           "moe_route_backward")


def _row_ptrs(a, b):
    """Two [rows, f] tensors or views whose rows are the same number of elements apart: both addresses, and that number."""
    (rows, f), ld = a.shape, a.stride(0)
    assert a.is_cuda and b.is_cuda and a.shape == b.shape and a.stride(1) == b.stride(1) == 1, "device tensors, rows of one piece"
    assert rows == 1 or ld == b.stride(0), "rows the same number of elements apart"
    return a.data_ptr(), b.data_ptr(), ld if rows > 1 else f


def moe_swiglu(p, g, u, counts, h, codes, scales, stream=None):
    gp, up, ld = _row_ptrs(g, u)
    _check(_lib.moe_swiglu(ctypes.byref(p), gp, up, ld, _ptr(counts), _ptr(h), _ptr(codes), _ptr(scales), _stream(stream)),
           "moe_swiglu")


def moe_swiglu_backward(p, dh, codes, scales, counts, dg, du, h, stream=None):
    gp, up, ld = _row_ptrs(dg, du)
    _check(_lib.moe_swiglu_backward(ctypes.byref(p), _ptr(dh), _ptr(codes), _ptr(scales), _ptr(counts), gp, up, ld, _ptr(h),
                                    _stream(stream)), "moe_swiglu_backward")


def moe_ffn_workspace_bytes(p: MoeProblem) -> int:
    return int(_lib.moe_ffn_workspace_bytes(ctypes.byref(p)))


def _here(*tensors):
    """The tensors are the current device's, which the launch goes to."""
    device = torch._C._cuda_getDevice()  # (torch.cuda.current_device() takes twice as long)
    for t in tensors:
        assert t is None or t.get_device() == device, "tensors of the current device"


def _like_rows(*tensors):
    """[rows, f] tensors or views (or None) whose rows are the same number of elements apart: that number, and their addresses."""
    shape = None
    out = [0]
    for t in tensors:
        if t is None:
            out.append(None)
            continue
        if shape is None:
            shape = t.shape
            rows, f = shape
            out[0] = ld = t.stride(0) if rows > 1 else f
        step = t.stride()
        assert t.is_cuda and t.shape == shape and (step[1] == 1 or f == 1), "device tensors, rows of one piece"
        assert rows == 1 or step[0] == ld, "rows the same number of elements apart"
        out.append(t.data_ptr())
    return out


def _like_matrices(*tensors):
    """[E, d, f] tensors or views (or None), matrix behind matrix, whose rows are the same number of elements apart: as _like_rows."""
    shape = None
    out = [0]
    for t in tensors:
        if t is None:
            out.append(None)
            continue
        if shape is None:
            shape = t.shape
            E, d, f = shape
            out[0] = ld = t.stride(1) if d > 1 else t.stride(0) if E > 1 else f
        step = t.stride()
        assert t.is_cuda and t.shape == shape and (step[2] == 1 or f == 1), "device tensors, rows of one piece"
        assert (d == 1 or step[1] == ld) and (E == 1 or step[0] == d * ld), "rows the same number of elements apart, matrix behind matrix"
        out.append(t.data_ptr())
    return out


def _fit(p, counts, rows_d=(), rows_f=(), matrices=(), views=(), matrix_views=()):
    """Tensors (or None) of the types that the calls read and write, and not shorter: contiguous [rows, d], [rows, f] and [E, f, d], views [rows, f]
    and [E, d, f].  (The C calls see addresses.)"""
    dtype, E, d, f, capacity = torch.float32 if p.dtype == MOE_DT_F32 else torch.bfloat16, p.E, p.d, p.f, p.capacity
    assert counts is None or counts.dtype == torch.int32 and counts.numel() >= E, "counts: int32, one per expert"
    rows = E * capacity if capacity else p.T * p.k
    for size, tensors in ((rows * d, rows_d), (rows * f, rows_f), (E * d * f, matrices)):
        for t in tensors:
            assert t is None or t.dtype == dtype and t.numel() >= size, "tensors of the problem's type and size"
    for t in views:
        assert t is None or t.dtype == dtype and t.shape[0] >= rows and t.shape[1] == f, "rows of the problem's type and size"
    for t in matrix_views:
        assert t is None or t.dtype == dtype and t.shape[0] >= E and t.shape[1] == d and t.shape[2] == f, "matrices of the problem's type and size"


def _ffn_workspace(p, workspace):
    """Its address; the C call cannot see how long it is."""
    assert workspace is None or workspace.nbytes >= _lib.moe_ffn_workspace_bytes(ctypes.byref(p)), "a workspace of moe_ffn_workspace_bytes()"
    return _ptr(workspace)


def moe_ffn_up(p, x_perm, W1, W3, counts, g, u, h, workspace, stream=None):
    _here(x_perm, W1, W3, counts, g, u, h, workspace)
    _fit(p, counts, (x_perm,), (h,), (), (g, u), (W1, W3))
    ldw, w1, w3 = _like_matrices(W1, W3)
    ld, gp, up = _like_rows(g, u)
    _check(_lib.moe_ffn_up(ctypes.byref(p), _ptr(x_perm), w1, w3, ldw, _ptr(counts), gp, up, ld, _ptr(h), _ffn_workspace(p, workspace),
                           _stream(stream)), "moe_ffn_up")


def moe_ffn_down(p, h, W2, counts, y, workspace, stream=None):
    _here(h, W2, counts, y, workspace)
    _fit(p, counts, (y,), (h,), (W2,))
    _check(_lib.moe_ffn_down(ctypes.byref(p), _ptr(h), _ptr(W2), _ptr(counts), _ptr(y), _ffn_workspace(p, workspace), _stream(stream)),
           "moe_ffn_down")


def moe_ffn_down_backward(p, dy, W2, h, g, u, counts, dh, dg, du, dW2, workspace, stream=None):
    _here(dy, W2, h, g, u, counts, dh, dg, du, dW2, workspace)
    _fit(p, counts, (dy,), (h, dh), (W2, dW2), (g, u, dg, du))
    ld, gp, up, dgp, dup = _like_rows(g, u, dg, du)
    _check(_lib.moe_ffn_down_backward(ctypes.byref(p), _ptr(dy), _ptr(W2), _ptr(h), gp, up, _ptr(counts), _ptr(dh), dgp, dup, ld,
                                      _ptr(dW2), _ffn_workspace(p, workspace), _stream(stream)), "moe_ffn_down_backward")


def moe_ffn_up_backward(p, x_perm, W1, W3, dg, du, counts, dx, dW1, dW3, workspace, stream=None):
    _here(x_perm, W1, W3, dg, du, counts, dx, dW1, dW3, workspace)
    _fit(p, counts, (x_perm, dx), (), (), (dg, du), (W1, W3, dW1, dW3))
    ldw, w1, w3, dw1, dw3 = _like_matrices(W1, W3, dW1, dW3)
    ld, dgp, dup = _like_rows(dg, du)
    _check(_lib.moe_ffn_up_backward(ctypes.byref(p), _ptr(x_perm), w1, w3, ldw, dgp, dup, ld, _ptr(counts), _ptr(dx), dw1, dw3,
                                    _ffn_workspace(p, workspace), _stream(stream)), "moe_ffn_up_backward")


class TensorList:
    """Gradients, and where they go, as moe_grad_norm and moe_grad_clip take them; holds the tensors."""

    def __init__(self, ins, outs):
        assert len(ins) == len(outs), "an output for every input"
        for i, o in zip(ins, outs):
            assert i.is_cuda and i.is_contiguous() and o.is_contiguous() and o.device == i.device, "device tensors, contiguous"
            assert i.dtype == o.dtype and i.numel() == o.numel() and i.dtype in (torch.float32, torch.bfloat16), "fp32 or bf16, both the same"
        # (one named twice would be counted twice, and scaled by whoever comes first or by both)
        spans = []
        for i, o in zip(ins, outs):
            for t in (i,) if i.data_ptr() == o.data_ptr() else (i, o):
                if t.numel():
                    spans.append((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()))
        spans.sort()
        assert all(a[1] <= b[0] for a, b in zip(spans, spans[1:])), "tensors that do not overlap"
        assert len({t.get_device() for t in ins}) <= 1, "tensors of one device"
        self.one = ins[0] if len(ins) else None
        self.tensors = list(ins), list(outs)
        self.n = len(self.tensors[0])
        self.array = (MoeTensor * max(1, self.n))(*(MoeTensor(i.data_ptr(), o.data_ptr(), i.numel(), MOE_DT_F32 if i.dtype == torch.float32 else MOE_DT_BF16, 0)
                                                    for i, o in zip(*self.tensors)))
        self.workspace_bytes = int(_lib.moe_grad_workspace_bytes(self.array, self.n))


def tensor_list(ins, outs=None) -> TensorList:
    """What moe_grad_norm and moe_grad_clip work on; without `outs` the tensors themselves are scaled."""
    return TensorList(ins, ins if outs is None else outs)


def moe_grad_workspace_bytes(tensors: TensorList) -> int:
    return tensors.workspace_bytes


def _norm_fits(sum_squares, norm=None):
    assert sum_squares is None or sum_squares.dtype == torch.float64 and sum_squares.numel(), "sum_squares: float64"
    assert norm is None or norm.dtype == torch.float32 and norm.numel(), "norm: float32"


def moe_grad_norm(tensors, sum_squares, norm, workspace, stream=None):
    _here(tensors.one, sum_squares, norm, workspace)
    _norm_fits(sum_squares, norm)
    assert workspace is None or workspace.nbytes >= tensors.workspace_bytes, "a workspace of moe_grad_workspace_bytes()"
    _check(_lib.moe_grad_norm(tensors.array, tensors.n, _ptr(sum_squares), _ptr(norm), _ptr(workspace), _stream(stream)), "moe_grad_norm")


def moe_grad_clip(tensors, sum_squares, max_norm, stream=None):
    _here(tensors.one, sum_squares)
    _norm_fits(sum_squares)
    _check(_lib.moe_grad_clip(tensors.array, tensors.n, _ptr(sum_squares), float(max_norm), _stream(stream)), "moe_grad_clip")


def moe_probe_mfma(frag, iters, workgroups, sink, stream=None):
    _check(_lib.moe_probe_mfma(_ptr(frag), int(iters), int(workgroups), _ptr(sink), _stream(stream)), "moe_probe_mfma")


def moe_probe_stream(buf, span_bytes, stride_bytes, bytes_per_workgroup, workgroups, wavefronts, to_lds, sink, stream=None):
    _check(_lib.moe_probe_stream(_ptr(buf), int(span_bytes), int(stride_bytes), int(bytes_per_workgroup), int(workgroups),
                                 int(wavefronts), int(to_lds), _ptr(sink), _stream(stream)), "moe_probe_stream")


class Buffers:
    """Device buffers for one problem shape (allocation only; no arithmetic)."""

    def __init__(self, p: MoeProblem, device="cuda"):
        dt = torch.float32 if p.dtype == MOE_DT_F32 else torch.bfloat16
        N = p.T * p.k
        i32 = dict(dtype=torch.int32, device=device)
        self.p = p
        self.topk_idx = torch.empty((p.T, p.k), **i32)
        self.topk_w = torch.empty((p.T, p.k), dtype=torch.float32, device=device)
        self.counts = torch.empty(p.E, **i32)
        self.offsets = torch.empty(p.E + 1, **i32)
        self.perm = torch.empty(p.E * p.capacity if p.capacity > 0 else N, **i32)  # sorted rows, padded or ragged
        self.inv_perm = torch.empty(N, **i32)
        self.slot_flag = torch.empty(N, **i32)
        self.staging = torch.empty((N, p.d), dtype=dt, device=device)
        self.out = torch.empty((p.T, p.d), dtype=dt, device=device)
        self.flags = torch.zeros(max(1, moe_num_flags(p)), **i32)
        self.stats = torch.zeros(MOE_NUM_STATS, dtype=torch.int64, device=device)
        nbytes = moe_workspace_bytes(p)
        if nbytes == 0:
            raise MoeError(MOE_ERR_UNSUPPORTED, "moe_workspace_bytes")
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
        off = (-self.workspace.data_ptr()) % 256
        self.workspace = self.workspace[off:off + nbytes]
        moe_workspace_init(p, self.workspace)


def forward(p: MoeProblem, buf: Buffers, x, Wg, gate_bias, W1, W3, W2, stream=None):
    """One pass of the whole hot path.  With Wg None, buf.topk_idx / buf.topk_w are inputs."""
    moe_megakernel_forward(p, x, Wg, gate_bias, W1, W3, W2, buf.topk_idx, buf.topk_w, buf.counts, buf.offsets,
                           buf.perm, buf.inv_perm, buf.slot_flag, buf.staging, buf.flags, buf.out, buf.stats,
                           buf.workspace, stream)
    return buf.out

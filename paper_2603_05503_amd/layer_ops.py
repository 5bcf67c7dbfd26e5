"""ctypes marshalling of what a layer does around its attention: rotary positions with several axes, layer norm
and its gradients.  As in ``binding``: every step runs in the C/HIP library, torch supplies buffers and streams."""
from __future__ import annotations

import contextlib
import ctypes as C
from typing import Optional, Sequence

import numpy as np

from . import binding as _b

_NO_SWITCH = contextlib.nullcontext()


class _CRope(C.Structure):
    _fields_ = [("n_axes", C.c_int32), ("interleaved", C.c_int32), ("dims", C.c_int32 * 4), ("length", C.c_int32 * 4),
                ("table", C.c_void_p)]


class _CRopePlace(C.Structure):
    _fields_ = [("grid", C.c_int32 * 4), ("start", C.c_int32 * 4), ("positions", C.c_void_p), ("positions_b", C.c_int64)]


def declare(lib):
    """Argument types of the calls of this module."""
    i32p, f32p, i64p = C.POINTER(C.c_int32), C.POINTER(C.c_float), C.POINTER(C.c_int64)
    lib.calibatt_rope_table.restype = C.c_int
    lib.calibatt_rope_table.argtypes = [C.c_int, i32p, i32p, C.POINTER(C.c_double), C.c_double, f32p, C.c_int64, i64p]
    lib.calibatt_rope_axes.restype = C.c_int
    lib.calibatt_rope_axes.argtypes = [C.c_void_p] * 4 + [C.c_int] * 5 + [C.c_void_p] * 6 + [C.c_int, C.c_int, C.c_void_p]
    lib.calibatt_layer_norm_fwd.restype = C.c_int
    lib.calibatt_layer_norm_fwd.argtypes = [C.c_void_p] * 4 + [C.c_int64] * 3 + [C.c_int] + [C.c_void_p] * 2 + [
        C.c_float, C.c_int, C.c_int, C.c_int, C.c_void_p]
    lib.calibatt_layer_norm_bwd_workspace_bytes.restype = C.c_int
    lib.calibatt_layer_norm_bwd_workspace_bytes.argtypes = [C.c_int, i64p]
    lib.calibatt_layer_norm_bwd.restype = C.c_int
    lib.calibatt_layer_norm_bwd.argtypes = [C.c_void_p] * 6 + [C.c_int64] * 3 + [C.c_int] + [C.c_void_p] * 3 + [
        C.c_float, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_int64, C.c_void_p]
    lib.calibatt_window_attn_workspace_bytes.restype = C.c_int
    lib.calibatt_window_attn_workspace_bytes.argtypes = [C.c_int] * 6 + [C.c_void_p, i64p, i64p]
    lib.calibatt_window_attn_form.restype = C.c_int
    lib.calibatt_window_attn_form.argtypes = [C.c_int] * 6 + [C.c_void_p] * 2
    lib.calibatt_window_attn_fwd.restype = C.c_int
    lib.calibatt_window_attn_fwd.argtypes = [C.c_void_p] * 5 + [C.c_int] * 6 + [C.c_void_p, C.c_float] + [C.c_void_p] * 3 + [
        C.c_int, C.c_void_p, C.c_int64, C.c_void_p]
    lib.calibatt_window_attn_bwd.restype = C.c_int
    lib.calibatt_window_attn_bwd.argtypes = [C.c_void_p] * 9 + [C.c_int] * 6 + [C.c_void_p, C.c_float] + [C.c_void_p] * 6 + [
        C.c_int, C.c_void_p, C.c_int64, C.c_void_p]


_dtypes = None


def _dtype_of(t):
    """The library's number of a tensor's element type, or None."""
    global _dtypes
    if _dtypes is None:
        import torch

        _dtypes = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
    return _dtypes.get(t.dtype)


# What the checks of a call found, and the arguments that follow from shapes, strides and element types alone, by exactly
# these: a small call's time is the host's, and checking and laying them out again takes a third of it (q and k of two
# heads of 1024 tokens 11.3 us, with this 9.0; nothing of a tensor's memory or identity is kept).
_plans = {}


def _remember(key, plan):
    if len(_plans) >= 1024:
        _plans.clear()
    _plans[key] = plan
    return plan


def _on(device):
    """Context in which ``device`` is the current one: kernels are launched on the current device."""
    import torch

    return _NO_SWITCH if device.index == torch.cuda.current_device() else torch.cuda.device(device)


def _empty_like(t, other):
    """``torch.empty_like`` of the call's stream (see ``binding._stream_of``), to be returned."""
    import torch

    if other is None:
        return torch.empty_like(t)
    current = torch.cuda.current_stream(t.device)
    with torch.cuda.stream(other):
        out = torch.empty_like(t)
    out.record_stream(current)
    return out


def _strides(*tensors):
    """The b, h, n strides of [B, H, N, D] tensors as one array of int64, and the address of each tensor's three."""
    flat = []
    for t in tensors:
        flat += t.stride()[:3]
    array = (C.c_int64 * len(flat))(*flat)
    at = C.addressof(array)
    return array, [at + 24 * i for i in range(len(tensors))]


class RotaryAxes:
    """Cosines and sines of rotary positions with several axes, on the GPU.

    ``dims``: channels of each axis (even; their pairs follow each other), ``lengths``: positions that each axis may
    take, ``scale``: factor of each axis's positions.  ``interleaved``: pairs are channels 2j and 2j + 1, else j and j +
    sum(dims) / 2.  Pair i of an axis turns by pos * scale * theta^(-2 i / dims).  The angles are computed in 64 bits."""

    def __init__(self, dims: Sequence[int], lengths: Sequence[int], theta: float = 10000.0,
                 scale: Optional[Sequence[float]] = None, interleaved: bool = True, device="cuda"):
        import torch

        lib = _b.load_library()
        self.dims, self.lengths = tuple(int(d) for d in dims), tuple(int(n) for n in lengths)
        if not (1 <= len(self.dims) <= 4 and len(self.lengths) == len(self.dims)):
            raise ValueError("one to four axes, with as many lengths")
        if scale is not None and len(scale) != len(self.dims):
            raise ValueError("one scale per axis")
        n = len(self.dims)
        d, ln = (C.c_int32 * n)(*self.dims), (C.c_int32 * n)(*self.lengths)
        sc = None if scale is None else (C.c_double * n)(*(float(s) for s in scale))
        entries = C.c_int64(0)
        st = lib.calibatt_rope_table(n, d, ln, sc, float(theta), None, 0, C.byref(entries))
        if st == 0:
            host = np.empty((max(entries.value, 1), 2), np.float32)
            st = lib.calibatt_rope_table(n, d, ln, sc, float(theta), _b._ptr(host, C.c_float), entries.value, C.byref(entries))
        if st != 0:
            raise _b.CalibattError(st, "calibatt_rope_table")
        self.interleaved = bool(interleaved)
        self.host_table = host
        self.table = torch.from_numpy(host).to(device)
        self._c = _CRope(n, 1 if interleaved else 0, (C.c_int32 * 4)(*self.dims), (C.c_int32 * 4)(*self.lengths),
                         self.table.data_ptr())
        self._c_at = C.addressof(self._c)


def rope_axes(q, k, rope: RotaryAxes, grid=None, start=None, positions=None, q_out=None, k_out=None, inverse: bool = False,
              stream=None):
    """calibatt_rope_axes on CUDA tensors q [B, Hq, N, D] and k [B, Hk, N, D] (or None) of one element type (bf16, fp16 or
    fp32), strided views with contiguous D allowed; returns (q_out, k_out), new tensors unless given.

    ``grid``: the first grid[0] * grid[1] * ... tokens are that row-major grid, the first of them at ``start`` (default: all
    zeros); tokens behind it are copied.  Or ``positions``: int32 CUDA tensor [N, axes] or [B, N, axes]; a negative position
    leaves the axis's channels as they are, one behind the table's length gives NaN.  ``inverse`` turns back: with it the
    call takes a gradient of its outputs to that of its inputs.  ``q_out=q, k_out=k`` turns in place."""
    lib = _b.load_library()
    device = q.device
    key = ("rope", rope.dims, rope.lengths, q.shape, q.stride(), q.dtype, k is not None and (k.shape, k.stride(), k.dtype), q.is_cuda,
           q_out is not None and (q_out.shape, q_out.stride(), q_out.dtype),
           k_out is not None and (k_out.shape, k_out.stride(), k_out.dtype),
           positions is not None and (positions.shape, positions.stride(), positions.dtype),
           None if grid is None else tuple(grid), None if start is None else tuple(start))
    plan = _plans.get(key)
    if plan is None:
        plan = _rope_plan(key, q, k, rope, grid, start, positions, q_out, k_out)
    for t in (rope.table, k, q_out, k_out, positions):
        if t is not None and t.device != device:
            raise ValueError("all tensors, and the tables of the axes, must be on one device")
    place, dims, dtype, keep, at = plan
    stream, other = _b._stream_of(stream, device)
    with _on(device):
        if q_out is None:
            q_out = _empty_like(q, other)
        if k is not None and k_out is None:
            k_out = _empty_like(k, other)
        if place is None:
            place = _CRopePlace((C.c_int32 * 4)(), (C.c_int32 * 4)(), positions.data_ptr(),
                                positions.stride(0) if positions.dim() == 3 else 0)
        st = lib.calibatt_rope_axes(q.data_ptr(), q_out.data_ptr(), None if k is None else k.data_ptr(),
                                    None if k is None else k_out.data_ptr(), *dims, rope._c_at, C.addressof(place), *at, dtype,
                                    1 if inverse else 0, stream)
    if st != 0:
        raise _b.CalibattError(st, "calibatt_rope_axes")
    return q_out, k_out


def _rope_plan(key, q, k, rope, grid, start, positions, q_out, k_out):
    """Checks of a ``rope_axes`` call; (place or None, sizes, element type, array of strides, their addresses)."""
    import torch

    shape, dtype, n = q.shape, _dtype_of(q), len(rope.dims)
    if not (q.is_cuda and dtype is not None and len(shape) == 4 and q.stride(3) == 1):
        raise ValueError("q must be a bf16, fp16 or fp32 CUDA tensor [B, H, N, D] with contiguous D")
    if k is not None and not (k.dtype == q.dtype and k.dim() == 4 and k.stride(3) == 1 and k.shape[0] == shape[0]
                              and k.shape[2:] == shape[2:]):
        raise ValueError("k must have q's element type and shape but for the heads, with contiguous D")
    if (grid is None) == (positions is None):
        raise ValueError("either a grid or positions")
    place = None
    if positions is None:
        grid, start = tuple(grid), (0,) * n if start is None else tuple(start)
        if len(grid) != n or len(start) != n:
            raise ValueError(f"grid and start have one entry per axis ({n})")
        place = _CRopePlace((C.c_int32 * 4)(*grid), (C.c_int32 * 4)(*start), None, 0)
    elif start is not None:
        raise ValueError("start belongs to a grid")
    elif not (positions.is_cuda and positions.dtype == torch.int32
              and tuple(positions.shape) in ((shape[2], n), (shape[0], shape[2], n))
              and positions.stride(-1) == 1 and positions.stride(-2) == n):
        raise ValueError(f"positions must be an int32 CUDA tensor [N, {n}] or [B, N, {n}] with contiguous rows")
    for x, x_out in ((q, q_out), (k, k_out)):
        if x_out is not None and (x is None or not (x_out.shape == x.shape and x_out.dtype == x.dtype and x_out.stride(3) == 1)):
            raise ValueError("an output must have its input's shape and element type, with contiguous D")
    # a new output is dense, with its input's order of axes
    tensors = [q, q_out if q_out is not None else torch.empty_like(q, device="meta")]
    if k is not None:
        tensors += [k, k_out if k_out is not None else torch.empty_like(k, device="meta")]
    keep, at = _strides(*tensors)
    return _remember(key, (place, (shape[0], shape[1], 0 if k is None else k.shape[1], shape[2], shape[3]), dtype, keep,
                           at + [None] * (4 - len(at))))


def _rows(t, what):
    """(shape, strides) of a tensor [..., C] as three indices of rows."""
    if not (t.is_cuda and 1 <= t.dim() <= 4 and _dtype_of(t) is not None and (t.stride(-1) == 1 or t.shape[-1] == 1)):
        raise ValueError(f"{what} must be a bf16, fp16 or fp32 CUDA tensor of one to four axes with a contiguous last one")
    pad = 4 - t.dim()
    return (1,) * pad + tuple(t.shape[:-1]), (0,) * pad + t.stride()[:-1]


def _norm_plan(key, x, weight, bias, others):
    """Checks of a layer norm's call; (n0, n1, n2, C), array of the strides of x and of every tensor of ``others`` (None: new,
    dense, with x's order of axes), its address, element types of x and of the weight."""
    import torch

    rows, s = _rows(x, "x")
    flat = list(s)
    for name, t in others:
        if t is None:
            t = torch.empty_like(x, device="meta")
        elif not (t.shape == x.shape and t.dtype == x.dtype):
            raise ValueError(f"{name} must have the shape and element type of x")
        else:
            _rows(t, name)
        flat += (0,) * (4 - t.dim()) + t.stride()[:-1]
    if bias is not None and weight is None:
        raise ValueError("a bias needs a weight")
    dtype = _dtype_of(x)
    for t in (weight, bias):
        if t is not None and not (t.is_cuda and tuple(t.shape) == tuple(x.shape[-1:]) and t.is_contiguous()
                                  and _dtype_of(t) in (dtype, 2) and t.dtype == weight.dtype):
            raise ValueError("weight and bias must be contiguous CUDA tensors [C], both of x's element type or both fp32")
    array = (C.c_int64 * len(flat))(*flat)
    return _remember(key, ((*rows, x.shape[-1]), array, C.addressof(array), dtype, dtype if weight is None else _dtype_of(weight)))


def _like(t):
    return t is not None and (t.shape, t.stride(), t.dtype, t.is_cuda)


def _on_one_device(device, *tensors):
    for t in tensors:
        if t is not None and t.device != device:
            raise ValueError("all tensors must be on one device")


def layer_norm_fwd(x, weight=None, bias=None, eps: float = 1e-6, center: bool = True, out=None, stream=None):
    """calibatt_layer_norm_fwd over the last axis of a CUDA tensor [..., C] of one to four axes (bf16, fp16 or fp32; views
    with a contiguous last axis).  ``weight``, ``bias``: [C] of x's element type or fp32, or None.  ``center=False``: root
    mean square, no mean is taken off.  Returns a new tensor, or ``out`` (which may be x)."""
    lib = _b.load_library()
    key = ("norm", _like(x), _like(weight), _like(bias), _like(out))
    plan = _plans.get(key) or _norm_plan(key, x, weight, bias, (("out", out),))
    sizes, keep, at, dtype, wtype = plan
    device = x.device
    _on_one_device(device, weight, bias, out)
    stream, other = _b._stream_of(stream, device)
    with _on(device):
        y = _empty_like(x, other) if out is None else out
        st = lib.calibatt_layer_norm_fwd(x.data_ptr(), None if weight is None else weight.data_ptr(),
                                         None if bias is None else bias.data_ptr(), y.data_ptr(), *sizes, at, at + 24, float(eps),
                                         1 if center else 0, dtype, wtype, stream)
    if st != 0:
        raise _b.CalibattError(st, "calibatt_layer_norm_fwd")
    return y


_norm_workspace_rows = {}  # device index -> bytes of the workspace for one column


def layer_norm_bwd(dy, x, weight=None, bias=None, eps: float = 1e-6, center: bool = True, dx=None, stream=None):
    """calibatt_layer_norm_bwd: (dx, dweight, dbias) for ``dy``, the gradient of what ``layer_norm_fwd`` gives for the same
    x, weight and bias (of the bias only its presence counts).  dweight and dbias have their parameter's type, None where
    there is none.  ``dx``: optional tensor to receive the gradient of x, which may be dy or x."""
    import torch

    lib = _b.load_library()
    key = ("norm grads", _like(x), _like(dy), _like(weight), _like(bias), _like(dx))
    plan = _plans.get(key) or _norm_plan(key, x, weight, bias, (("dy", dy), ("dx", dx)))
    sizes, keep, at, dtype, wtype = plan
    device = x.device
    _on_one_device(device, dy, weight, bias, dx)
    stream, other = _b._stream_of(stream, device)
    with _on(device):
        to = _empty_like(x, other) if dx is None else dx
        dweight = dbias = workspace = None
        nbytes = 0
        if weight is not None:
            per_column = _norm_workspace_rows.get(device.index)
            if per_column is None:
                n = C.c_int64(0)
                st = lib.calibatt_layer_norm_bwd_workspace_bytes(1, C.byref(n))
                if st != 0:
                    raise _b.CalibattError(st, "calibatt_layer_norm_bwd_workspace_bytes")
                per_column = _norm_workspace_rows[device.index] = n.value
            nbytes = per_column * sizes[3]
            workspace = _b._empty(nbytes // 4, torch.float32, device, other)
            dweight = _empty_like(weight, other)
            dbias = None if bias is None else _empty_like(bias, other)
        st = lib.calibatt_layer_norm_bwd(dy.data_ptr(), x.data_ptr(), None if weight is None else weight.data_ptr(),
                                         to.data_ptr(), None if dweight is None else dweight.data_ptr(),
                                         None if dbias is None else dbias.data_ptr(), *sizes, at + 24, at, at + 48, float(eps),
                                         1 if center else 0, dtype, wtype,
                                         None if workspace is None else workspace.data_ptr(), nbytes, stream)
    if st != 0:
        raise _b.CalibattError(st, "calibatt_layer_norm_bwd")
    return to, dweight, dbias


class _CWindow(C.Structure):
    _fields_ = [("left", C.c_int32), ("right", C.c_int32), ("sinks", C.c_int32), ("frame", C.c_int32), ("offset", C.c_int32),
                ("q_start", C.c_void_p), ("q_len", C.c_void_p), ("k_len", C.c_void_p)]


class _CWindowForm(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("forward", "forward_parts", "dq_parts", "dkv_parts", "sink_parts", "sink_blocks")]


# forms of a window's forward, see Window.form
WINDOW_BLOCKS_128, WINDOW_BLOCKS_32, WINDOW_SHARED_ROWS = 0, 1, 2


class Window:
    """Which keys a query sees (``calibatt_window``): those of ``left`` frames before its own to ``right`` frames behind it
    (-1: all), and the first ``sinks`` keys that are not ahead of that.  ``frame``: tokens of a frame (1: a window of
    tokens).  ``offset``: position of the first query, for calls without ``q_start``: ``Nk - Nq`` where the queries are the
    last of the keys."""

    def __init__(self, left: int, right: int = 0, sinks: int = 0, frame: int = 1, offset: int = 0):
        values = dict(left=left, right=right, sinks=sinks, frame=frame, offset=offset)
        for name, v in values.items():
            if not -(2 ** 31) <= int(v) < 2 ** 31:
                raise ValueError(f"{name} does not fit 32 bits")
        self._values = tuple(int(v) for v in values.values())  # (not to be changed: what is known of a call's sizes hangs on them)
        self._bytes = {}  # sizes of a call -> workspace bytes of its forward and of its gradients

    left, right, sinks, frame, offset = (property(lambda self, i=i: self._values[i]) for i in range(5))

    def _c(self, q_start, q_len, k_len, B, device):
        """The C struct of one call."""
        import torch

        c = _CWindow(*self._values)
        for name, t in (("q_start", q_start), ("q_len", q_len), ("k_len", k_len)):
            if t is not None:
                if not (t.device == device and t.dtype == torch.int32 and t.dim() == 1 and t.shape[0] == B and t.is_contiguous()):
                    raise ValueError(f"{name} must be a contiguous int32 CUDA tensor with one entry per batch entry")
                setattr(c, name, t.data_ptr())
        return c

    def workspace_bytes(self, B: int, Hq: int, Hkv: int, Nq: int, Nk: int, D: int):
        """calibatt_window_attn_workspace_bytes: (forward, backward)."""
        key = (B, Hq, Hkv, Nq, Nk, D)
        n = self._bytes.get(key)
        if n is None:
            c, fwd, bwd = _CWindow(*self._values), C.c_int64(0), C.c_int64(0)
            st = _b.load_library().calibatt_window_attn_workspace_bytes(*key, C.addressof(c), C.byref(fwd), C.byref(bwd))
            if st != 0:
                raise _b.CalibattError(st, "calibatt_window_attn_workspace_bytes")
            if len(self._bytes) >= 256:
                self._bytes.clear()
            n = self._bytes[key] = fwd.value, bwd.value
        return n

    def form(self, B: int, Hq: int, Hkv: int, Nq: int, Nk: int, D: int):
        """calibatt_window_attn_form: how a call of these sizes is run, as a dict (``forward``: WINDOW_*)."""
        c, f = _CWindow(*self._values), _CWindowForm()
        st = _b.load_library().calibatt_window_attn_form(B, Hq, Hkv, Nq, Nk, D, C.addressof(c), C.addressof(f))
        if st != 0:
            raise _b.CalibattError(st, "calibatt_window_attn_form")
        return {name: getattr(f, name) for name, _ in f._fields_}


def _window_plan(key, window, q, k, v, others, kv_like=()):
    """Checks of a call; (sizes, element type, workspace bytes, array of strides, their addresses): of q, k and every tensor
    of ``others`` (like q; None: new and dense) and ``kv_like`` (like k; None: new and dense)."""
    import torch

    dtype = _dtype_of(q)
    if not (q.is_cuda and dtype in (0, 1) and q.dim() == 4 and q.stride(3) == 1):
        raise ValueError("q must be a bf16 or fp16 CUDA tensor [B, H, N, D] with contiguous D")
    B, Hq, Nq, D = q.shape
    for t in (k, v):
        if not (t.dim() == 4 and t.dtype == q.dtype and t.stride(3) == 1 and t.shape[0] == B and t.shape[3] == D):
            raise ValueError("k and v must be [B, Hkv, Nk, D] of q's element type, with contiguous D")
    if k.shape != v.shape or k.stride() != v.stride():
        raise ValueError("k and v must share their shape and strides")
    if k.shape[1] == 0 or Hq % k.shape[1]:
        raise ValueError("the query heads must be a multiple of the key heads")
    tensors = [q, k]
    for like, names in ((q, others), (k, kv_like)):
        for name, t in names:
            if t is None:
                t = torch.empty_like(like, device="meta")
            elif not (t.shape == like.shape and t.dtype == q.dtype and t.stride(3) == 1):
                raise ValueError(f"{name} must have the shape and element type of {'q' if like is q else 'k'}, with contiguous D")
            tensors.append(t)
    sizes = (B, Hq, k.shape[1], Nq, k.shape[2], D)
    nbytes = window.workspace_bytes(*sizes)
    keep, at = _strides(*tensors)
    return _remember(key, (sizes, dtype, nbytes, keep, at))


def _check_lse(lse, q):
    import torch

    if not (lse.dtype == torch.float32 and lse.device == q.device and lse.shape == q.shape[:3] and lse.is_contiguous()):
        raise ValueError("lse must be a contiguous fp32 CUDA tensor [B, H, N] on q's device")


def window_attn_fwd(q, k, v, out, window: Window, scale: float, lse=None, q_start=None, q_len=None, k_len=None, stream=None):
    """calibatt_window_attn_fwd on bf16 or fp16 CUDA tensors: q, out [B, Hq, Nq, D], k, v [B, Hkv, Nk, D] (views with
    contiguous D; k and v share their strides; Hq a multiple of Hkv).  ``lse``: optional contiguous fp32 CUDA tensor [B,
    Hq, Nq].  ``q_start``, ``q_len``, ``k_len``: optional int32 CUDA tensors [B]: position of a batch entry's first query,
    how many queries and keys it has; rows behind these lengths may hold anything, their outputs are zeros.  Cut along the
    keys where a few rows of queries would not fill the GPU, with a workspace of the call's own."""
    import torch

    lib = _b.load_library()
    device = q.device
    key = ("window", window._values, _like(q), _like(k), _like(v), _like(out))
    sizes, dtype, nbytes, keep, at = _plans.get(key) or _window_plan(key, window, q, k, v, (("out", out),))
    nbytes = nbytes[0]
    _on_one_device(device, k, v, out)
    if lse is not None:
        _check_lse(lse, q)
    stream, other = _b._stream_of(stream, device)
    c = window._c(q_start, q_len, k_len, sizes[0], device)
    with _on(device):
        workspace = None
        if nbytes:
            try:
                workspace = _b._empty(nbytes // 4, torch.float32, device, other)
            except torch.OutOfMemoryError:
                pass  # whole rows, which take none
        st = lib.calibatt_window_attn_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                                          None if lse is None else lse.data_ptr(), *sizes, C.addressof(c), float(scale), *at, dtype,
                                          None if workspace is None else workspace.data_ptr(), nbytes, stream)
    if st != 0:
        raise _b.CalibattError(st, "calibatt_window_attn_fwd")
    return out


def window_attn_bwd(dout, q, k, v, out, lse, window: Window, scale: float, dq=None, dk=None, dv=None, q_start=None, q_len=None,
                    k_len=None, stream=None):
    """calibatt_window_attn_bwd: (dq, dk, dv) for ``dout``, the gradient of what ``window_attn_fwd`` left in ``out`` for the same
    arguments, and its ``lse``; new tensors unless given (dk and dv share their strides, no result may be an input).  fp16: dout
    may be of any size, that of a scaled loss among them, as long as the gradients themselves are within the type."""
    import torch

    lib = _b.load_library()
    if (dk is None) != (dv is None):
        raise ValueError("dk and dv are given together")
    device = q.device
    key = ("window grads", window._values, _like(q), _like(k), _like(v), _like(dout), _like(out), _like(dq), _like(dk))
    sizes, dtype, nbytes, keep, at = _plans.get(key) or _window_plan(
        key, window, q, k, v, (("dout", dout), ("out", out), ("dq", dq)), (("dk", dk),))
    if dk is not None and not (dv.shape == dk.shape and dv.stride() == dk.stride() and dv.dtype == dk.dtype):
        raise ValueError("dk and dv must share their shape, strides and element type")
    _on_one_device(device, k, v, dout, out, dq, dk, dv)
    _check_lse(lse, q)
    stream, other = _b._stream_of(stream, device)
    c = window._c(q_start, q_len, k_len, sizes[0], device)
    at_q, at_k, at_dout, at_out, at_dq, at_dk = at
    with _on(device):
        dq = _empty_like(q, other) if dq is None else dq
        if dk is None:
            dk, dv = _empty_like(k, other), _empty_like(k, other)
        workspace = _b._empty(nbytes[1] // 4, torch.float32, device, other)
        st = lib.calibatt_window_attn_bwd(dout.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(),
                                          dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), *sizes, C.addressof(c), float(scale), at_dout, at_q,
                                          at_k, at_out, at_dq, at_dk, dtype, workspace.data_ptr(), nbytes[1], stream)
    if st != 0:
        raise _b.CalibattError(st, "calibatt_window_attn_bwd")
    return dq, dk, dv

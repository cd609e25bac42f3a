"""Projections of language models on 1x1 layers: experts with ragged row counts, the router in front of them, the
weighted sum behind them, and low-rank adapters of many requests beside one projection.

The names mirror include/snn_conv.h (snn_conv_experts_create -> SnnConvExperts(...), snn_conv_experts_route ->
route(...), snn_conv_experts_combine -> combine(...), snn_conv_adapters_create -> SnnConvAdapters(...)).  As in
binding.py, tensors are torch CUDA tensors used purely as device memory, and there is no fallback.

Rows of activations, outputs and logits may lie further apart than they are long (a slice of a wider buffer); all
other tensors are contiguous.  Calls are asynchronous on `stream` (default: torch's current stream); nothing is
recorded for autograd.
"""
from __future__ import annotations

import ctypes
import struct

from . import binding
from .binding import ACT_F16, OUT_F32, SnnConv, SnnError, _check, _load_fast, _raw_stream, load_library

ACT_BF16 = 2
OUT_F16, OUT_BF16 = 3, 4


def _types():
    import torch
    return ({torch.float16: ACT_F16, torch.bfloat16: ACT_BF16},
            {torch.float32: OUT_F32, torch.float16: OUT_F16, torch.bfloat16: OUT_BF16})


def _dtype(out_type):
    import torch
    try:
        return {OUT_F32: torch.float32, OUT_F16: torch.float16, OUT_BF16: torch.bfloat16}[out_type]
    except (KeyError, TypeError):
        raise SnnError(1, f"out_type={out_type} is not OUT_F32, OUT_F16 or OUT_BF16") from None


def _here(t, name, device):
    if t.get_device() != device:
        raise SnnError(1, f"{name} must live on cuda:{device}")
    if t.is_neg():   # (the imaginary part of a conjugated tensor)
        raise SnnError(1, f"{name} is a view of negated memory: resolve_neg() copies it")


def _matrix(t, name, device, columns=None, aligned=False):
    """Elements between the rows of a matrix whose rows are dense."""
    _here(t, name, device)
    if t.dim() != 2 or (columns is not None and t.shape[1] != columns):
        raise SnnError(1, f"{name} must have the shape (rows, {columns if columns is not None else 'columns'})")
    n = t.shape[1]
    if n > 1 and t.stride(1) != 1:
        raise SnnError(1, f"rows of {name} must be dense")
    ld = t.stride(0) if t.shape[0] > 1 else (n + 7) // 8 * 8
    if ld < n:
        raise SnnError(1, f"rows of {name} must not overlap")
    if aligned and (ld % 8 or t.data_ptr() % 16):
        raise SnnError(1, f"rows of {name} must be 16-byte aligned")
    return ld


def _ints(t, name, device, *shape):
    import torch
    _here(t, name, device)
    if t.dtype != torch.int32 or tuple(t.shape) != shape or not t.is_contiguous():
        raise SnnError(1, f"{name} must be a contiguous int32 tensor of shape {shape} on cuda:{device}")
    return t.data_ptr()


def _floats(t, name, device, *shape):
    import torch
    _here(t, name, device)
    if t.dtype != torch.float32 or tuple(t.shape) != shape or not t.is_contiguous():
        raise SnnError(1, f"{name} must be a contiguous float32 tensor of shape {shape} on cuda:{device}")
    return t.data_ptr()


def _output(out, out_type, default, rows, columns, device, exact_rows=True):
    """(out, its rows, elements between them, its SNN_OUT_* type); made where there is none."""
    import torch
    outs = _types()[1]
    if out is None:
        dtype = default if out_type is None else _dtype(out_type)
        out = torch.empty((rows, columns), dtype=dtype, device=f"cuda:{device}")
    elif out.dtype not in outs or (out_type is not None and outs[out.dtype] != out_type):
        raise SnnError(1, "out has the wrong dtype")
    ld = _matrix(out, "out", device, columns)
    if exact_rows and out.shape[0] != rows:
        raise SnnError(1, f"out must have {rows} rows")
    return out, int(out.shape[0]), ld, outs[out.dtype]


def _act_type(x):
    acts = _types()[0]
    if x.dtype not in acts:
        raise SnnError(1, "activations must be float16 or bfloat16")
    return acts[x.dtype]


def _on(stream):
    """Allocations of a call on a stream of the caller's belong to that stream."""
    import contextlib

    import torch
    return torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext()


class SnnConvExperts:
    """Projections of one shape, one for each expert, and rows in the order of their experts (wraps
    snn_conv_experts_t).  `layers` are SnnConv objects with ksize=1 and stride 1; their weights are copied, so they
    may be destroyed afterwards."""

    _h = _desc = None

    def __init__(self, layers):
        lib = load_library()
        layers = list(layers)
        if not layers or not all(isinstance(l, SnnConv) and l._h is not None for l in layers):
            raise SnnError(1, "experts need at least one SnnConv layer")
        hs = (ctypes.c_void_p * len(layers))(*[l._h for l in layers])
        h = ctypes.c_void_p()
        self._h = None
        _check(lib.snn_conv_experts_create(hs, len(layers), ctypes.byref(h)))
        self._h = h
        self.count, self.device = len(layers), layers[0].device
        self.c_in, self.c_out = layers[0].c_in, layers[0].c_out
        self._desc = struct.pack("=Q4i", h.value, self.device, self.count, self.c_in, self.c_out)

    def forward(self, x, offsets, rows=None, out=None, out_type=None, stream=None):
        """snn_conv_experts_forward: out[i] = projection_e(x[rows[i]]) for offsets[e] <= i < offsets[e + 1] (rows None:
        x[i]).  `offsets` (count + 1) and `rows` are int32 tensors that the kernels read: nothing waits for them here.
        `out` has a row for each of `rows` (without rows: any number, by default one for each row of x); its rows
        outside the experts' ranges are left as they are.  Outputs are of the type of `out`, else out_type, else x's."""
        if out is not None and out_type is None and stream is None:
            st = (binding._fast or _load_fast()).experts_forward(self._desc, x, offsets, rows, out)
            if st == 0:
                return out
            if st > 0:
                _check(st)
        if self._h is None:
            raise SnnError(1, "the experts were destroyed")
        act_type = _act_type(x)
        ld_x = _matrix(x, "x", self.device, self.c_in, aligned=True)
        off = _ints(offsets, "offsets", self.device, self.count + 1)
        n = int(x.shape[0] if rows is None else rows.numel())
        row_ptr = None if rows is None else _ints(rows, "rows", self.device, n)
        with _on(stream):
            out, n, ld_out, ot = _output(out, out_type, x.dtype, n, self.c_out, self.device, exact_rows=rows is not None)
        _check(load_library().snn_conv_experts_forward(self._h, x.data_ptr(), act_type, int(x.shape[0]), ld_x, row_ptr, off,
                                                       n, out.data_ptr(), ot, ld_out, _raw_stream(self.device, stream)))
        return out

    def destroy(self):
        if getattr(self, "_h", None) is not None:
            self._desc = None
            load_library().snn_conv_experts_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


class Route:
    """What route() writes: ids, weights and slots [tokens, top_k], offsets [experts + 1], rows [tokens * top_k], in
    this order when iterated over; `work` is the call's workspace."""

    __slots__ = ("ids", "weights", "offsets", "rows", "slots", "work")

    def __init__(self, ids, weights, offsets, rows, slots, work):
        self.ids, self.weights, self.offsets, self.rows, self.slots, self.work = ids, weights, offsets, rows, slots, work

    def __iter__(self):
        return iter((self.ids, self.weights, self.offsets, self.rows, self.slots))


def alloc_route(tokens, experts, top_k, device=0):
    """Tensors for route(..., out=) of these sizes.  Calls that may run at the same time need one each."""
    import torch
    t, e, k = int(tokens), int(experts), int(top_k)
    if t < 0 or e < 1 or k < 1 or t * k >= 1 << 31:
        raise SnnError(1, f"{tokens} tokens, {experts} experts, {top_k} of them for each token")

    def make(dtype, *shape):
        return torch.empty(shape, dtype=dtype, device=f"cuda:{device}")
    work = int(load_library().snn_conv_experts_route_work(t, e)) // 4
    return Route(make(torch.int32, t, k), make(torch.float32, t, k), make(torch.int32, e + 1), make(torch.int32, t * k),
                 make(torch.int32, t, k), make(torch.int32, work))


def route(logits, top_k, normalise=True, out=None, stream=None):
    """snn_conv_experts_route: the top_k experts of each row of `logits` [tokens, experts] (float32, float16 or bfloat16),
    their weights (softmax over the chosen, or over all experts with normalise=False), and the order of the rows by
    expert that SnnConvExperts.forward and combine take.  Returns `out`, or a new Route."""
    if out is not None and stream is None:
        st = (binding._fast or _load_fast()).route(logits, top_k, normalise, out.ids, out.weights, out.offsets, out.rows, out.slots, out.work)
        if st == 0:
            return out
        if st > 0:
            _check(st)
    device = logits.get_device()
    if device < 0:
        raise SnnError(1, "logits must live on a CUDA device")
    types = _types()[1]
    if logits.dtype not in types:
        raise SnnError(1, "logits must be float32, float16 or bfloat16")
    ld = _matrix(logits, "logits", device)
    t, e, k = int(logits.shape[0]), int(logits.shape[1]), int(top_k)
    if out is None:
        with _on(stream):
            out = alloc_route(t, e, k, device)
    lib = load_library()
    ids, weights = _ints(out.ids, "ids", device, t, k), _floats(out.weights, "weights", device, t, k)
    offsets, rows = _ints(out.offsets, "offsets", device, e + 1), _ints(out.rows, "rows", device, t * k)
    slots = _ints(out.slots, "slots", device, t, k)
    need = int(lib.snn_conv_experts_route_work(t, e)) // 4
    if need > out.work.numel():
        raise SnnError(1, "the workspace is for fewer tokens or experts")
    work = _ints(out.work, "work", device, out.work.numel())
    _check(lib.snn_conv_experts_route(logits.data_ptr(), types[logits.dtype], t, e, ld, k, int(bool(normalise)), ids, weights,
                                      offsets, rows, slots, work, device, _raw_stream(device, stream)))
    return out


def combine(y, slots, weights, out=None, out_type=None, stream=None):
    """snn_conv_experts_combine: out[t] = sum_j weights[t, j] * y[slots[t, j]]; a slot outside y counts nothing.  Outputs
    are of the type of `out`, else out_type, else y's."""
    if out is not None and out_type is None and stream is None:
        st = (binding._fast or _load_fast()).combine(y, slots, weights, out)
        if st == 0:
            return out
        if st > 0:
            _check(st)
    device = y.get_device()
    if device < 0:
        raise SnnError(1, "y must live on a CUDA device")
    types = _types()[1]
    if y.dtype not in types:
        raise SnnError(1, "y must be float32, float16 or bfloat16")
    ld_y = _matrix(y, "y", device)
    if slots.dim() != 2:
        raise SnnError(1, "slots must have the shape (tokens, top_k)")
    t, k, c = int(slots.shape[0]), int(slots.shape[1]), int(y.shape[1])
    sp, wp = _ints(slots, "slots", device, t, k), _floats(weights, "weights", device, t, k)
    with _on(stream):
        out, _, ld_out, ot = _output(out, out_type, y.dtype, t, c, device)
    _check(load_library().snn_conv_experts_combine(y.data_ptr(), types[y.dtype], int(y.shape[0]), ld_y, sp, wp, t, k, c,
                                                   out.data_ptr(), ot, ld_out, device, _raw_stream(device, stream)))
    return out


class SnnConvAdapters:
    """One projection shared by many requests, each with a low-rank adapter of its own or none (wraps
    snn_conv_adapters_t).  `layer` is an SnnConv object with ksize=1 and stride 1; its weights are copied."""

    _h = _desc = None

    def __init__(self, layer):
        lib = load_library()
        if not isinstance(layer, SnnConv) or layer._h is None:
            raise SnnError(1, "adapters need an SnnConv layer")
        h = ctypes.c_void_p()
        self._h = None
        _check(lib.snn_conv_adapters_create(layer._h, ctypes.byref(h)))
        self._h = h
        self.device, self.c_in, self.c_out = layer.device, layer.c_in, layer.c_out
        self._desc = struct.pack("=Q4i", h.value, self.device, 1, self.c_in, self.c_out)

    def forward(self, x, adapter, a, b, scale, out=None, out_type=None, stream=None):
        """snn_conv_adapters_forward: out[r] = projection(x[r]) + scale[i] * b[i] @ (a[i] @ x[r]) with i = adapter[r], or
        the projection alone where i is outside [0, adapters).  a [adapters, rank, c_in] and b [adapters, c_out, rank]
        are contiguous and of x's type, scale [adapters] float32, adapter [rows] int32.  Outputs are of the type of
        `out`, else out_type, else x's."""
        if out is not None and out_type is None and stream is None:
            st = (binding._fast or _load_fast()).adapters_forward(self._desc, x, adapter, a, b, scale, out)
            if st == 0:
                return out
            if st > 0:
                _check(st)
        import torch
        if self._h is None:
            raise SnnError(1, "the adapters were destroyed")
        act_type = _act_type(x)
        ld_x = _matrix(x, "x", self.device, self.c_in, aligned=True)
        r = int(x.shape[0])
        ap = _ints(adapter, "adapter", self.device, r)
        if a.dim() != 3 or b.dim() != 3:
            raise SnnError(1, "a must be (adapters, rank, c_in) and b (adapters, c_out, rank)")
        n, rank = int(a.shape[0]), int(a.shape[1])
        for t, name, shape in ((a, "a", (n, rank, self.c_in)), (b, "b", (n, self.c_out, rank))):
            _here(t, name, self.device)
            if t.dtype != x.dtype or tuple(t.shape) != shape or not t.is_contiguous():
                raise SnnError(1, f"{name} must be a contiguous tensor of x's type and shape {shape} on cuda:{self.device}")
        sp = _floats(scale, "scale", self.device, n)
        with _on(stream):
            out, _, ld_out, ot = _output(out, out_type, x.dtype, r, self.c_out, self.device)
            work = torch.empty(r * rank, dtype=torch.float32, device=f"cuda:{self.device}")
        _check(load_library().snn_conv_adapters_forward(self._h, x.data_ptr(), act_type, r, ld_x, ap, a.data_ptr(), b.data_ptr(), sp,
                                                        n, rank, work.data_ptr(), out.data_ptr(), ot, ld_out,
                                                        _raw_stream(self.device, stream)))
        return out

    def destroy(self):
        if getattr(self, "_h", None) is not None:
            self._desc = None
            load_library().snn_conv_adapters_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

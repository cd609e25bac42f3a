"""Whole mixtures of experts for a few tokens, the activation between two projections, and projections in 8-bit floating
point with a scale for each block of 128.

The names mirror include/snn_conv.h (snn_conv_moe_create -> SnnConvMoe(...), snn_conv_experts_activate -> activate(...),
snn_conv_scaled_create -> SnnConvScaled(...), snn_conv_scaled_quantise -> quantise(...)), and the calls behave as those
of projections.py: tensors are torch CUDA tensors used purely as device memory, rows may lie further apart than they are
long, calls are asynchronous on `stream` (default: torch's current stream), and nothing is recorded for autograd.
"""
from __future__ import annotations

import ctypes
import struct
from collections import namedtuple

from . import binding
from .binding import SnnError, _check, _load_fast, _raw_stream, load_library
from .projections import OUT_BF16, SnnConvExperts, _act_type, _dtype, _floats, _here, _ints, _matrix, _on, _output, _types

FN_NONE, FN_RELU, FN_SILU, FN_GELU = 0, 1, 2, 3
MOE_TOKENS_MAX = 64
BLOCK = 128   # of channels with one scale

Quantised = namedtuple("Quantised", "values scales")


def _between(up, gate):
    """Device, type, rows, columns and row lengths of the inputs of an activation."""
    device, types = up.get_device(), _types()[1]
    if device < 0:
        raise SnnError(1, "up must live on a CUDA device")
    if up.dtype not in types:
        raise SnnError(1, "up must be float32, float16 or bfloat16")
    ld_up = _matrix(up, "up", device)
    ld_gate = 0
    if gate is not None:
        ld_gate = _matrix(gate, "gate", device, int(up.shape[1]))
        if gate.dtype != up.dtype or gate.shape[0] != up.shape[0]:
            raise SnnError(1, "gate must be of up's type and shape")
    return device, types[up.dtype], int(up.shape[0]), int(up.shape[1]), ld_up, ld_gate


def _pointer(t):
    return None if t is None else t.data_ptr()


def activate(up, gate=None, fn=FN_SILU, out=None, out_type=None, stream=None):
    """snn_conv_experts_activate: fn(gate) * up, or fn(up) without a gate, for matrices float32, float16 or bfloat16.
    Outputs are of the type of `out`, else out_type, else up's; `out` may be up or gate itself."""
    if out is not None and out_type is None and stream is None:
        st = (binding._fast or _load_fast()).activate(up, gate, fn, out)
        if st == 0:
            return out
        if st > 0:
            _check(st)
    device, kind, rows, columns, ld_up, ld_gate = _between(up, gate)
    with _on(stream):
        out, _, ld_out, ot = _output(out, out_type, up.dtype, rows, columns, device)
    _check(load_library().snn_conv_experts_activate(_pointer(gate), ld_gate, up.data_ptr(), ld_up, kind, rows, columns, int(fn), out.data_ptr(), ot,
                                                    ld_out, device, _raw_stream(device, stream)))
    return out


class SnnConvMoe:
    """A whole mixture of experts for at most MOE_TOKENS_MAX tokens (wraps snn_conv_moe_t).  `up`, `down` and `gate` are
    SnnConvExperts, kept (and kept alive) by reference; do not destroy them before the mixture."""

    _h = _desc = None

    def __init__(self, up, down, gate=None, fn=FN_SILU):
        lib = load_library()
        for x in (up, down) if gate is None else (up, down, gate):
            if not isinstance(x, SnnConvExperts) or x._h is None:
                raise SnnError(1, "a mixture needs SnnConvExperts")
        h = ctypes.c_void_p()
        _check(lib.snn_conv_moe_create(None if gate is None else gate._h, up._h, down._h, int(fn), ctypes.byref(h)))
        self._h, self._experts = h, (up, down, gate)
        self.device, self.count, self.c_in, self.hidden, self.c_out = up.device, up.count, up.c_in, up.c_out, down.c_out
        self._desc = struct.pack("=Q4i", h.value, self.device, self.count, self.c_in, self.c_out)

    def forward(self, x, logits, top_k, normalise=True, out=None, out_type=None, stream=None):
        """snn_conv_moe_forward: out[t] = sum_j w_j down_e(fn(gate_e(x[t])) * up_e(x[t])) over the top_k experts e of
        logits[t], w their weights as route() gives them.  Outputs are of the type of `out`, else out_type, else x's."""
        import torch
        if self._h is None or any(e is not None and e._h is None for e in self._experts):
            raise SnnError(1, "the mixture or its experts were destroyed")
        if out is not None and out_type is None and stream is None:
            st = (binding._fast or _load_fast()).moe_forward(self._desc, x, logits, top_k, normalise, out)
            if st == 0:
                return out
            if st > 0:
                _check(st)
        act_type = _act_type(x)
        ld_x = _matrix(x, "x", self.device, self.c_in, aligned=True)
        types = _types()[1]
        if logits.dtype not in types:
            raise SnnError(1, "logits must be float32, float16 or bfloat16")
        ld_logits, t, k = _matrix(logits, "logits", self.device, self.count), int(x.shape[0]), int(top_k)
        if logits.shape[0] != t:
            raise SnnError(1, f"logits must have {t} rows")
        lib = load_library()
        with _on(stream):
            out, _, ld_out, ot = _output(out, out_type, x.dtype, t, self.c_out, self.device)
            work = torch.empty(max(0, int(lib.snn_conv_moe_work(self._h, t, k))), dtype=torch.uint8, device=f"cuda:{self.device}")
        _check(lib.snn_conv_moe_forward(self._h, x.data_ptr(), act_type, t, ld_x, logits.data_ptr(), types[logits.dtype], ld_logits, k, int(bool(normalise)),
                                        work.data_ptr(), out.data_ptr(), ot, ld_out, _raw_stream(self.device, stream)))
        return out

    def destroy(self):
        if getattr(self, "_h", None) is not None:
            self._desc = None
            load_library().snn_conv_moe_destroy(self._h)
            self._h = self._experts = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def _values(t, name, device, columns, align=1):
    """Bytes between the rows of a matrix of e4m3 values whose rows are dense."""
    import torch
    _here(t, name, device)
    if t.dtype != torch.float8_e4m3fn or t.dim() != 2 or t.shape[1] != columns:
        raise SnnError(1, f"{name} must be float8_e4m3fn of the shape (rows, {columns})")
    if columns > 1 and t.stride(1) != 1:
        raise SnnError(1, f"rows of {name} must be dense")
    ld = t.stride(0) if t.shape[0] > 1 else -(-columns // 16) * 16
    if ld < columns:
        raise SnnError(1, f"rows of {name} must not overlap")
    if ld % align or t.data_ptr() % align:
        raise SnnError(1, f"rows of {name} must be {align}-byte aligned")
    return ld


def _scales(t, name, device, rows, blocks):
    import torch
    if t.dtype != torch.float32:
        raise SnnError(1, f"{name} must be float32")
    ld = _matrix(t, name, device, blocks)
    if t.shape[0] != rows:
        raise SnnError(1, f"{name} must have {rows} rows")
    return ld


def alloc_quantised(rows, columns, device=0):
    """Tensors for quantise(..., out=): values float8_e4m3fn (rows 16-byte aligned) and scales float32."""
    import torch
    r, c = int(rows), int(columns)
    if r < 0 or c < 1:
        raise SnnError(1, f"{rows} rows of {columns} columns")
    values = torch.empty((r, -(-c // 16) * 16), dtype=torch.float8_e4m3fn, device=f"cuda:{device}")[:, :c]
    return Quantised(values, torch.empty((r, -(-c // BLOCK)), dtype=torch.float32, device=f"cuda:{device}"))


def quantise(up, gate=None, fn=FN_NONE, rows=None, out=None, stream=None):
    """snn_conv_scaled_quantise: rows of `up` (float32, float16 or bfloat16) as e4m3 values with a scale for each 128
    columns, behind an activation where fn says so; output row i is of row rows[i] (int32) where there is an index.
    Returns `out`, or a new Quantised(values, scales)."""
    if out is not None and stream is None:
        values, scales = out
        st = (binding._fast or _load_fast()).quantise(up, gate, fn, rows, values, scales)
        if st == 0:
            return out
        if st > 0:
            _check(st)
    device, kind, n, columns, ld_up, ld_gate = _between(up, gate)
    row_ptr, m = None, n
    if rows is not None:
        m = int(rows.numel())
        row_ptr = _ints(rows, "rows", device, m)
    if out is None:
        with _on(stream):
            out = alloc_quantised(m, columns, device)
    values, scales = out
    ld_values = _values(values, "values", device, columns)
    if values.shape[0] != m:
        raise SnnError(1, f"values must have {m} rows")
    ld_scales = _scales(scales, "scales", device, m, -(-columns // BLOCK))
    _check(load_library().snn_conv_scaled_quantise(_pointer(gate), ld_gate, up.data_ptr(), ld_up, kind, n, row_ptr, m, columns, int(fn), values.data_ptr(),
                                                   ld_values, scales.data_ptr(), ld_scales, device, _raw_stream(device, stream)))
    return out


class SnnConvScaled:
    """Projections in e4m3 with a scale for each 128 x 128 weights (wraps snn_conv_scaled_t).  `weights` float8_e4m3fn
    (c_out, c_in) or (projections, c_out, c_in) and `scales` float32 (..., ceil(c_out / 128), ceil(c_in / 128)) are
    contiguous CUDA tensors; they are copied."""

    _h = _desc = None

    def __init__(self, weights, scales, stream=None):
        import torch
        lib = load_library()
        device = weights.get_device()
        if device < 0:
            raise SnnError(1, "weights must live on a CUDA device")
        if weights.dim() == 2:
            weights, scales = weights[None], scales[None]
        if weights.dtype != torch.float8_e4m3fn or weights.dim() != 3 or not weights.is_contiguous():
            raise SnnError(1, "weights must be a contiguous float8_e4m3fn tensor of the shape (projections, c_out, c_in)")
        e, k, c = (int(n) for n in weights.shape)
        sp = _floats(scales, "scales", device, e, -(-k // BLOCK), -(-c // BLOCK))
        h = ctypes.c_void_p()
        _check(lib.snn_conv_scaled_create(weights.data_ptr(), sp, e, c, k, device, _raw_stream(device, stream), ctypes.byref(h)))
        self._h, self.device, self.count, self.c_in, self.c_out = h, device, e, c, k
        self._desc = struct.pack("=Q4i", h.value, device, e, c, k)

    def forward(self, x, scales, offsets=None, out=None, out_type=None, stream=None):
        """snn_conv_scaled_forward: x float8_e4m3fn (rows, c_in) with its scales (rows, ceil(c_in / 128)), as quantise()
        gives them; row i goes through projection e with offsets[e] <= i < offsets[e + 1] (int32, count + 1), without offsets all
        through the first.  Outputs are of the type of `out`, else out_type, else bfloat16; rows outside the
        projections' ranges are left as they are."""
        if out is not None and out_type is None and stream is None:
            st = (binding._fast or _load_fast()).scaled_forward(self._desc, x, scales, offsets, out)
            if st == 0:
                return out
            if st > 0:
                _check(st)
        if self._h is None:
            raise SnnError(1, "the projections were destroyed")
        ld_x = _values(x, "x", self.device, self.c_in, align=16)
        n = int(x.shape[0])
        ld_scales = _scales(scales, "scales", self.device, n, -(-self.c_in // BLOCK))
        off = None if offsets is None else _ints(offsets, "offsets", self.device, self.count + 1)
        with _on(stream):
            out, _, ld_out, ot = _output(out, out_type, _dtype(OUT_BF16), n, self.c_out, self.device)
        _check(load_library().snn_conv_scaled_forward(self._h, x.data_ptr(), ld_x, scales.data_ptr(), ld_scales, off, n, out.data_ptr(), ot, ld_out,
                                                      _raw_stream(self.device, stream)))
        return out

    def destroy(self):
        if getattr(self, "_h", None) is not None:
            self._desc = None
            load_library().snn_conv_scaled_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

"""Projections of language models where there is no GPU: what the C entry points and the binding refuse."""
import ctypes

import pytest
import torch

import paper_2110_09195_b200 as snn
from paper_2110_09195_b200 import binding, projections


@pytest.fixture(scope="module")
def lib():
    from paper_2110_09195_b200 import build
    build.build()
    return binding.load_library()


def test_null_handles(lib):
    h = ctypes.c_void_p(1)
    assert lib.snn_conv_experts_create(None, 1, ctypes.byref(h)) == 1 and not h.value
    assert lib.snn_conv_experts_create(None, 1, None) == 1
    none = (ctypes.c_void_p * 2)(None, None)
    for count, text in ((0, b"experts"), (1025, b"experts"), (2, b"null handle")):
        assert lib.snn_conv_experts_create(none, count, ctypes.byref(h)) == 1 and text in lib.snn_last_error()
    assert lib.snn_conv_adapters_create(None, ctypes.byref(h)) == 1 and b"null handle" in lib.snn_last_error()
    assert lib.snn_conv_experts_forward(None, None, 1, 0, 8, None, None, 0, None, 0, 8, None) == 1
    assert lib.snn_conv_adapters_forward(None, None, 1, 0, 8, None, None, None, None, 0, 8, None, None, 0, 8, None) == 1
    assert lib.snn_conv_experts_destroy(None) == 0 and lib.snn_conv_adapters_destroy(None) == 0


def _route(lib, **changed):
    a = dict(logits=64, type=0, tokens=4, experts=8, ld=8, top_k=2, normalise=1, ids=64, weights=64, offsets=64, rows=64, slots=64, work=None,
             device=-1)
    a.update(changed)
    return lib.snn_conv_experts_route(a["logits"], a["type"], a["tokens"], a["experts"], a["ld"], a["top_k"], a["normalise"], a["ids"], a["weights"],
                                      a["offsets"], a["rows"], a["slots"], a["work"], a["device"], None)


@pytest.mark.parametrize("changed,text", [
    (dict(type=1), b"logits are"), (dict(type=9), b"logits are"), (dict(experts=0), b"experts"), (dict(experts=1025), b"experts"),
    (dict(top_k=0), b"top_k"), (dict(top_k=9), b"top_k"), (dict(top_k=17, experts=64, ld=64), b"top_k"), (dict(tokens=-1), b"tokens"),
    (dict(tokens=1 << 30), b"tokens"), (dict(ld=7), b"rows of 7"), (dict(logits=None), b"null"), (dict(offsets=None), b"null"), (dict(ids=None), b"null"),
    (dict(tokens=65), b"null workspace"), (dict(logits=66), b"misaligned"), (dict(slots=65), b"misaligned"),
])
def test_route_refuses(lib, changed, text):
    assert _route(lib, **changed) == 1 and text in lib.snn_last_error()


def test_route_workspace(lib):
    assert lib.snn_conv_experts_route_work(64, 128) == 0 and lib.snn_conv_experts_route_work(0, 5) == 0
    assert lib.snn_conv_experts_route_work(65, 128) == 2 * 128 * 4


def _combine(lib, **changed):
    a = dict(y=64, y_type=0, y_rows=4, ld_y=8, slots=64, weights=64, tokens=2, top_k=2, columns=8, out=64, out_type=0, ld_out=8, device=-1)
    a.update(changed)
    return lib.snn_conv_experts_combine(*a.values(), None)


@pytest.mark.parametrize("changed,text", [
    (dict(y_type=1), b"inputs and outputs"), (dict(out_type=2), b"inputs and outputs"), (dict(tokens=-1), b"tokens"), (dict(columns=0), b"columns"),
    (dict(top_k=0), b"top_k"), (dict(top_k=17), b"top_k"), (dict(y_rows=-1), b"y_rows"), (dict(ld_y=7), b"columns"), (dict(ld_out=7), b"columns"),
    (dict(slots=None), b"null"), (dict(out=None), b"null"), (dict(y=None), b"null"), (dict(y=66), b"misaligned"), (dict(weights=66), b"misaligned"),
])
def test_combine_refuses(lib, changed, text):
    assert _combine(lib, **changed) == 1 and text in lib.snn_last_error()


def test_combine_without_tokens_is_nothing(lib):
    assert _combine(lib, tokens=0, slots=None, weights=None, out=None) == 0


def test_no_device_is_a_loud_error(lib):
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    assert _route(lib) == 3 and _combine(lib) == 3 and b"no CPU path" in lib.snn_last_error()


def _experts(cls=snn.SnnConvExperts):
    h = cls.__new__(cls)   # (where torch says that CPU tensors live: device -1; the checks come before the library)
    h._h, h.device, h.count, h.c_in, h.c_out = ctypes.c_void_p(None), -1, 3, 16, 5
    return h


class _Refuses:
    """Stands in for the C library: no call is expected."""

    def __getattr__(self, name):
        if name == "snn_conv_experts_route_work":
            return lambda t, e: 0 if t <= 64 else (t + 63) // 64 * e * 4
        raise AssertionError(f"{name} was called")


@pytest.fixture
def no_library(monkeypatch):
    monkeypatch.setattr(projections, "load_library", lambda: _Refuses())


X = dict(dtype=torch.bfloat16)
I = dict(dtype=torch.int32)


@pytest.mark.parametrize("x,offsets,rows,out,out_type", [
    (torch.zeros(4, 16), torch.zeros(4, **I), None, None, None),                                     # fp32 activations
    (torch.zeros(4, 24, **X), torch.zeros(4, **I), None, None, None),                                # c_in
    (torch.zeros(16, 4, **X).T, torch.zeros(4, **I), None, None, None),                              # rows not dense
    (torch.zeros(4, 20, **X)[:, 4:], torch.zeros(4, **I), None, None, None),                         # rows not 16-byte aligned
    (torch.zeros(1, 16, **X).expand(4, 16), torch.zeros(4, **I), None, None, None),                  # rows that overlap
    (torch.zeros(16, **X), torch.zeros(4, **I), None, None, None),
    (torch.zeros(4, 16, **X), torch.zeros(3, **I), None, None, None),                                # count + 1 offsets
    (torch.zeros(4, 16, **X), torch.zeros(4, dtype=torch.int64), None, None, None),
    (torch.zeros(4, 16, **X), torch.zeros(8, **I)[::2], None, None, None),
    (torch.zeros(4, 16, **X), torch.zeros(4, **I), torch.zeros(2, 2, **I), None, None),
    (torch.zeros(4, 16, **X), torch.zeros(4, **I), torch.zeros(4), None, None),
    (torch.zeros(4, 16, **X), torch.zeros(4, **I), torch.zeros(6, **I), torch.zeros(4, 5, **X), None),   # a row of out for each of rows
    (torch.zeros(4, 16, **X), torch.zeros(4, **I), None, torch.zeros(4, 6, **X), None),
    (torch.zeros(4, 16, **X), torch.zeros(4, **I), None, torch.zeros(4, 5, **I), None),
    (torch.zeros(4, 16, **X), torch.zeros(4, **I), None, torch.zeros(4, 5, **X), snn.OUT_F32),
    (torch.zeros(4, 16, **X), torch.zeros(4, **I), None, torch.zeros(1, 5, **X).expand(4, 5), None),
    (torch.zeros(4, 16, **X), torch.zeros(4, **I), None, None, snn.OUT_I32),
    (torch.zeros(4, 16, **X), torch.zeros(4, **I), None, None, snn.OUT_BITS),
])
def test_experts_refuse(no_library, x, offsets, rows, out, out_type):
    h = _experts()
    with pytest.raises(snn.SnnError) as ei:
        h.forward(x, offsets, rows=rows, out=out, out_type=out_type)
    assert ei.value.status == 1
    h._h = None


@pytest.mark.parametrize("change", [
    dict(a=torch.zeros(2, 8, 16)), dict(a=torch.zeros(2, 8, 24, **X)), dict(b=torch.zeros(2, 5, 16, **X)), dict(b=torch.zeros(3, 5, 8, **X)),
    dict(a=torch.zeros(8, 16, **X)), dict(scale=torch.zeros(3)), dict(scale=torch.zeros(2, **X)), dict(adapter=torch.zeros(3, **I)),
    dict(adapter=torch.zeros(4, dtype=torch.int64)), dict(a=torch.zeros(2, 16, 8, **X).transpose(1, 2)), dict(out=torch.zeros(3, 5, **X)),
])
def test_adapters_refuse(no_library, change):
    h = _experts(snn.SnnConvAdapters)
    args = dict(x=torch.zeros(4, 16, **X), adapter=torch.zeros(4, **I), a=torch.zeros(2, 8, 16, **X), b=torch.zeros(2, 5, 8, **X), scale=torch.zeros(2))
    args.update(change)
    with pytest.raises(snn.SnnError) as ei:
        h.forward(**args)
    assert ei.value.status == 1
    h._h = None


def test_what_is_not_a_layer_or_not_on_a_device(no_library):
    for bad in ([], [None], ["layer"]):
        with pytest.raises(snn.SnnError):
            snn.SnnConvExperts(bad)
    with pytest.raises(snn.SnnError):
        snn.SnnConvAdapters(None)
    with pytest.raises(snn.SnnError):
        snn.route(torch.zeros(2, 4), 1)
    with pytest.raises(snn.SnnError):
        snn.combine(torch.zeros(2, 4), torch.zeros(1, 1, **I), torch.zeros(1, 1))
    for t, e, k in ((-1, 4, 1), (1, 0, 1), (1, 4, 0), (1 << 30, 4, 2)):
        with pytest.raises(snn.SnnError):
            snn.alloc_route(t, e, k, device=-1)

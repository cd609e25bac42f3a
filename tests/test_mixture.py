"""The whole mixture, activations and 8-bit projections where there is no GPU: what the C entry points and the binding refuse."""
import ctypes

import pytest
import torch

import paper_2110_09195_b200 as snn
from paper_2110_09195_b200 import binding, mixture


@pytest.fixture(scope="module")
def lib():
    from paper_2110_09195_b200 import build
    build.build()
    return binding.load_library()


def test_null_handles(lib):
    h = ctypes.c_void_p(1)
    assert lib.snn_conv_moe_create(None, None, None, 2, ctypes.byref(h)) == 1 and not h.value
    assert lib.snn_conv_moe_create(None, None, None, 2, None) == 1
    assert lib.snn_conv_moe_work(None, 1, 1) == -1
    assert lib.snn_conv_moe_forward(None, None, 1, 0, 8, None, 0, 8, 1, 1, None, None, 0, 8, None) == 1 and b"null handle" in lib.snn_last_error()
    assert lib.snn_conv_scaled_forward(None, None, 16, None, 1, None, 0, None, 0, 8, None) == 1 and b"null handle" in lib.snn_last_error()
    assert lib.snn_conv_moe_destroy(None) == 0 and lib.snn_conv_scaled_destroy(None) == 0


def _scaled(lib, **changed):
    a = dict(weights=64, scales=64, count=2, c_in=64, c_out=8, device=-1, stream=None)
    a.update(changed)
    h = ctypes.c_void_p(1)
    st = lib.snn_conv_scaled_create(*a.values(), ctypes.byref(h))
    assert not h.value
    return st


@pytest.mark.parametrize("changed,text", [
    (dict(weights=None), b"null"), (dict(scales=None), b"null"), (dict(count=0), b"projections"), (dict(count=1025), b"projections"), (dict(c_in=0), b"c_in"),
    (dict(c_in=24), b"c_in"), (dict(c_out=0), b"c_out"), (dict(weights=72), b"misaligned"), (dict(scales=66), b"misaligned"),
])
def test_scaled_create_refuses(lib, changed, text):
    assert _scaled(lib, **changed) == 1 and text in lib.snn_last_error()


def _activate(lib, **changed):
    a = dict(gate=64, ld_gate=8, up=64, ld_up=8, type=0, rows=2, columns=8, fn=2, out=64, out_type=0, ld_out=8, device=-1)
    a.update(changed)
    return lib.snn_conv_experts_activate(*a.values(), None)


@pytest.mark.parametrize("changed,text", [
    (dict(type=1), b"inputs are"), (dict(out_type=2), b"outputs are"), (dict(fn=-1), b"fn"), (dict(fn=4), b"fn"), (dict(rows=-1), b"rows"), (dict(columns=0), b"columns"),
    (dict(ld_up=7), b"columns"), (dict(ld_gate=7), b"columns"), (dict(ld_out=7), b"columns"), (dict(up=None), b"null"), (dict(out=None), b"null"), (dict(up=66), b"misaligned"),
    (dict(gate=66), b"misaligned"), (dict(out=66), b"misaligned"),
])
def test_activate_refuses(lib, changed, text):
    assert _activate(lib, **changed) == 1 and text in lib.snn_last_error()


def _quantise(lib, **changed):
    a = dict(gate=None, ld_gate=0, up=64, ld_up=200, type=0, in_rows=2, rows=None, out_rows=2, columns=200, fn=0, values=64, ld_values=200, scales=64, ld_scales=2, device=-1)
    a.update(changed)
    return lib.snn_conv_scaled_quantise(*a.values(), None)


@pytest.mark.parametrize("changed,text", [
    (dict(type=2), b"inputs are"), (dict(fn=4), b"fn"), (dict(in_rows=-1), b"rows"), (dict(columns=0), b"columns"), (dict(ld_up=199), b"columns"),
    (dict(gate=64, ld_gate=9), b"columns"), (dict(out_rows=3), b"without an index"), (dict(out_rows=-1, rows=64), b"rows"), (dict(ld_values=199), b"columns"),
    (dict(ld_scales=1), b"columns"), (dict(up=None), b"null"), (dict(values=None), b"null"), (dict(scales=None), b"null"), (dict(up=66), b"misaligned"),
    (dict(rows=66), b"misaligned"), (dict(scales=66), b"misaligned"),
])
def test_quantise_refuses(lib, changed, text):
    assert _quantise(lib, **changed) == 1 and text in lib.snn_last_error()


def test_no_rows_are_nothing(lib):
    assert _activate(lib, rows=0, up=None, gate=None, out=None) == 0
    assert _quantise(lib, in_rows=0, out_rows=0, up=None, values=None, scales=None) == 0


def test_no_device_is_a_loud_error(lib):
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    assert _scaled(lib) == 3 and _activate(lib) == 3 and _quantise(lib) == 3 and b"no CPU path" in lib.snn_last_error()


class _Refuses:
    """Stands in for the C library: no call is expected."""

    def __getattr__(self, name):
        raise AssertionError(f"{name} was called")


@pytest.fixture
def no_library(monkeypatch):
    monkeypatch.setattr(mixture, "load_library", lambda: _Refuses())


X = dict(dtype=torch.bfloat16)
I = dict(dtype=torch.int32)


def _q(*shape):
    return torch.zeros(*shape).to(torch.float8_e4m3fn)


def _bare(cls, **fields):
    h = cls.__new__(cls)   # (where torch says that CPU tensors live: device -1; the checks come before the library)
    h._h, h.device = ctypes.c_void_p(None), -1
    for k, v in fields.items():
        setattr(h, k, v)
    return h


@pytest.mark.parametrize("change", [
    dict(x=torch.zeros(4, 144)), dict(x=_q(4, 160)), dict(x=_q(144, 4).T), dict(x=_q(4, 152)[:, :144]), dict(x=_q(4, 176)[:, 8:152]), dict(x=_q(1, 144).expand(4, 144)),
    dict(x=_q(144)), dict(scales=torch.zeros(4, 3)), dict(scales=torch.zeros(5, 2)), dict(scales=torch.zeros(4, 2, **X)), dict(scales=torch.zeros(2, 4).T),
    dict(offsets=torch.zeros(3, **I)), dict(offsets=torch.zeros(4, dtype=torch.int64)), dict(offsets=torch.zeros(8, **I)[::2]), dict(out=torch.zeros(4, 6)),
    dict(out=torch.zeros(3, 5)), dict(out=torch.zeros(4, 5, **I)), dict(out=torch.zeros(4, 5), out_type=snn.OUT_BF16), dict(out_type=snn.OUT_BITS),
    dict(scales=torch._neg_view(torch.zeros(4, 2))), dict(out=torch._neg_view(torch.zeros(4, 5))),
])
def test_scaled_refuses(no_library, change):
    h = _bare(snn.SnnConvScaled, count=3, c_in=144, c_out=5)
    args = dict(x=_q(4, 144), scales=torch.zeros(4, 2), offsets=torch.zeros(4, **I))
    args.update(change)
    with pytest.raises(snn.SnnError) as ei:
        h.forward(**args)
    assert ei.value.status == 1
    h._h = None


@pytest.mark.parametrize("change", [
    dict(x=torch.zeros(4, 16)), dict(x=torch.zeros(4, 24, **X)), dict(x=torch.zeros(4, 20, **X)[:, 4:]), dict(logits=torch.zeros(4, 4)), dict(logits=torch.zeros(5, 3)),
    dict(logits=torch.zeros(4, 3, **I)), dict(logits=torch.zeros(3, 4).T), dict(logits=torch._neg_view(torch.zeros(4, 3))),
])
def test_moe_refuses(no_library, change):
    h = _bare(snn.SnnConvMoe, count=3, c_in=16, hidden=8, c_out=5, _experts=())
    args = dict(x=torch.zeros(4, 16, **X), logits=torch.zeros(4, 3), top_k=2)
    args.update(change)
    with pytest.raises(snn.SnnError) as ei:
        h.forward(**args)
    assert ei.value.status == 1
    h._h = None


def test_what_is_not_on_a_device_or_no_handle(no_library):
    for call in (lambda: snn.activate(torch.zeros(2, 4)), lambda: snn.quantise(torch.zeros(2, 4)), lambda: snn.SnnConvScaled(_q(4, 16), torch.zeros(1, 1)),
                 lambda: snn.SnnConvMoe(None, None), lambda: snn.SnnConvMoe("up", "down"), lambda: snn.alloc_quantised(-1, 4), lambda: snn.alloc_quantised(1, 0)):
        with pytest.raises(snn.SnnError) as ei:
            call()
        assert ei.value.status == 1

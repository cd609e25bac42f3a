"""SiLU and GELU over all fp32 numbers for which they are normal ones, and down to where they end, against 64 bits."""
import pytest
import torch

from test_gpu_moe_sums import _layer
from test_gpu_projections import BF16, F16, F32, _gen, snn  # noqa: F401
from test_gpu_scaled import _fn64

pytestmark = pytest.mark.gpu

NORMAL = torch.finfo(F32).smallest_normal


def _every(low, high, step):
    """Every `step`-th fp32 number between two of one sign."""
    a, b = (torch.tensor([v], dtype=F32).view(torch.int32).item() for v in (low, high))
    return torch.arange(min(a, b), max(a, b), step, dtype=torch.int32, device="cuda").view(F32)


def _inputs():
    """From 2^-126 to 3.38e38, some 4 million of either sign; and closely where the results come to their end."""
    return torch.cat([_every(NORMAL, 3.38e38, 509), _every(-NORMAL, -3.38e38, 509), _every(-80.0, -95.0, 3), _every(-5.0, -14.0, 7)])[None]


@pytest.mark.parametrize("fn", ["FN_SILU", "FN_GELU"])
@pytest.mark.parametrize("out", [F32, BF16, F16])
def test_every_binade(snn, fn, out):  # noqa: F811
    """SiLU: the exponential within 2 steps of the approximation by the device (2^-22) and two roundings of the factor behind it; 1 + it, its reciprocal within a step, and the product:
    2^-20.5.  GELU: 2^-20.4 for the distribution's function, as fitted, and a rounding.  Where the result is not a normal number, a step of the smallest ones, and what is below
    the smallest normal one in the function may be lost before it is multiplied by the value: 14 times that."""
    v = _inputs()
    want = _fn64(fn, v.double())
    got = snn.activate(v, fn=getattr(snn, fn), out=torch.empty(v.shape, dtype=out, device="cuda")).double()
    low = 14 * 2.0 ** -149 if out != F16 else torch.finfo(F16).smallest_normal * 2.0 ** -11
    ok = (got - want).abs() <= (2.0 ** -20 + torch.finfo(out).eps / 2) * want.abs() + low
    if out == BF16:   # (its numbers below the smallest normal one are further apart)
        ok |= (got - want).abs() <= 2.0 ** -134
    if fn == "FN_GELU":
        ok |= (want.abs() < NORMAL) & ((got - want).abs() <= NORMAL)
    if out == F16:
        ok |= (want > 65519.9) & torch.isinf(got)
    assert ok.all(), (v[~ok][:8], got[~ok][:8], want[~ok][:8])


@pytest.mark.parametrize("C", [256, 77])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_far_values_behind_a_gate(snn, C, dtype):  # noqa: F811
    """Small factors times large ones: numbers of a usual size.  (2^-20 as above, a rounding of the product, half a step of the 8-bit value.)"""
    g = _gen(C)
    gate = (-80 - 11 * torch.rand(5, C, generator=g, device="cuda")).to(dtype)
    up = (2.0 ** 120 * (1 + torch.rand(5, C, generator=g, device="cuda"))).to(dtype)
    want = _fn64("FN_SILU", gate.double()) * up.double()
    got = snn.activate(up, gate=gate, fn=snn.FN_SILU, out_type=snn.OUT_F32).double()
    assert (want != 0).all() and ((got - want).abs() <= (2.0 ** -20 + 2.0 ** -23) * want.abs()).all()
    values, scales = snn.quantise(up, gate=gate, fn=snn.FN_SILU)
    wide = scales.double().repeat_interleave(128, 1)[:, :C]
    assert ((values.double() * wide - want).abs() <= (2.0 ** -4 + 2.0 ** -19) * want.abs() + 2.0 ** -10 * wide).all()


@pytest.mark.parametrize("T", [1, 9])
def test_far_values_in_a_mixture(snn, T):  # noqa: F811
    x = torch.zeros(T, 16, dtype=BF16, device="cuda")
    x[:, 3] = 1.0
    gate, _ = _layer(snn, 16, 40, 600, lambda w: -90 * w[:, 3])
    up, _ = _layer(snn, 16, 40, 601, lambda w: 2.0 ** 100 * w[:, 3])
    down, w = _layer(snn, 40, 24, 602, lambda w: torch.ones(24))
    y = snn.SnnConvMoe(up, down, gate=gate, fn=snn.FN_SILU).forward(x, torch.zeros(T, 1, device="cuda"), 1, out_type=snn.OUT_F32)
    h = _fn64("FN_SILU", torch.tensor(-90.0, dtype=torch.float64)).item() * 2.0 ** 100
    # (one value 40 times: a sum of 40, off by 40 cut additions of 2^-23 of 40 values)
    assert ((y.double() - h * w.sum(1)).abs() <= 2.0 ** -19 * abs(h) * w.sum(1).abs() + 40 * 2.0 ** -23 * 40 * abs(h)).all()

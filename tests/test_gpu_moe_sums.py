"""What the whole mixture keeps of its sums, and of the values between its projections: all 24 bits, whatever the outputs' type.

One-hot activations and a scale of its own for each channel put chosen numbers between the projections, so that an output has one correct value, or
one that fp32 sums miss by a number of roundings that is counted."""
import numpy as np
import pytest
import torch

import workloads as wl
from test_gpu_projections import BF16, F16, F32, _decode, _gen, snn  # noqa: F401

pytestmark = pytest.mark.gpu


def _layer(snn, c_in, c_out, seed, alpha=None):
    """Experts of one layer and its decoded weights [c_out, c_in] in 64 bits; alpha: a function of the weights."""
    p = wl.draw_layer_params(wl.LayerShape(c_in, c_out, 1, 1, 1, 0, 1), 5, seed)
    w = _decode(p, c_in, c_out)
    a = np.ones(c_out, np.float32) if alpha is None else alpha(w).float().cpu().numpy()
    layer = snn.SnnConv(c_in, c_out, 5, p.codebook, p.idx_packed, a, pad=0, ksize=1, act_type=snn.ACT_F16)
    experts = snn.SnnConvExperts([layer])
    layer.destroy()
    return experts, w


@pytest.mark.parametrize("fn,gated", [("FN_SILU", True), ("FN_GELU", False)])
@pytest.mark.parametrize("T,E,k,c_in,hidden,c_out", [(1, 8, 2, 1024, 1024, 4096), (6, 12, 3, 328, 1000, 3003), (40, 16, 4, 512, 520, 2048)])
@pytest.mark.parametrize("act", [BF16, F16])
def test_outputs_of_16_bits_are_the_rounded_ones_of_32(snn, fn, gated, T, E, k, c_in, hidden, c_out, act):  # noqa: F811
    """The same sums and one rounding.  (With 16 bits of the values between the projections about one output in a thousand was another.)"""
    def experts(a, b, seed):
        layers = []
        for e in range(E):
            p = wl.draw_layer_params(wl.LayerShape(a, b, 1, 1, 1, 0, 1), 5, seed + e)
            layers.append(snn.SnnConv(a, b, 5, p.codebook, p.idx_packed, p.alpha, pad=0, ksize=1, act_type=snn.ACT_F16))
        return snn.SnnConvExperts(layers)
    up, down = experts(c_in, hidden, 10), experts(hidden, c_out, 200)
    h = snn.SnnConvMoe(up, down, gate=experts(c_in, hidden, 400) if gated else None, fn=getattr(snn, fn))
    g = _gen(T)
    x, logits = torch.randn(T, c_in, generator=g, device="cuda").to(act), torch.randn(T, E, generator=g, device="cuda")
    y = h.forward(x, logits, k, out_type=snn.OUT_F32)
    for dtype, out_type in ((BF16, snn.OUT_BF16), (F16, snn.OUT_F16)):
        assert torch.equal(h.forward(x, logits, k, out_type=out_type), y.to(dtype))


def _bf16_parts(v, n):
    """What n bf16 numbers hold of an fp32 value: 8 bits at a time."""
    rest = v.clone()
    for i in range(n):
        rest = rest - (rest.view(torch.int32) & -65536).view(F32)
    return v - rest


@pytest.mark.parametrize("T", [1, 5, 8, 21])
@pytest.mark.parametrize("hidden", [8, 40, 264, 1000, 2048])
@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("act,out", [(BF16, F32), (F16, F32), (BF16, BF16), (F16, F16)])
def test_the_third_part(snn, T, hidden, gated, act, out):  # noqa: F811
    """Eight values between the projections, odd whole numbers below 2^20 (for fp16 outputs, which end at 65504, over 2^12): every sum of them and of their parts is exact."""
    g = _gen(T + hidden)
    values = torch.zeros(hidden, dtype=torch.float64, device="cuda")
    at = torch.randperm(hidden, generator=g, device="cuda")[:8]
    values[at] = (2 * torch.randint(1 << 16, 1 << 19, (8,), generator=g, device="cuda") + 1).double() * (2.0 ** -12 if out == F16 else 1.0)
    assert (_bf16_parts(values.float(), 2) != values.float()).any() and torch.equal(_bf16_parts(values.float(), 3), values.float())
    up, w_up = _layer(snn, 72, hidden, 500, lambda w: values)
    gate, w_gate = _layer(snn, 72, hidden, 501)
    down, w_down = _layer(snn, hidden, 75, 502)
    h = snn.SnnConvMoe(up, down, gate=gate if gated else None, fn=snn.FN_NONE)
    x = torch.zeros(T, 72, dtype=torch.float64, device="cuda")
    x[torch.arange(T), torch.randint(72, (T,), generator=g, device="cuda")] = 1.0
    between = x @ w_up.T * values
    if gated:
        between = between * (x @ w_gate.T)
    y = h.forward(x.to(act), torch.zeros(T, 1, device="cuda"), 1, out=torch.empty(T, 75, dtype=out, device="cuda"))
    assert torch.equal(y, (between @ w_down.T).float().to(out))


@pytest.mark.parametrize("T", [1, 8, 9])
@pytest.mark.parametrize("hidden", [256, 512])
def test_sums_of_the_lower_parts(snn, T, hidden):  # noqa: F811
    """256 times 65536 + 255.9921875.  The upper 8 bits add up to 2^24 and the lower ones to 65534, both exactly; so is their sum, 16842750, and twice that.  (In one sum that the matrix instructions cut,
    what is below 2 would be lost as soon as 2^24 is near.)"""
    value = 65536 + 255.9921875
    down, w_down = _layer(snn, hidden, 8, 510)
    up, w_up = _layer(snn, 16, hidden, 511, lambda w: value * w_down[0] * w[:, 5])
    x = torch.zeros(T, 16, dtype=BF16, device="cuda")
    x[:, 5] = 1.0
    y = snn.SnnConvMoe(up, down, fn=snn.FN_NONE).forward(x, torch.zeros(T, 1, device="cuda"), 1, out_type=snn.OUT_F32)
    assert value * hidden == 16842750 * (hidden // 256) and (y[:, 0] == value * hidden).all()


@pytest.mark.parametrize("T", [1, 7, 12])
@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("act,unit", [(BF16, 1.0), (F16, 2.0 ** -9)])
def test_long_sums_are_rounded_and_not_cut(snn, T, gated, act, unit):  # noqa: F811
    """32768 channels, in 128 blocks of 256 one of which is not zero; the eight warps that share them have every eighth block.  First 2^24 or, every second warp,
    -2^24, then 15 times 1.5 where it was 2^24: 90 in all.  Rounded to nearest, 2^24 + 1.5 misses by half of 2 at most, 60 times, and adding up the warps' sums, none
    above 2^24 + 32, seven times: 67.  Cut, the 1.5 are lost: 90.  With a gate it is the same projection: the square, and its rounding."""
    up, w = _layer(snn, 32768, 8, 520, lambda w: torch.tensor([1.0] + [0.0] * 7))
    down, w_down = _layer(snn, 8, 40, 521)
    v = torch.zeros(32768, dtype=torch.float64, device="cuda")
    for b in range(128):
        v[256 * b + 37 * b % 256] = (2.0 ** 24 if b < 8 else 1.5) * (1.0 if b % 2 == 0 else -1.0 if b < 8 else 0.0)
    assert v.sum() == 90
    x = (v * w[0] * unit).to(act).expand(T, -1).contiguous()
    h = snn.SnnConvMoe(up, down, gate=up if gated else None, fn=snn.FN_NONE)
    y = h.forward(x, torch.zeros(T, 1, device="cuda"), 1, out_type=snn.OUT_F32).double() / w_down[:, 0] / unit
    if gated:
        y = torch.sqrt(y / unit)
    assert ((y - 90).abs() <= 67 + 2.0 ** -22 * 200).all()

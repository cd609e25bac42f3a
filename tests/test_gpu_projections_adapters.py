"""Adapters of many rows: as many different ones in a tile as are added by the matrix instructions, and more; ranks of which several share a
pass; rows that change adapter inside a tile; factors with infinities and NaN beside rows that do not use them."""
import pytest
import torch

import test_gpu_projections as one
from test_gpu_projections import BF16, F16, F32, _gen, _layers, _whole, snn  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def many(monkeypatch):
    monkeypatch.setenv("SNN_FORCE_ROWS", "many")


@pytest.mark.parametrize("rank", [8, 16, 24, 40])
@pytest.mark.parametrize("n,run", [(2, 1), (3, 33), (17, 1), (47, 2), (60, 1), (400, 1), (9, 97)])
def test_numbers_of_adapters(snn, rank, n, run):
    one.test_adapters_whole_numbers(snn, 430, 264, 300, 5, n, rank, run, BF16, F32)


@pytest.mark.parametrize("R", [300, 1000, 2500])
@pytest.mark.parametrize("rank", [8, 32, 72, 128])
@pytest.mark.parametrize("run", [1, 13, 100])
def test_numbers_of_rows(snn, R, rank, run):
    one.test_adapters_whole_numbers(snn, R, 520, 270, 5, 11, rank, run, F16, BF16)


@pytest.mark.parametrize("rank", [8, 16, 48])
@pytest.mark.parametrize("n", [5, 70])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_second_factor_with_infinities(snn, rank, n, bad):
    """Adapter 1 has a bad value in channel 3 of B (its other channels are fine), adapter 2's A x is infinite in some rows; all in turn."""
    R, c_in, c_out = 300, 128, 140
    g = _gen(50)
    layers, w, _ = _layers(snn, 1, c_in, c_out, 5, 2000, alpha=0.5)
    ad = snn.SnnConvAdapters(layers[0])
    x = _whole(g, 2, R, c_in).to(BF16)
    a, b = _whole(g, 1, n, rank, c_in).to(BF16), _whole(g, 1, n, c_out, rank).to(BF16)
    b[1, 3, rank - 1] = bad
    a[2, 0, 0] = float("inf")
    a[2, :, 1:] = 0
    x[:, 0] = 1
    adapter = (torch.arange(R, device="cuda") % (n + 1)).to(torch.int32)
    scale = torch.full((n,), 0.5, device="cuda")
    y = ad.forward(x, adapter, a, b, scale, out_type=snn.OUT_F32)
    ref = 0.5 * (x.double() @ w[0].T)
    for i in range(n):
        m = adapter == i
        h = 0.5 * (x[m].double() @ a[i].double().T)
        ref[m] += torch.where(torch.isfinite(b[i].double()), b[i].double(), 0.0).matmul(h.nan_to_num(posinf=0, neginf=0, nan=0).T).T
    bad_row, inf_row = adapter == 1, adapter == 2
    fine = ~(bad_row | inf_row)
    assert torch.equal(y[fine], ref[fine].float())
    keep = torch.arange(c_out, device="cuda") != 3
    assert torch.equal(y[bad_row][:, keep], ref[bad_row][:, keep].float())
    hb = x[bad_row].double() @ a[1].double().T
    assert torch.equal(torch.isfinite(y[bad_row][:, 3]), torch.zeros_like(y[bad_row][:, 3], dtype=torch.bool))
    if bad == float("inf"):   # (its sign is that of A x; 0 times infinity is NaN)
        last = hb[:, rank - 1]
        assert torch.equal(torch.isnan(y[bad_row][:, 3]), last == 0)
        assert (torch.sign(y[bad_row][:, 3])[last != 0] == torch.sign(last)[last != 0]).all()
    # A x = (infinity, then x_0 * 0 and such): infinite or NaN wherever B's first value says so
    assert not torch.isfinite(y[inf_row]).any()


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_second_factor_with_infinities_beside_more_adapters_than_passes(snn, bad):
    test_second_factor_with_infinities(snn, 16, 150, bad)


@pytest.mark.parametrize("rank", [8, 16, 40])
@pytest.mark.parametrize("n", [71, 72, 73, 74])
def test_as_many_adapters_as_passes_are_made_for(snn, rank, n):
    """192 rows, a tile, with n adapters in turn: exactly n different ones."""
    c_in, c_out, R = 128, 130, 192
    g = _gen(60 + n)
    layers, w, _ = _layers(snn, 1, c_in, c_out, 5, 2100, alpha=0.5)
    x = _whole(g, 2, R, c_in).to(F16)
    a, b = _whole(g, 1, n, rank, c_in).to(F16), _whole(g, 1, n, c_out, rank).to(F16)
    adapter = (torch.arange(R, device="cuda") % n).to(torch.int32)
    y = snn.SnnConvAdapters(layers[0]).forward(x, adapter, a, b, torch.ones(n, device="cuda"), out_type=snn.OUT_F32)
    h = torch.einsum("rc,rjc->rj", x.double(), a.double()[adapter.long()])
    ref = 0.5 * (x.double() @ w[0].T) + torch.einsum("rj,rkj->rk", h, b.double()[adapter.long()])
    assert torch.equal(y, ref.float())

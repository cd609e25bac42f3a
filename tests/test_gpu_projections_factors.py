"""What adapters' two factors hold: infinities and NaN in both at once, by both kernels."""
import pytest
import torch

from test_gpu_projections import BF16, F16, _gen, _layers, _whole, snn  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["few", "many"])
def rows(request, monkeypatch):
    monkeypatch.setenv("SNN_FORCE_ROWS", request.param)
    return request.param


@pytest.mark.parametrize("act", [F16, BF16])
@pytest.mark.parametrize("n", [3, 50, 150])   # (150 in turn: more in a tile than the matrix instructions add)
@pytest.mark.parametrize("rank", [8, 16, 24, 40])
def test_infinities_in_both_factors(snn, rows, rank, n, act):
    """Adapter 1: A x is infinite, or NaN, at one place of the rank, and B there is finite, 0, an infinity or NaN by the channel.  Every output is the
    formula's: B h summed in 64 bits, whole numbers elsewhere, so that there is one right value and one right infinity for each."""
    R, c_in, c_out, at = 330, 128, 140, rank - 3
    g = _gen(70 + rank + n)
    layers, w, _ = _layers(snn, 1, c_in, c_out, 5, 2200, alpha=0.5)
    ad = snn.SnnConvAdapters(layers[0])
    x = _whole(g, 2, R, c_in).to(act)
    x[:, 0] = (torch.arange(R, device="cuda") % 3 - 1).to(act)   # (-1, 0, 1: A x is -infinity, NaN, infinity)
    a, b = _whole(g, 1, n, rank, c_in).to(act), _whole(g, 1, n, c_out, rank).to(act)
    a[1, at, 0] = float("inf")
    inf = float("inf")
    for channel, value in ((0, inf), (1, -inf), (2, float("nan")), (3, 0.0), (64, inf), (130, -inf), (139, inf)):
        b[1, channel, at] = value
    b[1, 5, 0], b[1, 6, 0] = inf, -inf      # (where A x is finite: there are two places that are not, of one sign or of both)
    b[1, 6, at] = 1.0
    adapter = (torch.arange(R, device="cuda") // 2 % (n + 1)).to(torch.int32)
    y = ad.forward(x, adapter, a, b, torch.ones(n, device="cuda"), out_type=snn.OUT_F32)
    ref = 0.5 * (x.double() @ w[0].T)
    for i in range(n):
        m = adapter == i
        h = (x[m].double()[:, None, :] * a[i].double()).sum(2)
        ref[m] += (h[:, None, :] * b[i].double()).sum(2)
    own = adapter == 1
    assert torch.isposinf(ref[own]).any() and torch.isneginf(ref[own]).any() and torch.isnan(ref[own]).any()
    assert torch.isfinite(ref[~own]).all()
    assert torch.equal(torch.isnan(y), torch.isnan(ref))
    assert torch.equal(y.nan_to_num(nan=7.5, posinf=inf, neginf=-inf), ref.float().nan_to_num(nan=7.5, posinf=inf, neginf=-inf))

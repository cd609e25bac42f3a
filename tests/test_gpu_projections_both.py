"""Both kernels of the projections, the one for few rows and the one for many, at sizes where the library would take the other:
the cases of test_gpu_projections with the choice taken from it (SNN_FORCE_ROWS), and larger ones that reach several tiles, waves and
adapters of every bound of the rank."""
import numpy as np
import pytest
import torch

import test_gpu_projections as one
from test_gpu_projections import BF16, F16, F32, _bound, _gen, _layers, _whole, snn  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["few", "many"])
def rows(request, monkeypatch):
    monkeypatch.setenv("SNN_FORCE_ROWS", request.param)
    return request.param


@pytest.mark.parametrize("act,out", [(F16, F16), (BF16, F32), (BF16, F16)])
@pytest.mark.parametrize("c_in,c_out,tau,sizes", one.EXPERT_CASES)
def test_experts(snn, rows, c_in, c_out, tau, sizes, act, out):
    one.test_experts_whole_numbers(snn, c_in, c_out, tau, sizes, act, out)


@pytest.mark.parametrize("n_tok,sizes", [(5, [3, 0, 4, 1]), (300, [300, 512, 0, 290])])
def test_gathered(snn, rows, n_tok, sizes):
    one.test_experts_gathered_rows_with_strides(snn, n_tok, sizes, BF16)


def test_edges(snn, rows):
    one.test_experts_offsets_outside_the_rows(snn)
    one.test_experts_infinities_and_nan_stay_in_their_rows(snn, 5)
    one.test_experts_infinities_and_nan_stay_in_their_rows(snn, 200)
    one.test_experts_fp16_overflow_is_an_infinity(snn)
    one.test_experts_many(snn)
    one.test_experts_without_rows(snn)
    one.test_adapters_infinities_stay_in_their_rows(snn)
    one.test_adapters_without_rows_or_adapters(snn)


@pytest.mark.parametrize("act,out", [(F16, F32), (BF16, BF16)])
@pytest.mark.parametrize("case", one.ADAPTER_CASES)
def test_adapters(snn, rows, case, act, out):
    one.test_adapters_whole_numbers(snn, *case, act, out)


def test_normal_values(snn, rows):
    one.test_experts_normal_values(snn, 1000, 77, [1, 0, 12], F16)
    one.test_experts_normal_values(snn, 2048, 1024, [700, 1100], BF16)
    one.test_adapters_normal_values(snn, 40, 1024, 512, 16, 32, 1, F16)
    one.test_adapters_normal_values(snn, 600, 2048, 256, 3, 64, 250, BF16)


@pytest.mark.parametrize("c_in,c_out,sizes", [
    (64, 1300, [4000, 3, 0, 193]),         # one block of input channels, several waves of tiles
    (136, 2048, [385, 0, 0, 1, 1536]),     # three blocks: the two warpgroups of the weights have different numbers of them
    (1096, 1003, [1021, 33, 2000]),
    (2056, 257, [192, 191, 97, 96, 32, 31]),
])
@pytest.mark.parametrize("gather", [False, True])
def test_many_rows(snn, c_in, c_out, sizes, gather):
    g = _gen(c_in)
    layers, w, al = _layers(snn, len(sizes), c_in, c_out, 5, 1400)
    ex = snn.SnnConvExperts(layers)
    R = sum(sizes)
    x = _whole(g, 4, 777 if gather else R, c_in).to(BF16)
    rows = torch.randint(-1, 778, (R,), generator=g, device="cuda", dtype=torch.int32) if gather else None
    xr = x.double()
    if gather:   # (-1 and 777: rows of zeros)
        xr = torch.cat([xr, torch.zeros(2, c_in, dtype=torch.float64, device="cuda")])[rows.long()]
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32, device="cuda")
    y = ex.forward(x, offsets, rows=rows, out_type=snn.OUT_F32)
    lo = 0
    for e, n in enumerate(sizes):
        assert torch.equal(y[lo:lo + n], (xr[lo:lo + n] @ w[e].T).float() * al[e])
        lo += n


def test_many_rows_of_which_none_or_few_are_used(snn):
    """The number of rows is a bound: what the experts do not have is left alone, and no work is not an endless wait."""
    layers, w, al = _layers(snn, 3, 1024, 2048, 5, 1500)
    ex = snn.SnnConvExperts(layers)
    x = _whole(_gen(9), 4, 4000, 1024).to(F16)
    out = torch.full((4000, 2048), 7.0, dtype=F16, device="cuda")
    for offsets in ([0, 0, 0, 0], [4000] * 4, [123] * 4):
        ex.forward(x, torch.tensor(offsets, dtype=torch.int32, device="cuda"), out=out)
    assert (out == 7).all()
    ex.forward(x, torch.tensor([2000, 2000, 2001, 2005], dtype=torch.int32, device="cuda"), out=out)
    assert (out[:2000] == 7).all() and (out[2005:] == 7).all()
    assert torch.equal(out[2000], ((x[2000].double() @ w[1].T).float() * al[1]).to(F16))
    assert torch.equal(out[2001:2005], ((x[2001:2005].double() @ w[2].T).float() * al[2]).to(F16))


@pytest.mark.parametrize("rank", [8, 16, 24, 32, 64, 72, 128])
@pytest.mark.parametrize("run", [1, 5, 600])
def test_many_rows_with_adapters(snn, monkeypatch, rank, run):
    monkeypatch.setenv("SNN_FORCE_ROWS", "many")
    one.test_adapters_whole_numbers(snn, 1111, 520, 1027, 5, 6, rank, run, BF16, BF16)
    one.test_adapters_whole_numbers(snn, 401, 264, 300, 5, 6, rank, run, F16, F32)


def test_rows_and_outputs_that_no_vector_fits(snn, rows):
    """Rows of outputs at odd distances, from an odd element on, with and without adapters."""
    R, c_in, c_out, n, rank = 230, 256, 203, 2, 16
    g = _gen(5)
    layers, w, _ = _layers(snn, 1, c_in, c_out, 5, 1600, alpha=0.5)
    x = _whole(g, 4, R, c_in).to(F16)
    a, b = _whole(g, 1, n, rank, c_in).to(F16), _whole(g, 1, n, c_out, rank).to(F16)
    adapter = (torch.arange(R, device="cuda") // 100 % 3).to(torch.int32)
    ref = 0.5 * (x.double() @ w[0].T)
    low = torch.zeros_like(ref)
    for i in range(n):
        low[adapter == i] = (x[adapter == i].double() @ a[i].double().T) @ b[i].double().T
    buffer = torch.full((R * 211 + 1,), 3.0, dtype=F16, device="cuda")
    out = buffer[1:].reshape(R, 211)[:, 2:2 + c_out]
    snn.SnnConvExperts(layers).forward(x, torch.tensor([0, R], dtype=torch.int32, device="cuda"), out=out)
    assert torch.equal(out, ref.float().to(F16))
    snn.SnnConvAdapters(layers[0]).forward(x, adapter, a, b, torch.ones(n, device="cuda"), out=out)
    assert torch.equal(out, (ref + low).float().to(F16))
    assert (buffer[1:].reshape(R, 211)[:, :2] == 3).all() and (buffer[1:].reshape(R, 211)[:, 2 + c_out:] == 3).all() and buffer[0] == 3


def test_calls_among_the_layers_kernels(snn):
    """One stream, no waits between: layers, a group, experts and adapters launched one behind the other give what each gives alone (their launches
    overlap, and both tensor-core kernels take all of the tensor memory)."""
    import workloads as wl
    shape = wl.LayerShape(64, 64, 14, 14, 1, 1)
    p = wl.draw_layer_params(shape, 5, 77)
    conv = snn.SnnConv(64, 64, 5, p.codebook, p.idx_packed, p.alpha)
    act = torch.from_numpy(wl.pack_activation_bits(wl.draw_activation_bits(shape, 4, 77)).view(np.int32)).cuda()
    layers, _, _ = _layers(snn, 2, 512, 1024, 5, 1700)
    ex, ad = snn.SnnConvExperts(layers), snn.SnnConvAdapters(layers[0])
    g = _gen(6)
    x = torch.randn(2500, 512, generator=g, device="cuda").to(BF16)
    offsets = torch.tensor([0, 1200, 2500], dtype=torch.int32, device="cuda")
    a, b = torch.randn(3, 32, 512, generator=g, device="cuda").to(BF16), torch.randn(3, 1024, 32, generator=g, device="cuda").to(BF16)
    adapter, scale = (torch.arange(2500, device="cuda") // 400 % 4).to(torch.int32), torch.rand(3, generator=g, device="cuda")
    calls = [lambda: conv.forward(act), lambda: ex.forward(x, offsets), lambda: ad.forward(x, adapter, a, b, scale),
             lambda: conv.forward(act, out_type=snn.OUT_I32), lambda: ex.forward(x[:9], torch.tensor([0, 4, 9], dtype=torch.int32, device="cuda")),
             lambda: ad.forward(x[:9], adapter[:9], a, b, scale), lambda: snn.route(x[:, :64].contiguous(), 4).rows]
    alone = []
    for c in calls:
        alone.append(c())
        torch.cuda.synchronize()
    for _ in range(5):
        got = [c() for c in calls + calls[::-1]]
        torch.cuda.synchronize()
        for y, ref in zip(got, alone + alone[::-1]):
            assert torch.equal(y, ref)

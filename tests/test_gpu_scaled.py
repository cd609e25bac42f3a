"""Projections in 8-bit floating point with a scale for each block of 128, and the rows in that form, against plain arithmetic in
64 bits.

Whole numbers with scales that are powers of two: every partial sum is exact in fp32, so the outputs have one correct value each and are
compared bit by bit.  Normal values: the tolerance of an output is derived in _bound."""
import numpy as np
import pytest
import torch

from test_gpu_projections import BF16, F16, F32, _gen, snn  # noqa: F401

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn


@pytest.fixture(params=["few", "many"])
def kernel(request, monkeypatch):
    monkeypatch.setenv("SNN_FORCE_ROWS", request.param)
    return request.param


def _offsets(sizes, lead=0):
    return torch.tensor(lead + np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32, device="cuda")


def _whole8(g, *shape):
    return torch.randint(-4, 5, shape, generator=g, device="cuda").float().to(E4M3)


def _powers(g, low, high, *shape):
    return torch.exp2(torch.randint(low, high + 1, shape, generator=g, device="cuda").float())


def _wide(scales, columns):
    return scales.double().repeat_interleave(128, -1)[..., :columns]


def _reference(x, xs, w, ws):
    """In 64 bits, and the sum of the magnitudes; w [c_out, c_in]."""
    a = x.double() * _wide(xs, x.shape[1])
    b = w.double() * _wide(_wide(ws, w.shape[1]).T, w.shape[0]).T
    return a @ b.T, a.abs() @ b.abs().T


def _bound(ref, size, c_in, dtype):
    """Half a step of the output type; of a block's sum 128 additions, each off by at most 2^-23 of what has been added up (a matrix instruction
    may cut instead of rounding); two roundings of its scale and one of their product; a sum over the blocks, which up to eight warps share: all
    relative to the sum of the magnitudes."""
    return (torch.finfo(dtype).eps / 2 + 2.0 ** -23) * ref.abs() + (128 + 3 + -(-c_in // 128) + 8) * 2.0 ** -23 * size + 2.0 ** -24


CASES = [
    # c_in, c_out, rows of each projection
    (16, 1, [1]),
    (128, 16, [8]),
    (144, 17, [0, 1, 0, 2]),
    (256, 128, [3, 0, 0, 9, 8, 1]),
    (272, 300, [17, 5, 0, 33]),
    (384, 129, [1, 1, 1, 1, 0, 64]),
    (1008, 1003, [31, 2, 70]),
    (2048, 256, [130, 0, 7, 255, 1]),
    (4096, 520, [2]),
    (512, 640, [257, 300, 0, 191]),
    (1104, 136, [1021]),
    (1024, 2048, [0, 0, 513]),
]


@pytest.mark.parametrize("out", [BF16, F16, F32])
@pytest.mark.parametrize("c_in,c_out,sizes", CASES)
def test_whole_numbers(snn, kernel, c_in, c_out, sizes, out):  # noqa: F811
    g = _gen(c_in + c_out)
    E, R, nb, nk = len(sizes), sum(sizes), -(-c_in // 128), -(-c_out // 128)
    w, ws = _whole8(g, E, c_out, c_in), _powers(g, -2, 0, E, nk, nb)
    x, xs = _whole8(g, R, c_in), _powers(g, -2, 0, R, nb)
    h = snn.SnnConvScaled(w, ws)
    before = snn.kernel_launches()
    y = h.forward(x, xs, offsets=_offsets(sizes), out_type={F16: snn.OUT_F16, BF16: snn.OUT_BF16, F32: snn.OUT_F32}[out])
    assert snn.kernel_launches() > before and y.dtype == out
    lo = 0
    for e, n in enumerate(sizes):
        ref, size = _reference(x[lo:lo + n], xs[lo:lo + n], w[e], ws[e])
        assert n == 0 or size.max() < 2.0 ** 20   # (in steps of 2^-4: exact)
        assert torch.equal(y[lo:lo + n], ref.float().to(out)), f"projection {e}"
        lo += n
    h.destroy()


@pytest.mark.parametrize("c_in,c_out,sizes", [(4096, 200, [3, 40, 300]), (1008, 77, [1, 0, 12]), (2048, 1024, [700, 1100])])
def test_normal_values(snn, kernel, c_in, c_out, sizes):  # noqa: F811
    g = _gen(8)
    E, R, nb, nk = len(sizes), sum(sizes), -(-c_in // 128), -(-c_out // 128)
    w = (100 * torch.randn(E, c_out, c_in, generator=g, device="cuda")).clamp(-448, 448).to(E4M3)
    x = (100 * torch.randn(R, c_in, generator=g, device="cuda")).clamp(-448, 448).to(E4M3)
    ws, xs = 1e-3 * torch.rand(E, nk, nb, generator=g, device="cuda"), 1e-2 * torch.rand(R, nb, generator=g, device="cuda")
    h = snn.SnnConvScaled(w, ws)
    for out in (BF16, F32):
        y = h.forward(x, xs, offsets=_offsets(sizes), out=torch.empty(R, c_out, dtype=out, device="cuda"))
        lo = 0
        for e, n in enumerate(sizes):
            ref, size = _reference(x[lo:lo + n], xs[lo:lo + n], w[e], ws[e])
            assert ((y[lo:lo + n].double() - ref).abs() <= _bound(ref, size, c_in, out)).all()
            lo += n


@pytest.mark.parametrize("rows", [1, 8, 9, 31, 129, 1000])
def test_one_projection_for_all_rows(snn, kernel, rows):  # noqa: F811
    g = _gen(rows)
    w, ws = _whole8(g, 200, 656), _powers(g, -2, 0, 2, 6)
    x, xs = _whole8(g, rows, 656), _powers(g, -2, 0, rows, 6)
    h = snn.SnnConvScaled(w, ws)
    y = h.forward(x, xs)
    assert y.dtype == BF16 and torch.equal(y, _reference(x, xs, w, ws)[0].float().to(BF16))
    buffer = torch.full((rows, 200), 9.0, dtype=F32, device="cuda")
    assert h.forward(x, xs, out=buffer) is buffer and torch.equal(buffer.double(), _reference(x, xs, w, ws)[0])


@pytest.mark.parametrize("rows", [5, 300])
@pytest.mark.parametrize("big,small", [(448.0, 2.0 ** -5), (256.0, 2.0 ** -6), (0.5, 2.0 ** -9)])
def test_sums_of_a_block_have_24_bits(snn, kernel, rows, big, small):  # noqa: F811
    w = torch.ones(130, 256, device="cuda")
    w[:, 0] = big
    x = torch.zeros(rows, 256, device="cuda")
    x[:, 0], x[:, 77] = big, small
    h = snn.SnnConvScaled(w.to(E4M3), torch.ones(2, 2, device="cuda"))
    y = h.forward(x.to(E4M3), torch.ones(rows, 2, device="cuda"), out_type=snn.OUT_F32)
    assert big * big + small == np.float32(big * big + small) and (y == big * big + small).all()


@pytest.mark.parametrize("sizes", [[3, 0, 4, 1], [40, 0, 128, 3], [300, 512, 0, 290]])
def test_strides_and_rows_outside(snn, kernel, sizes):  # noqa: F811
    """Rows of wider buffers; offsets that leave rows before and behind."""
    c_in, c_out, lead, tail = 336, 200, 2, 5
    g = _gen(sum(sizes))
    E, R = len(sizes), lead + sum(sizes) + tail
    w, ws = _whole8(g, E, c_out, c_in), _powers(g, -2, 0, E, 2, 3)
    x = _whole8(g, R, c_in + 48)[:, 16:16 + c_in]
    xs = _powers(g, -2, 0, R, 7)[:, 2:5]
    buffer = torch.full((R, c_out + 13), 77.0, dtype=BF16, device="cuda")
    out = buffer[:, 3:3 + c_out]
    assert snn.SnnConvScaled(w, ws).forward(x, xs, offsets=_offsets(sizes, lead), out=out) is out
    lo = lead
    for e, n in enumerate(sizes):
        assert torch.equal(out[lo:lo + n], _reference(x[lo:lo + n], xs[lo:lo + n], w[e], ws[e])[0].float().to(BF16))
        lo += n
    assert (buffer[:lead] == 77).all() and (buffer[lo:] == 77).all()
    assert (buffer[:, :3] == 77).all() and (buffer[:, 3 + c_out:] == 77).all()


def test_offsets_outside_the_rows(snn, kernel):  # noqa: F811
    g = _gen(3)
    w, ws = _whole8(g, 3, 40, 64), _powers(g, -2, 0, 3, 1, 1)
    x, xs = _whole8(g, 6, 64), _powers(g, -2, 0, 6, 1)
    buffer = torch.full((8, 40), 5.0, dtype=BF16, device="cuda")
    snn.SnnConvScaled(w, ws).forward(x, xs, offsets=torch.tensor([-7, 2, 2, 900], dtype=torch.int32, device="cuda"), out=buffer[1:7])
    for part, e in ((slice(0, 2), 0), (slice(2, 6), 2)):
        assert torch.equal(buffer[1:7][part], _reference(x[part], xs[part], w[e], ws[e])[0].float().to(BF16))
    assert (buffer[0] == 5).all() and (buffer[7] == 5).all()


@pytest.mark.parametrize("n", [5, 200])
def test_nan_and_infinite_scales_stay_in_their_rows(snn, kernel, n):  # noqa: F811
    g = _gen(4)
    w, ws = _whole8(g, 2, 130, 400), _powers(g, -2, 0, 2, 2, 4)
    x, xs = _whole8(g, 2 * n, 400).float(), _powers(g, -2, 0, 2 * n, 4)
    clean = _reference(x[:n], xs[:n], w[0], ws[0])[0].float().to(F32)
    x[1, 5], x[n, 399] = float("nan"), float("nan")
    xs[n - 1, 3], xs[3, 0] = float("inf"), float("nan")
    y = snn.SnnConvScaled(w, ws).forward(x.to(E4M3), xs, offsets=_offsets([n, n]), out_type=snn.OUT_F32)
    bad = [1, 3, n - 1]
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    keep[bad] = False
    assert torch.equal(y[:n][keep], clean[keep])
    assert torch.isnan(y[1]).all() and torch.isnan(y[3]).all() and not torch.isfinite(y[n - 1]).any()
    assert torch.isnan(y[n]).all() and torch.isfinite(y[n + 1:]).all()


def test_many_projections_and_none(snn, kernel):  # noqa: F811
    """More projections than a warp has lanes, most of them without rows; twice the same call gives the same bits; no rows at all."""
    sizes = np.zeros(200, int)
    sizes[[0, 3, 31, 32, 64, 150, 199]] = [1, 20, 2, 5, 40, 1, 9]
    g = _gen(5)
    w, ws = _whole8(g, 200, 70, 144), torch.rand(200, 1, 2, generator=g, device="cuda")
    x, xs = _whole8(g, int(sizes.sum()), 144), torch.rand(int(sizes.sum()), 2, generator=g, device="cuda")
    h, offsets = snn.SnnConvScaled(w, ws), _offsets(sizes)
    y, again = (h.forward(x, xs, offsets=offsets, out_type=snn.OUT_F32) for _ in range(2))
    assert torch.equal(y, again)
    for e in sizes.nonzero()[0]:
        part = slice(int(offsets[e]), int(offsets[e + 1]))
        ref, size = _reference(x[part], xs[part], w[e], ws[e])
        assert ((y[part].double() - ref).abs() <= _bound(ref, size, 144, F32)).all()
    out = torch.full((4, 70), 3.0, dtype=F16, device="cuda")
    h.forward(x[:4], xs[:4], offsets=torch.zeros(201, dtype=torch.int32, device="cuda"), out=out)
    assert (out == 3).all()
    assert h.forward(x[:0], xs[:0]).shape == (0, 70)


def test_weights_are_copied_and_the_handle_ends(snn):  # noqa: F811
    g = _gen(6)
    w, ws = _whole8(g, 33, 64), _powers(g, -2, 0, 1, 1)
    x, xs = _whole8(g, 4, 64), _powers(g, -2, 0, 4, 1)
    ref = _reference(x, xs, w, ws)[0].float().to(BF16)
    h = snn.SnnConvScaled(w, ws)
    w.zero_()
    ws.zero_()
    assert torch.equal(h.forward(x, xs), ref)
    h.destroy()
    with pytest.raises(snn.SnnError, match="destroyed"):
        h.forward(x, xs)


def test_weights_written_on_another_stream(snn):  # noqa: F811
    """The copy follows what the stream has before it."""
    g = _gen(7)
    w, ws, x, xs = _whole8(g, 300, 256), _powers(g, -2, 0, 3, 2), _whole8(g, 9, 256), _powers(g, -2, 0, 9, 2)
    ref = _reference(x, xs, w, ws)[0].float().to(BF16)
    s, late = torch.cuda.Stream(), torch.zeros(300, 256, device="cuda").to(E4M3)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        late.copy_(w)
        h = snn.SnnConvScaled(late, ws)
        y = h.forward(x, xs)
    s.synchronize()
    assert torch.equal(y, ref)


def test_captured_and_replayed(snn, kernel):  # noqa: F811
    """Quantisation and products in one graph, replayed on other inputs; a second graph of the same handle on another stream."""
    g = _gen(9)
    w, ws = _whole8(g, 272, 384), _powers(g, -2, 0, 3, 3)
    h = snn.SnnConvScaled(w, ws)
    rows, graphs = 70, []
    for _ in range(2):
        x, q, y = torch.zeros(rows, 384, dtype=BF16, device="cuda"), snn.alloc_quantised(rows, 384), torch.empty(rows, 272, dtype=F32, device="cuda")
        h.forward(*snn.quantise(x, out=q), out=y)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            snn.quantise(x, out=q)
            h.forward(q.values, q.scales, out=y)
        graphs.append((graph, x, q, y, torch.cuda.Stream()))
    for turn in range(3):
        for graph, x, q, y, s in graphs:
            x.copy_(torch.randn(rows, 384, generator=g, device="cuda"))
        torch.cuda.synchronize()
        for graph, x, q, y, s in graphs:
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for graph, x, q, y, s in graphs:
            _check_quantised(q, x.float(), exact=True)
            ref, size = _reference(q.values, q.scales, w, ws)
            assert ((y.double() - ref).abs() <= _bound(ref, size, 384, F32)).all()


# ------------------------------------------------------------------------------------------------------------ quantise

def _grid(q):
    """The e4m3 number nearest to q, ties to even, in 64 bits."""
    step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(q / step) * step


def _check_quantised(got, v, exact):
    """`v`: the rows in fp32 as they are, or in fp64 behind an activation.  exact: the formula's bits; else the scale within the activation's error,
    and values within half a step, by the scale that came out, and what the error of v can move."""
    values, scales = got
    finite = torch.isfinite(v)
    clean = torch.where(finite, v, torch.zeros_like(v))
    C = v.shape[1]
    blocks = torch.nn.functional.pad(clean.abs(), (0, -C % 128)).reshape(len(v), -1, 128)
    if exact:
        most = blocks.amax(2)
        want = torch.maximum(most / torch.full_like(most, 448.0), torch.full_like(most, 2.0 ** -70))
        assert torch.equal(scales, want)
        q = (clean / want.repeat_interleave(128, 1)[:, :C]).double()
        assert torch.equal(torch.where(finite, values.double(), torch.zeros_like(q)), torch.where(finite, _grid(q), torch.zeros_like(q)))
        assert torch.isnan(values.double()[~finite]).all()
        return
    # the error of v: the function's, 2^-20 of the value (test_activate), and so of the largest of a block, and a division's half step
    want = (blocks.amax(2) / 448).clamp(min=2.0 ** -70)
    assert ((scales.double() - want).abs() <= 2.0 ** -19 * want).all()
    q = clean / scales.double().repeat_interleave(128, 1)[:, :C]
    step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
    assert ((values.double() - q).abs() <= 0.5 * step * (1 + 2.0 ** -10) + 2.0 ** -19 * q.abs()).all()


@pytest.mark.parametrize("R,C", [(1, 1), (1, 128), (3, 129), (17, 1003), (64, 4096), (5, 16), (301, 264), (2, 8200)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_quantise(snn, R, C, dtype):  # noqa: F811
    g = _gen(R + C)
    x = (torch.randn(R, C, generator=g, device="cuda") * torch.exp2(torch.randint(-9, 6, (R, 1), generator=g, device="cuda").float())).to(dtype)
    got = snn.quantise(x)
    assert got.values.shape == (R, C) and got.scales.shape == (R, -(-C // 128)) and got.values.stride(0) % 16 == 0
    _check_quantised(got, x.float(), exact=True)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_quantise_corners(snn, dtype):  # noqa: F811
    """Blocks of zeros and of tiny values, infinities and NaN, the type's largest, ties."""
    x = torch.randn(9, 300, generator=_gen(2), device="cuda").to(dtype)
    x[0] = 0
    x[1, :128] *= 1e-30
    x[2, 7], x[2, 200] = float("nan"), float("inf")
    x[3] = -float("inf")
    x[4, 0], x[4, 130] = torch.finfo(dtype).max, -torch.finfo(dtype).max
    x[5] = torch.arange(300, device="cuda").to(dtype)
    x[5, 127] = 448
    x[6, :128] = 1e-25
    x[7, 5] = -0.0
    x[8, :] = torch.finfo(dtype).tiny
    _check_quantised(snn.quantise(x), x.float(), exact=True)
    got = snn.quantise(x)
    assert (got.scales[0] == 2.0 ** -70).all() and (got.values[0].float() == 0).all()
    assert got.values.view(torch.uint8)[3].eq(0x7f).all()


@pytest.mark.parametrize("C,lead", [(256, 8), (256, 3), (136, 8), (1003, 5)])
@pytest.mark.parametrize("dtype", [F32, F16])
def test_quantise_by_an_index_with_strides(snn, C, lead, dtype):  # noqa: F811
    g = _gen(C + lead)
    n, m = 11, 40
    x = torch.randn(n, C + 16, generator=g, device="cuda").to(dtype)[:, lead:lead + C]
    rows = torch.randint(0, n, (m,), generator=g, device="cuda", dtype=torch.int32)
    rows[0], rows[1], rows[-1] = -1, n, 2 ** 31 - 1
    values = torch.full((m, C + 21), 3.0, device="cuda").to(E4M3)
    scales = torch.full((m, -(-C // 128) + 3), 5.0, device="cuda")
    out = (values[:, 2:2 + C], scales[:, 1:-2])
    got = snn.quantise(x, rows=rows, out=out)
    assert got is out
    v = torch.zeros(m, C, dtype=dtype, device="cuda")
    ok = (rows >= 0) & (rows < n)
    v[ok] = x[rows[ok].long()]
    _check_quantised(got, v.float(), exact=True)
    assert (values[:, :2].float() == 3).all() and (values[:, 2 + C:].float() == 3).all()
    assert (scales[:, :1] == 5).all() and (scales[:, -2:] == 5).all()


def _fn64(name, v):
    if name == "FN_SILU":
        return v * torch.sigmoid(v)
    if name == "FN_GELU":
        return 0.5 * v * torch.special.erfc(-v / 2 ** 0.5)
    return v.clamp(min=0) if name == "FN_RELU" else v


@pytest.mark.parametrize("fn", ["FN_SILU", "FN_GELU", "FN_RELU", "FN_NONE"])
@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("R,C", [(3, 200), (70, 1024), (9, 77)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_quantise_behind_an_activation(snn, fn, gated, R, C, dtype):  # noqa: F811
    g = _gen(R + C)
    up, gate = (2 * torch.randn(R, C, generator=g, device="cuda").to(dtype) for _ in range(2))
    v = _fn64(fn, gate.double()) * up.double() if gated else _fn64(fn, up.double())
    got = snn.quantise(up, gate=gate if gated else None, fn=getattr(snn, fn))
    _check_quantised(got, v, exact=False)


def test_quantise_nothing(snn):  # noqa: F811
    assert snn.quantise(torch.empty(0, 40, device="cuda")).values.shape == (0, 40)
    none = torch.empty(0, 40, dtype=F16, device="cuda")
    got = snn.quantise(none, rows=torch.zeros(3, dtype=torch.int32, device="cuda"))   # rows of an input without any are zeros
    assert (got.values.float() == 0).all() and (got.scales == 2.0 ** -70).all()


# ------------------------------------------------------------------------------------------------------------ activate

@pytest.mark.parametrize("fn", ["FN_SILU", "FN_GELU", "FN_RELU", "FN_NONE"])
@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("R,C", [(1, 1), (3, 200), (70, 1024), (9, 77), (515, 8)])
@pytest.mark.parametrize("dtype,out", [(F32, F32), (F16, F16), (BF16, BF16), (BF16, F32), (F32, F16)])
def test_activate(snn, fn, gated, R, C, dtype, out):  # noqa: F811
    """The exponential within 2 steps (of a number up to 1 + it), an addition, a division and a product: 2^-21 of the value; the normal
    distribution's function within 5 steps by CUDA's documentation, where it is not below the smallest normal number: 2^-20 with the products."""
    g = _gen(R + C)
    up, gate = (2 * torch.randn(R, C, generator=g, device="cuda").to(dtype) for _ in range(2))
    v = _fn64(fn, gate.double()) * up.double() if gated else _fn64(fn, up.double())
    got = snn.activate(up, gate=gate if gated else None, fn=getattr(snn, fn), out=torch.empty(R, C, dtype=out, device="cuda"))
    assert ((got.double() - v).abs() <= (torch.finfo(out).eps / 2 + 2.0 ** -20) * v.abs() + torch.finfo(out).smallest_normal).all()


def test_activate_values_at_the_ends(snn):  # noqa: F811
    inf, nan = float("inf"), float("nan")
    v = torch.tensor([[0.0, -0.0, inf, nan, 100.0, -100.0, 3e38, -3e38]], device="cuda")
    silu, gelu, relu = (snn.activate(v, fn=f)[0].tolist() for f in (snn.FN_SILU, snn.FN_GELU, snn.FN_RELU))
    for got in (silu, gelu, relu):
        assert got[0] == 0 and got[1] == 0 and got[2] == inf and got[3] != got[3] and got[4] == 100 and abs(got[5]) < 1e-37 and got[6] == np.float32(3e38) and got[7] == 0
    assert torch.isnan(snn.activate(torch.full((1, 1), -inf, device="cuda"), fn=snn.FN_SILU)).all()


@pytest.mark.parametrize("C,lead", [(256, 8), (256, 3), (77, 5)])
def test_activate_with_strides_and_in_place(snn, C, lead):  # noqa: F811
    g = _gen(C)
    both = torch.randn(13, 2 * C + 16, generator=g, device="cuda").to(BF16)
    gate, up = both[:, lead:lead + C], both[:, lead + C:lead + 2 * C]   # (as one projection of twice the columns leaves them)
    want = snn.activate(up.contiguous(), gate=gate.contiguous(), fn=snn.FN_SILU)
    rest = both.clone()
    assert snn.activate(up, gate=gate, fn=snn.FN_SILU, out=up) is up and torch.equal(up, want)
    rest[:, lead + C:lead + 2 * C] = want
    assert torch.equal(both, rest)
    assert snn.activate(torch.empty(0, 5, device="cuda")).shape == (0, 5)

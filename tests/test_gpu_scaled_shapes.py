"""Every kernel of the 8-bit projections at sizes where the library would take another: the cases of test_gpu_scaled by tiles of 64, 128 and 256 output
channels, and with several CTAs that share a tile's input channels; and larger ones that reach several tiles, turns and rounds of buffers."""
import numpy as np
import pytest
import torch

import test_gpu_scaled as one
from test_gpu_projections import BF16, F16, F32, _gen, snn  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["few", "64", "64/2", "64/4", "128", "256"])
def kernel(request, monkeypatch):
    monkeypatch.setenv("SNN_FORCE_ROWS", request.param)
    return request.param


@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("c_in,c_out,sizes", one.CASES)
def test_whole_numbers(snn, kernel, c_in, c_out, sizes, out):  # noqa: F811
    one.test_whole_numbers(snn, kernel, c_in, c_out, sizes, out)


@pytest.mark.parametrize("rows", [1, 16, 33, 129, 700])
def test_one_projection(snn, kernel, rows):  # noqa: F811
    one.test_one_projection_for_all_rows(snn, kernel, rows)
    one.test_sums_of_a_block_have_24_bits(snn, kernel, rows, 448.0, 2.0 ** -5)


def test_edges(snn, kernel):  # noqa: F811
    one.test_strides_and_rows_outside(snn, kernel, [300, 512, 0, 290])
    one.test_offsets_outside_the_rows(snn, kernel)
    one.test_nan_and_infinite_scales_stay_in_their_rows(snn, kernel, 5)
    one.test_nan_and_infinite_scales_stay_in_their_rows(snn, kernel, 200)
    one.test_many_projections_and_none(snn, kernel)
    one.test_captured_and_replayed(snn, kernel)


@pytest.mark.parametrize("c_in,c_out,rows,out", [
    (2048, 48, 100, F32), (4096, 200, 65, BF16), (1552, 129, 250, F16),   # few tiles: shared by all that can share
    (640, 1300, 700, BF16), (4096, 512, 40, F32), (144, 4100, 513, F16), (272, 2500, 2000, BF16), (1040, 255, 5000, F32),
    (2560, 300, 30, BF16), (2560, 2500, 64, F32), (1280, 128, 128, F16),   # shares that begin at blocks that four does not divide
])
def test_larger(snn, kernel, c_in, c_out, rows, out):  # noqa: F811
    g = _gen(rows)
    nb, nk = -(-c_in // 128), -(-c_out // 128)
    w, ws = one._whole8(g, c_out, c_in), one._powers(g, -2, 0, nk, nb)
    x, xs = one._whole8(g, rows, c_in), one._powers(g, -2, 0, rows, nb)
    buffer = torch.full((rows + 2, c_out + 3), 5.0, dtype=out, device="cuda")   # (rows that are not 16-byte aligned)
    h = snn.SnnConvScaled(w, ws)
    ref, size = one._reference(x, xs, w, ws)
    assert size.max() < 2.0 ** 20
    want = ref.float().to(out)
    for y in (buffer[1:-1, 2:2 + c_out], torch.empty(rows, c_out, dtype=out, device="cuda")):
        h.forward(x, xs, out=y)
        assert torch.equal(y, want)
    assert (buffer[0] == 5).all() and (buffer[-1] == 5).all() and (buffer[:, :2] == 5).all() and (buffer[:, -1] == 5).all()


@pytest.mark.parametrize("E", [150, 1024])
def test_as_many_projections_as_there_can_be(snn, kernel, E):  # noqa: F811
    """The ranges of all take shared memory from the stages; each projection several tiles away from the one before."""
    g = _gen(E)
    sizes = np.zeros(E, int)
    sizes[::max(1, E // 40)] = 3
    sizes[[0, E // 2, E - 1]] = [300, 130, 257]
    w, ws = one._whole8(g, E, 40, 528), one._powers(g, -2, 0, E, 1, 5)
    R = int(sizes.sum())
    x, xs, offsets = one._whole8(g, R, 528), one._powers(g, -2, 0, R, 5), one._offsets(sizes)
    h = snn.SnnConvScaled(w, ws)
    for _ in range(3):
        y = h.forward(x, xs, offsets=offsets, out_type=snn.OUT_F32)
    lo = 0
    for e in sizes.nonzero()[0]:
        n = int(sizes[e])
        assert torch.equal(y[lo:lo + n].double(), one._reference(x[lo:lo + n], xs[lo:lo + n], w[e], ws[e])[0]), f"projection {e}"
        lo += n


@pytest.mark.parametrize("E,each,c_in,c_out", [(64, 1, 2048, 1024), (200, 1, 1152, 520), (24, 7, 640, 2048), (40, 100, 1664, 640)])
def test_many_tiles_of_few_rows(snn, kernel, E, each, c_in, c_out):  # noqa: F811
    """Each CTA has several tiles, of an odd number of blocks too: the two warps that multiply take turns over them, with few stages and with many."""
    g = _gen(E * each)
    nb, nk = -(-c_in // 128), -(-c_out // 128)
    w, ws = one._whole8(g, E, c_out, c_in), one._powers(g, -2, 0, E, nk, nb)
    x, xs, offsets = one._whole8(g, E * each, c_in), one._powers(g, -2, 0, E * each, nb), one._offsets([each] * E)
    h = snn.SnnConvScaled(w, ws)
    for _ in range(3):
        y = h.forward(x, xs, offsets=offsets, out_type=snn.OUT_F32)
    for e in range(0, E, 7):
        rows = slice(e * each, (e + 1) * each)
        ref, size = one._reference(x[rows], xs[rows], w[e], ws[e])
        assert size.max() < 2.0 ** 20 and torch.equal(y[rows].double(), ref), f"projection {e}"

"""Projections of language models on a GPU: experts with ragged row counts, the router, the weighted sum and low-rank adapters,
each against plain arithmetic in 64 bits.

Two kinds of inputs.  Whole numbers, small enough that every partial sum in any order is below 2^24: the fp32 sums are then exact and the
outputs have one correct value each, whatever the kernel, so they are compared bit by bit.  Normal values: the tolerance of an output
is derived in _bound."""
import numpy as np
import pytest
import torch

import workloads as wl

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def snn():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2110_09195_b200 import build
    build.build()
    import paper_2110_09195_b200 as m
    m.load_library()
    return m


def _decode(p, c_in, c_out):
    """+1 / -1 [c_out, c_in]: LSB-first tau-bit indices, element j of a vector is bit 7 - j of its code."""
    n = c_out * (c_in // 8)
    bits = np.unpackbits(p.idx_packed, bitorder="little")[: n * p.tau].reshape(n, p.tau).astype(np.int64)
    codes = p.codebook.astype(np.int64)[(bits << np.arange(p.tau)).sum(1)]
    signs = ((codes[:, None] >> (7 - np.arange(8))) & 1) * 2 - 1
    return torch.from_numpy(signs.reshape(c_out, c_in).astype(np.float64)).cuda()


def _layers(snn, count, c_in, c_out, tau, seed, alpha=None, act_type=None):
    layers, w, al = [], [], []
    for e in range(count):
        p = wl.draw_layer_params(wl.LayerShape(c_in, c_out, 1, 1, 1, 0, 1), tau, seed + e)
        a = p.alpha if alpha is None else np.full(c_out, alpha, np.float32)
        layers.append(snn.SnnConv(c_in, c_out, tau, p.codebook, p.idx_packed, a, pad=0, ksize=1,
                                  act_type=snn.ACT_F16 if act_type is None else act_type))
        w.append(_decode(p, c_in, c_out))
        al.append(torch.from_numpy(a).cuda())
    return layers, w, al


def _whole(g, most, *shape):
    return torch.randint(-most, most + 1, shape, generator=g, device="cuda").double()


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _bound(ref, norm, alpha, c_in, dtype):
    """Half a step of the output type, one rounding each of the scale's product and the sum, and the fp32 sum: at most c_in additions, each off by at most
    2^-23 of a partial sum (a matrix instruction may cut instead of rounding), and a partial sum of +/-x in any order
    stays within 6 |x|_2 (six standard deviations of a random walk)."""
    return (torch.finfo(dtype).eps / 2 + 2.0 ** -23) * ref.abs() + c_in * 2.0 ** -23 * 6 * norm * alpha.abs() + 2.0 ** -24


EXPERT_CASES = [
    # c_in, c_out, tau, rows of each expert
    (8, 1, 3, [1]),
    (64, 37, 4, [0, 1, 0, 2]),
    (72, 128, 5, [3, 0, 0, 9, 8, 1]),
    (256, 300, 8, [17, 5, 0, 33]),
    (264, 129, 5, [1, 1, 1, 1, 0, 64]),
    (1000, 1003, 7, [31, 2, 70]),
    (2048, 256, 5, [130, 0, 7, 255, 1]),
    (4096, 512, 5, [2]),
    (520, 640, 1, [257, 300, 0, 191]),
    (1096, 136, 6, [1021]),
    (64, 2048, 2, [0, 0, 513]),
]


@pytest.mark.parametrize("act,out", [(F16, F16), (BF16, BF16), (F16, F32), (BF16, F32), (BF16, F16)])
@pytest.mark.parametrize("c_in,c_out,tau,sizes", EXPERT_CASES)
def test_experts_whole_numbers(snn, c_in, c_out, tau, sizes, act, out):
    g = _gen(c_in + c_out)
    layers, w, al = _layers(snn, len(sizes), c_in, c_out, tau, 900 + c_in)
    ex = snn.SnnConvExperts(layers)
    for l in layers:
        l.destroy()   # (the weights were copied)
    R = sum(sizes)
    x = _whole(g, 8, R, c_in).to(act)
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32, device="cuda")
    before = snn.kernel_launches()
    y = ex.forward(x, offsets, out_type={F16: snn.OUT_F16, BF16: snn.OUT_BF16, F32: snn.OUT_F32}[out])
    assert snn.kernel_launches() > before and y.dtype == out
    lo = 0
    for e, n in enumerate(sizes):
        ref = ((x[lo:lo + n].double() @ w[e].T).float() * al[e]).to(out)
        assert torch.equal(y[lo:lo + n], ref), f"expert {e}"
        lo += n
    ex.destroy()


@pytest.mark.parametrize("act", [F16, BF16])
@pytest.mark.parametrize("c_in,c_out,sizes", [(4096, 200, [3, 40, 300]), (1000, 77, [1, 0, 12]), (2048, 1024, [700, 1100])])
def test_experts_normal_values(snn, c_in, c_out, sizes, act):
    g = _gen(7)
    layers, w, al = _layers(snn, len(sizes), c_in, c_out, 5, 930)
    ex = snn.SnnConvExperts(layers)
    x = torch.randn(sum(sizes), c_in, generator=g, device="cuda").to(act)
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32, device="cuda")
    for out in (act, F32):
        y = ex.forward(x, offsets, out=torch.empty(len(x), c_out, dtype=out, device="cuda"))
        lo = 0
        for e, n in enumerate(sizes):
            xe = x[lo:lo + n].double()
            ref = (xe @ w[e].T) * al[e].double()
            err = (y[lo:lo + n].double() - ref).abs()
            assert (err <= _bound(ref, xe.norm(dim=1, keepdim=True), al[e].double(), c_in, out)).all()
            lo += n


@pytest.mark.parametrize("n_tok,sizes", [(5, [3, 0, 4, 1]), (70, [40, 0, 128, 3]), (300, [300, 512, 0, 290])])
@pytest.mark.parametrize("act", [F16, BF16])
def test_experts_gathered_rows_with_strides(snn, n_tok, sizes, act):
    """Rows named by an index, some of them outside (zeros); rows of wider buffers; offsets that leave rows before and behind."""
    c_in, c_out, lead, tail = 328, 200, 2, 5
    g = _gen(n_tok)
    layers, w, al = _layers(snn, len(sizes), c_in, c_out, 5, 940)
    ex = snn.SnnConvExperts(layers)
    wide = _whole(g, 8, n_tok, c_in + 24).to(act)
    x = wide[:, 8:8 + c_in]
    R = lead + sum(sizes) + tail
    rows = torch.randint(0, n_tok, (R,), generator=g, device="cuda", dtype=torch.int32)
    rows[lead], rows[lead + 1] = -1, n_tok
    rows[-1] = 2 ** 31 - 1
    offsets = torch.tensor(lead + np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32, device="cuda")
    buffer = torch.full((R, c_out + 13), 77.0, dtype=act, device="cuda")
    out = buffer[:, 3:3 + c_out]
    assert ex.forward(x, offsets, rows=rows, out=out) is out
    xr = torch.zeros(R, c_in, dtype=torch.float64, device="cuda")
    ok = (rows >= 0) & (rows < n_tok)
    xr[ok] = x.double()[rows[ok].long()]
    lo = lead
    for e, n in enumerate(sizes):
        assert torch.equal(out[lo:lo + n], ((xr[lo:lo + n] @ w[e].T).float() * al[e]).to(act))
        lo += n
    assert (buffer[:lead] == 77).all() and (buffer[lo:] == 77).all()
    assert (buffer[:, :3] == 77).all() and (buffer[:, 3 + c_out:] == 77).all()


def test_experts_offsets_outside_the_rows(snn):
    """Offsets are held to the rows that there are: nothing is read or written elsewhere."""
    layers, w, al = _layers(snn, 3, 64, 40, 5, 950)
    ex = snn.SnnConvExperts(layers)
    x = _whole(_gen(3), 8, 6, 64).to(BF16)
    buffer = torch.full((8, 40), 5.0, dtype=BF16, device="cuda")
    ex.forward(x, torch.tensor([-7, 2, 2, 900], dtype=torch.int32, device="cuda"), out=buffer[1:7])
    for part, e in ((slice(0, 2), 0), (slice(2, 6), 2)):
        assert torch.equal(buffer[1:7][part], ((x[part].double() @ w[e].T).float() * al[e]).to(BF16))
    assert (buffer[0] == 5).all() and (buffer[7] == 5).all()


@pytest.mark.parametrize("n", [5, 200])
def test_experts_infinities_and_nan_stay_in_their_rows(snn, n):
    c_in, c_out = 192, 130
    layers, w, al = _layers(snn, 2, c_in, c_out, 5, 960)
    ex = snn.SnnConvExperts(layers)
    x = _whole(_gen(4), 8, 2 * n, c_in).to(F16)
    clean = ((x.double() @ w[0].T).float() * al[0]).to(F16)
    x[1, 5], x[n - 1, 0], x[n, 3] = float("nan"), float("inf"), float("nan")   # (row n is the other expert's)
    y = ex.forward(x, torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda"))
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    keep[1] = keep[n - 1] = False
    assert torch.equal(y[:n][keep], clean[:n][keep])
    assert torch.isnan(y[1]).all() and torch.isinf(y[n - 1]).all() and torch.isnan(y[n]).all()
    assert torch.equal(y[n - 1] > 0, (w[0][:, 0] * al[0] > 0)) and torch.isfinite(y[n + 1:]).all()


def test_experts_fp16_overflow_is_an_infinity(snn):
    layers, w, al = _layers(snn, 1, 64, 16, 5, 970, alpha=1024.0)
    y = snn.SnnConvExperts(layers).forward(torch.full((3, 64), 512.0, dtype=F16, device="cuda"), torch.tensor([0, 3], dtype=torch.int32, device="cuda"))
    ref = (w[0].sum(1).float() * 512 * 1024).to(F16)
    assert torch.equal(y, ref.expand(3, -1)) and torch.isinf(y).any()


def test_experts_many(snn):
    """More experts than a warp has lanes, most of them without rows; twice the same call gives the same bits."""
    sizes = np.zeros(200, int)
    sizes[[0, 3, 31, 32, 64, 150, 199]] = [1, 20, 2, 5, 40, 1, 9]
    c_in, c_out = 136, 70
    layers, w, al = _layers(snn, len(sizes), c_in, c_out, 4, 980)
    ex = snn.SnnConvExperts(layers)
    x = torch.randn(int(sizes.sum()), c_in, generator=_gen(5), device="cuda").to(BF16)
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32, device="cuda")
    y, again = ex.forward(x, offsets, out_type=snn.OUT_F32), ex.forward(x, offsets, out_type=snn.OUT_F32)
    assert torch.equal(y, again)
    for e in sizes.nonzero()[0]:
        part = slice(int(offsets[e]), int(offsets[e + 1]))
        ref = (x[part].double() @ w[e].T) * al[e].double()
        assert ((y[part].double() - ref).abs() <= _bound(ref, x[part].double().norm(dim=1, keepdim=True), al[e].double(), c_in, F32)).all()


def test_experts_without_rows(snn):
    layers, _, _ = _layers(snn, 2, 64, 32, 5, 985)
    ex = snn.SnnConvExperts(layers)
    offsets = torch.zeros(3, dtype=torch.int32, device="cuda")
    assert ex.forward(torch.empty(0, 64, dtype=F16, device="cuda"), offsets).shape == (0, 32)
    out = torch.full((4, 32), 3.0, dtype=F16, device="cuda")
    ex.forward(torch.empty(0, 64, dtype=F16, device="cuda"), offsets, out=out)
    ex.forward(torch.ones(4, 64, dtype=F16, device="cuda"), offsets, out=out)
    assert (out == 3).all()
    # rows of an input without any are zeros
    ex.forward(torch.empty(0, 64, dtype=F16, device="cuda"), torch.tensor([0, 4, 4], dtype=torch.int32, device="cuda"), out=out)
    assert (out == 0).all()


# ------------------------------------------------------------------------------------------------------------ router

def _route_ref(logits, k, normalise):
    v = logits.double().cpu().numpy()
    T, E = v.shape
    ids, weights = np.full((T, k), -1, np.int32), np.zeros((T, k))
    per = [[] for _ in range(E)]
    for t in range(T):
        able = [e for e in range(E) if v[t, e] > -np.inf]
        best = sorted(able, key=lambda e: (-v[t, e], e))[:k]
        if not best:
            continue
        top = v[t, best[0]]
        with np.errstate(invalid="ignore"):
            term = {e: 1.0 if v[t, e] == top else float(np.exp(v[t, e] - top)) for e in able}
        total = sum(term[e] for e in (best if normalise else able))
        for j, e in enumerate(best):
            ids[t, j], weights[t, j] = e, term[e] / total
            per[e].append((t, j))
    offsets, rows, slots = [0], np.full(T * k, -1, np.int32), np.full((T, k), -1, np.int32)
    for e in range(E):
        for i, (t, j) in enumerate(per[e]):
            rows[offsets[-1] + i], slots[t, j] = t, offsets[-1] + i
        offsets.append(offsets[-1] + len(per[e]))
    return ids, weights, np.array(offsets, np.int32), rows, slots


def _check_route(r, logits, k, normalise):
    ids, weights, offsets, rows, slots = _route_ref(logits, k, normalise)
    assert (r.ids.cpu().numpy() == ids).all()
    assert (r.offsets.cpu().numpy() == offsets).all()
    assert (r.rows.cpu().numpy() == rows).all() and (r.slots.cpu().numpy() == slots).all()
    # expf within 2 steps, a subtraction rounded before it (its error times the result), up to E + 1 additions, a division
    E = logits.shape[1]
    w, spread = r.weights.cpu().double().numpy(), 2.0 ** -24 * 200
    assert (np.abs(w - weights) <= (2.0 ** -23 * (E + 6) + spread) * weights + 1e-38).all()
    assert (w[ids < 0] == 0).all()


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 64, 2), (3, 8, 8), (63, 33, 3), (64, 60, 4), (65, 128, 8), (1000, 7, 2), (2111, 256, 8), (130, 1024, 16),
                                   (777, 300, 1), (129, 513, 5)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("normalise", [True, False])
def test_route(snn, T, E, k, dtype, normalise):
    logits = (2 * torch.randn(T, E, generator=_gen(T + E), device="cuda")).to(dtype)   # (16-bit logits: many are equal)
    r = snn.route(logits, k, normalise=normalise)
    _check_route(r, logits, k, normalise)
    assert snn.route(logits, k, normalise=normalise, out=r) is r
    _check_route(r, logits, k, normalise)


@pytest.mark.parametrize("T", [9, 200])
@pytest.mark.parametrize("normalise", [True, False])
def test_route_masks(snn, T, normalise):
    """Experts switched off, whole tokens switched off, NaN, equal logits, both zeros, the type's lowest value, infinities."""
    E, k = 40, 4
    logits = torch.randn(T, E, generator=_gen(T), device="cuda")
    logits[0] = -float("inf")
    logits[1] = float("nan")
    logits[2, 3:] = -float("inf")
    logits[3] = 0.0
    logits[4, ::2], logits[4, 1::2] = -0.0, 0.0
    logits[5] = torch.finfo(F32).min
    logits[5, 7] = 1.0
    logits[6, 11] = logits[6, 30] = float("inf")
    logits[7] = torch.finfo(F32).min
    logits[8, 20:] = float("nan")
    r = snn.route(logits, k, normalise=normalise)
    _check_route(r, logits, k, normalise)
    assert (r.ids[:2] == -1).all() and (r.slots[:2] == -1).all()
    assert r.ids[3].tolist() == r.ids[4].tolist() == r.ids[7].tolist() == [0, 1, 2, 3]
    r = snn.route(logits[:2].contiguous(), k)   # nothing for anybody
    assert (r.offsets == 0).all() and (r.rows == -1).all()


@pytest.mark.parametrize("T,E,k", [(16384, 20, 3), (16385, 40, 2), (40001, 300, 4)])
def test_route_long(snn, T, E, k):
    """Past 256 groups of 64 tokens the counts are summed up in a launch of their own; compared with sorts, all values being different."""
    g = _gen(T)
    logits = torch.rand(T, E, generator=g, device="cuda").argsort(1).float() / 8   # (no two equal in a row)
    r = snn.route(logits, k)
    top, ids = torch.sort(logits, dim=1, descending=True)
    assert torch.equal(r.ids, ids[:, :k].to(torch.int32))
    w = torch.softmax(top[:, :k].double(), 1)
    assert ((r.weights.double() - w).abs() <= 2.0 ** -20 * w).all()   # (differences of eighths: exact; expf, k sums, a division)
    order = torch.sort(ids[:, :k].reshape(-1), stable=True).indices
    assert torch.equal(r.rows, (order // k).to(torch.int32))
    counts = torch.bincount(ids[:, :k].reshape(-1), minlength=E)
    assert torch.equal(r.offsets[1:], torch.cumsum(counts, 0).to(torch.int32)) and r.offsets[0] == 0
    slots = torch.empty_like(order)
    slots[order] = torch.arange(T * k, device="cuda")
    assert torch.equal(r.slots.reshape(-1), slots.to(torch.int32))


def test_route_strided_and_empty(snn):
    wide = torch.randn(70, 50, generator=_gen(1), device="cuda")
    logits = wide[:, 5:38]
    _check_route(snn.route(logits, 3), logits.contiguous(), 3, True)
    r = snn.route(torch.empty(0, 12, device="cuda"), 2)
    assert (r.offsets == 0).all() and r.ids.shape == (0, 2)


# ------------------------------------------------------------------------------------------------------------ combine

@pytest.mark.parametrize("T,k,C", [(1, 1, 1), (3, 2, 8), (7, 4, 1003), (64, 8, 2048), (301, 2, 72), (33, 16, 260), (5, 3, 4104)])
@pytest.mark.parametrize("dtype,out", [(F32, F32), (F16, F16), (BF16, BF16), (BF16, F32), (F32, BF16), (F16, BF16)])
def test_combine(snn, T, k, C, dtype, out):
    g = _gen(T + C)
    n = T * k + 3
    y = torch.randn(n, C, generator=g, device="cuda").to(dtype)
    slots = torch.randperm(n, generator=g, device="cuda")[: T * k].reshape(T, k).to(torch.int32)
    weights = torch.rand(T, k, generator=g, device="cuda")
    slots[torch.rand(T, k, generator=g, device="cuda") < 0.2] = -1
    slots[0, 0] = n   # outside
    if T > 2:
        slots[2] = -1
    got = snn.combine(y, slots, weights, out=torch.empty(T, C, dtype=out, device="cuda"))
    ok = (slots >= 0) & (slots < n)
    terms = torch.where(ok[..., None], weights[..., None].double() * y.double()[slots.clamp(0, n - 1).long()], 0.0)
    ref = terms.sum(1)
    # each of the k products and sums is rounded once, relative to what has been summed; then the output type
    bound = torch.finfo(out).eps / 2 * ref.abs() + 2 * k * 2.0 ** -24 * terms.abs().sum(1) + 2.0 ** -24
    assert ((got.double() - ref).abs() <= bound).all()
    if T > 2:
        assert (got[2] == 0).all()


def test_combine_strides_and_what_no_slot_names(snn):
    g = _gen(2)
    wide = torch.randn(20, 90, generator=g, device="cuda").to(BF16)
    y = wide[:, 1:74]
    y[13] = float("nan")
    slots = torch.tensor([[0, 5], [12, -1], [-1, -1]], dtype=torch.int32, device="cuda")
    weights = torch.tensor([[0.5, 0.25], [1.0, float("nan")], [float("inf"), 2.0]], device="cuda")
    buffer = torch.full((3, 80), 9.0, device="cuda")
    got = snn.combine(y, slots, weights, out=buffer[:, 2:75])
    assert torch.equal(got[0], 0.5 * y[0].float() + 0.25 * y[5].float())
    assert torch.equal(got[1], y[12].float()) and (got[2] == 0).all()
    assert (buffer[:, :2] == 9).all() and (buffer[:, 75:] == 9).all()
    assert snn.combine(y, slots[:0], weights[:0]).shape == (0, 73)
    empty = snn.combine(y[:0], slots, weights)
    assert (empty == 0).all()


# ------------------------------------------------------------------------------------------------------------ adapters

ADAPTER_CASES = [
    # rows, c_in, c_out, tau, adapters, rank, rows of a run
    (1, 64, 40, 5, 1, 8, 1),
    (1, 4096, 256, 5, 4, 16, 1),
    (9, 72, 130, 4, 3, 24, 1),
    (33, 1000, 300, 8, 5, 64, 7),
    (48, 512, 1157, 5, 64, 16, 1),
    (130, 264, 256, 6, 4, 32, 40),
    (333, 1096, 129, 7, 5, 8, 23),
    (700, 2048, 384, 5, 3, 128, 300),
    (1500, 136, 512, 3, 8, 16, 1),
]


@pytest.mark.parametrize("act,out", [(F16, F16), (BF16, BF16), (BF16, F32), (F16, F32)])
@pytest.mark.parametrize("R,c_in,c_out,tau,n,rank,run", ADAPTER_CASES)
def test_adapters_whole_numbers(snn, R, c_in, c_out, tau, n, rank, run, act, out):
    """Scales are powers of two and the factors small, so that the second term is exact as well, and the sum of both has one correct
    value: |S| <= 2 c_in and |B (A x)| <= rank * c_in / 8 (one in 16 of A's elements is not 0) are far below 2^24."""
    g = _gen(R + c_in)
    layers, w, _ = _layers(snn, 1, c_in, c_out, tau, 990 + c_in, alpha=0.25)
    ad = snn.SnnConvAdapters(layers[0])
    layers[0].destroy()
    x = _whole(g, 2, R, c_in).to(act)
    a = (_whole(g, 1, n, rank, c_in) * (torch.rand(n, rank, c_in, generator=g, device="cuda") < 1 / 16)).to(act)
    b = _whole(g, 1, n, c_out, rank).to(act)
    scale = 2.0 ** torch.randint(-2, 2, (n,), generator=g, device="cuda").float()
    pick = torch.randint(-1, n + 1, ((R + run - 1) // run,), generator=g, device="cuda", dtype=torch.int32)
    adapter = pick.repeat_interleave(run)[:R].contiguous()
    y = ad.forward(x, adapter, a, b, scale, out=torch.empty(R, c_out, dtype=out, device="cuda"))
    ref = 0.25 * (x.double() @ w[0].T)
    for i in range(n):
        m = adapter == i
        ref[m] += scale[i].double() * (x[m].double() @ a[i].double().T) @ b[i].double().T
    assert (ref.float().double() == ref).all()
    assert torch.equal(y, ref.float().to(out))


@pytest.mark.parametrize("act", [F16, BF16])
@pytest.mark.parametrize("R,c_in,c_out,n,rank,run", [(1, 4096, 333, 2, 16, 1), (40, 1024, 512, 16, 32, 1), (600, 2048, 256, 3, 64, 250)])
def test_adapters_normal_values(snn, R, c_in, c_out, n, rank, run, act):
    g = _gen(11)
    layers, w, al = _layers(snn, 1, c_in, c_out, 5, 995)
    ad = snn.SnnConvAdapters(layers[0])
    x = torch.randn(R, c_in, generator=g, device="cuda").to(act)
    a = (torch.randn(n, rank, c_in, generator=g, device="cuda") / c_in ** 0.5).to(act)
    b = torch.randn(n, c_out, rank, generator=g, device="cuda").to(act)
    scale = torch.rand(n, generator=g, device="cuda")
    adapter = (torch.arange(R, device="cuda") // run % (n + 1)).to(torch.int32)   # (n: none)
    for out in (act, F32):
        y = ad.forward(x, adapter, a, b, scale, out=torch.empty(R, c_out, dtype=out, device="cuda"))
        ref = (x.double() @ w[0].T) * al[0].double()
        extra = torch.zeros_like(ref)
        for i in range(n):
            m = adapter == i
            h = x[m].double() @ a[i].double().T
            ref[m] += scale[i].double() * (h @ b[i].double().T)
            # the rank's products and sums are rounded once each; h itself as any sum of c_in products
            size = scale[i].double() * (h.abs() @ b[i].double().abs().T)
            hsize = scale[i].double() * (x[m].double().norm(dim=1, keepdim=True) * a[i].double().norm(dim=1)[None, :]) @ b[i].double().abs().T
            extra[m] = 2 * (rank + 2) * 2.0 ** -24 * size + c_in * 2.0 ** -23 * 6 * hsize
        bound = _bound(ref, x.double().norm(dim=1, keepdim=True), al[0].double(), c_in, out) + (1 + torch.finfo(out).eps) * extra
        assert ((y.double() - ref).abs() <= bound).all()


def test_adapters_infinities_stay_in_their_rows(snn):
    """An adapter that holds NaN, and rows that do, touch nobody else's outputs; one that nobody uses touches nothing."""
    R, c_in, c_out, n, rank = 21, 128, 70, 3, 8
    g = _gen(12)
    layers, w, _ = _layers(snn, 1, c_in, c_out, 5, 996, alpha=0.5)
    ad = snn.SnnConvAdapters(layers[0])
    x = _whole(g, 2, R, c_in).to(BF16)
    a, b = torch.zeros(n, rank, c_in, dtype=BF16, device="cuda"), torch.ones(n, c_out, rank, dtype=BF16, device="cuda")
    a[0, :, 0] = 1
    a[1] = float("nan")
    a[2], b[2] = float("inf"), float("nan")
    scale = torch.tensor([1.0, 1.0, float("nan")], device="cuda")
    adapter = (torch.arange(R, device="cuda") % 3).to(torch.int32)
    adapter[adapter == 2] = -1
    x[6, 9] = float("inf")
    y = ad.forward(x, adapter, a, b, scale, out_type=snn.OUT_F32)
    ref = 0.5 * (x.double() @ w[0].T) + torch.where(adapter[:, None] == 0, rank * x[:, :1].double(), 0.0)
    fine = (adapter != 1) & (torch.arange(R, device="cuda") != 6)
    assert torch.equal(y[fine], ref[fine].float())
    assert torch.isnan(y[adapter == 1]).all() and not torch.isfinite(y[6]).any()


def test_adapters_without_rows_or_adapters(snn):
    layers, w, al = _layers(snn, 1, 64, 48, 5, 997)
    ad = snn.SnnConvAdapters(layers[0])
    x = _whole(_gen(1), 8, 5, 64).to(F16)
    none = torch.empty(0, 8, 64, dtype=F16, device="cuda"), torch.empty(0, 48, 8, dtype=F16, device="cuda"), torch.empty(0, device="cuda")
    y = ad.forward(x, torch.zeros(5, dtype=torch.int32, device="cuda"), *none)
    assert torch.equal(y, ((x.double() @ w[0].T).float() * al[0]).to(F16))
    assert ad.forward(x[:0], torch.zeros(0, dtype=torch.int32, device="cuda"), *none).shape == (0, 48)


# ------------------------------------------------------------------------------------------------------------ together

@pytest.mark.parametrize("T", [1, 17, 400])
def test_a_block_of_experts_with_an_adapted_projection(snn, T):
    """As a model runs them: a projection with adapters, the router, both projections of the chosen experts, the weighted sum; eagerly, on
    another stream, and as a captured graph that is replayed on new inputs."""
    d, f, E, k, n, rank = 256, 512, 12, 3, 4, 16
    g = _gen(20 + T)
    shared, ws, als = _layers(snn, 1, d, d, 5, 1000)
    up, wu, alu = _layers(snn, E, d, f, 5, 1100)
    down, wd, ald = _layers(snn, E, f, d, 6, 1200)
    ad, ex_up, ex_down = snn.SnnConvAdapters(shared[0]), snn.SnnConvExperts(up), snn.SnnConvExperts(down)
    a = (torch.randn(n, rank, d, generator=g, device="cuda") / 16).to(BF16)
    b = torch.randn(n, d, rank, generator=g, device="cuda").to(BF16)
    scale = torch.rand(n, generator=g, device="cuda")
    gate = torch.randn(E, d, generator=g, device="cuda")

    def inputs(seed):
        gg = _gen(seed)
        return (torch.randn(T, d, generator=gg, device="cuda") / 16).to(BF16), torch.randint(-1, n, (T,), generator=gg, device="cuda", dtype=torch.int32)

    def block(x, adapter):
        h = ad.forward(x, adapter, a, b, scale)
        r = snn.route(h.float() @ gate.T, k)
        u = ex_up.forward(h, r.offsets, rows=r.rows)
        y = ex_down.forward(torch.relu(u), r.offsets)
        return h, r, y, snn.combine(y, r.slots, r.weights, out_type=snn.OUT_F32)

    def check(x, adapter, h, r, y, out):
        ref = (x.double() @ ws[0].T) * als[0].double()
        for i in range(n):
            m = adapter == i
            ref[m] += scale[i].double() * (x[m].double() @ a[i].double().T) @ b[i].double().T
        assert ((h.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 1e-3).all()
        _check_route(r, h.float() @ gate.T, k, True)
        hd, total = h.double(), torch.zeros(T, d, dtype=torch.float64, device="cuda")
        for t in range(T):
            for j in range(k):
                e = int(r.ids[t, j])
                u = ((hd[t] @ wu[e].T) * alu[e].double()).relu()
                total[t] += r.weights[t, j].double() * (u @ wd[e].T) * ald[e].double()
        # u rounded to bf16 (2^-8 of values that are summed with random signs), y as well
        size = total.abs().max()
        assert ((out.double() - total).norm() <= 2 * 2.0 ** -8 * total.norm()) and ((out.double() - total).abs().max() <= 0.05 * size)

    x, adapter = inputs(1)
    first = block(x, adapter)
    check(x, adapter, *first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = block(x, adapter)
    side.synchronize()
    assert torch.equal(other[3], first[3])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = block(x, adapter)
    for seed in (2, 3):
        nx, na = inputs(seed)
        x.copy_(nx)
        adapter.copy_(na)
        graph.replay()
        torch.cuda.synchronize()
        check(x, adapter, *captured)
        assert torch.equal(captured[3], block(x, adapter)[3])


def test_calls_on_two_streams_share_nothing(snn):
    """The same handle on two streams at once, each with a stream argument of its own."""
    layers, w, al = _layers(snn, 4, 512, 384, 5, 1300)
    ex, ad = snn.SnnConvExperts(layers), snn.SnnConvAdapters(layers[0])
    g = _gen(30)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    xs = [_whole(g, 2, 300, 512).to(BF16) for _ in streams]
    offs = [torch.tensor(o, dtype=torch.int32, device="cuda") for o in ([0, 100, 100, 250, 300], [0, 3, 290, 290, 300])]
    a = (_whole(g, 1, 2, 16, 512)).to(BF16)
    b = (_whole(g, 1, 2, 384, 16)).to(BF16)
    scale = torch.ones(2, device="cuda")
    adapters = [torch.randint(0, 2, (300,), generator=g, device="cuda", dtype=torch.int32) for _ in streams]
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        for s, x, o, ia in zip(streams, xs, offs, adapters):
            got.append((ex.forward(x, o, stream=s), ad.forward(x, ia, a, b, scale, stream=s), snn.route(x[:, :40].contiguous(), 4, stream=s)))
    torch.cuda.synchronize()
    for i, (y, z, r) in enumerate(got):
        x, o, ia = xs[i % 2], offs[i % 2].tolist(), adapters[i % 2]
        for e in range(4):
            part = slice(o[e], o[e + 1])
            assert torch.equal(y[part], ((x[part].double() @ w[e].T).float() * al[e]).to(BF16))
        assert torch.equal(z, got[i % 2][1])
        assert torch.equal(r.rows, got[i % 2][2].rows)

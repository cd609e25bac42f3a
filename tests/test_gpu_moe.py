"""A whole mixture of experts for a few tokens, against plain arithmetic in 64 bits and against the calls that it stands for.

Whole numbers: top_k experts of equal logits (weights 1 / top_k, a power of two), no activation or the ramp, scales that are powers of two, few enough
channels that every sum is exact in fp32: one correct value each, compared bit by bit.  Normal values: the tolerance is derived in _tolerance."""
import threading

import pytest
import torch

from test_gpu_projections import BF16, F16, F32, _gen, _layers, _whole, snn  # noqa: F401
from test_gpu_scaled import _fn64

pytestmark = pytest.mark.gpu


class Block:
    """Experts and their decoded weights in 64 bits."""

    def __init__(self, snn, E, c_in, hidden, c_out, tau, seed, gated, fn, alpha=None):
        def make(a, b, s):
            layers, w, al = _layers(snn, E, a, b, tau, s, alpha=alpha)
            ex = snn.SnnConvExperts(layers)
            for l in layers:
                l.destroy()
            return ex, w, [x.double() for x in al]
        self.snn, self.E, self.fn, self.sizes = snn, E, fn, (c_in, hidden, c_out)
        self.up, self.down = make(c_in, hidden, seed), make(hidden, c_out, seed + 1000)
        self.gate = make(c_in, hidden, seed + 2000) if gated else None
        self.h = snn.SnnConvMoe(self.up[0], self.down[0], gate=self.gate and self.gate[0], fn=getattr(snn, fn))

    def first(self, x, e):
        """The two factors and their product in 64 bits."""
        u = (x @ self.up[1][e].T) * self.up[2][e]
        if self.gate is None:
            return _fn64(self.fn, u), None, u
        v = (x @ self.gate[1][e].T) * self.gate[2][e]
        return _fn64(self.fn, v) * u, v, u

    def second(self, h, e):
        return (h @ self.down[1][e].T) * self.down[2][e]


def _choices(logits, k, normalise):
    """(token, expert, weight) of each choice, in 64 bits."""
    v, out = logits.double().cpu(), []
    for t in range(v.shape[0]):
        able = [e for e in range(v.shape[1]) if v[t, e] > -float("inf")]
        best = sorted(able, key=lambda e: (-v[t, e].item(), e))[:k]
        if best:
            top = v[t, best[0]]
            total = sum(torch.exp(v[t, e] - top).item() for e in (best if normalise else able))
            out += [(t, e, torch.exp(v[t, e] - top).item() / total) for e in best]
    return out


def _whole_case(snn, T, E, k, c_in, hidden, c_out, gated, act, out, tau=5):
    b = Block(snn, E, c_in, hidden, c_out, tau, 3000 + c_in + hidden, gated, "FN_RELU" if gated else "FN_NONE", alpha=0.25)
    g = _gen(T + E)
    x = _whole(g, 1, T, c_in).to(act)
    who = torch.rand(T, E, generator=g, device="cuda").argsort(1)[:, :k]
    logits = torch.full((T, E), -float("inf"), device="cuda").scatter_(1, who, 1.5)
    y = b.h.forward(x, logits, k, out=torch.empty(T, c_out, dtype=out, device="cuda"))
    ref, size = torch.zeros(T, c_out, dtype=torch.float64, device="cuda"), 0.0
    for t in range(T):
        for e in who[t].tolist():
            h = b.first(x[t:t + 1].double(), e)[0]
            if out != F32:   # two bf16 numbers hold the product
                first = (h.float().view(torch.int32) & -65536).view(F32).double()
                assert torch.equal((h - first).to(BF16).double(), h - first)
            ref[t] += b.second(h, e)[0] / k
            size = max(size, h.abs().sum().item())
    assert size < 2.0 ** 18   # (steps of 2^-8 at least: 2^-4 from both scales, 2^-4 from a sixteenth)
    assert torch.equal(y, ref.float().to(out))


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 8, 2), (3, 33, 4), (5, 60, 8), (8, 64, 2), (8, 300, 16), (7, 1000, 4), (9, 64, 2), (17, 5, 4), (40, 16, 1),
                                   (64, 64, 4), (64, 16, 16), (33, 256, 8)])
@pytest.mark.parametrize("gated", [True, False])
def test_whole_numbers_of_tokens_and_experts(snn, T, E, k, gated):  # noqa: F811
    _whole_case(snn, T, E, k, 72, 40, 70, gated, BF16, F32)


@pytest.mark.parametrize("c_in,hidden,c_out", [(8, 8, 1), (64, 256, 33), (264, 72, 129), (1000, 264, 64), (256, 1096, 31), (2048, 128, 300), (520, 520, 1003)])
@pytest.mark.parametrize("T", [1, 6, 20])
@pytest.mark.parametrize("act,out,gated", [(BF16, BF16, False), (F16, F16, False), (F16, F32, True), (BF16, F32, False)])
def test_whole_numbers_of_sizes(snn, c_in, hidden, c_out, T, act, out, gated):  # noqa: F811
    _whole_case(snn, T, 4, 2, c_in, hidden, c_out, gated, act, out, tau=4)


def _tolerance(b, x, choices, out, ref):
    """First projections: fp32 sums of C numbers, at most C additions, each off by at most 2^-23 of a partial sum, which stays within 6 |x|_2 (six standard
    deviations of a random walk), and two roundings.  The functions' slopes are at most 1.13, and they come out within 2^-20 of the value; then the
    product, and what the bf16 numbers leave (2^-16, or 2^-24).  All of h may be off by as much, in the worst signs.  Second projection and the sum over the choices: as the
    first, of H numbers in three parts, plus two roundings a choice; the weights within 2^-18 (exponentials of rounded differences up to 12, k sums); half a step
    of the output."""
    tol = torch.zeros_like(ref)
    C, H, _ = b.sizes
    for t, e, w in choices:
        xe = x[t:t + 1].double()
        h, v, u = b.first(xe, e)
        first = C * 2.0 ** -23 * 6 * xe.norm()
        du = first * b.up[2][e] + 2.0 ** -23 * u.abs()
        if v is None:
            dh = 1.13 * du + 2.0 ** -20 * h.abs()
        else:
            dv = first * b.gate[2][e] + 2.0 ** -23 * v.abs()
            f = _fn64(b.fn, v).abs()
            dh = 1.13 * dv * u.abs() + (f + 1.13 * dv) * du + 2.0 ** -19 * h.abs()
        dh = dh + (2.0 ** -24 if out == F32 else 2.0 ** -16) * h.abs()
        y = b.second(h, e).abs()
        tol[t] += (w * (b.down[2][e] * (dh.sum() + 3 * H * 2.0 ** -23 * 6 * h.norm()) + 2.0 ** -17 * y))[0]
    return tol + (torch.finfo(out).eps / 2 + 2.0 ** -22) * ref.abs() + 2.0 ** -24


def _check(b, x, logits, k, normalise, y):
    choices = _choices(logits, k, normalise)
    ref = torch.zeros(len(x), b.sizes[2], dtype=torch.float64, device="cuda")
    for t, e, w in choices:
        ref[t] += w * b.second(b.first(x[t:t + 1].double(), e)[0], e)[0]
    assert ((y.double() - ref).abs() <= _tolerance(b, x, choices, y.dtype, ref)).all()
    return ref


@pytest.mark.parametrize("fn", ["FN_SILU", "FN_GELU", "FN_RELU", "FN_NONE"])
@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("T,E,k,c_in,hidden,c_out", [(1, 8, 2, 1024, 512, 640), (6, 20, 3, 328, 200, 130), (21, 12, 4, 512, 264, 200)])
@pytest.mark.parametrize("normalise", [True, False])
def test_normal_values(snn, fn, gated, T, E, k, c_in, hidden, c_out, normalise):  # noqa: F811
    b = Block(snn, E, c_in, hidden, c_out, 5, 3100, gated, fn)
    g = _gen(T)
    x, logits = torch.randn(T, c_in, generator=g, device="cuda").to(BF16), torch.randn(T, E, generator=g, device="cuda")
    for out in (BF16, F32):
        _check(b, x, logits, k, normalise, b.h.forward(x, logits, k, normalise=normalise, out=torch.empty(T, c_out, dtype=out, device="cuda")))
    for dtype in (F16, BF16):   # logits of 16 bits: many are equal
        few = logits.to(dtype)
        _check(b, x, few, k, normalise, b.h.forward(x, few, k, normalise=normalise, out_type=snn.OUT_F32))


@pytest.mark.parametrize("T", [8, 30])
def test_masks(snn, T):  # noqa: F811
    """Tokens without any expert, fewer than top_k, NaN, equal logits, the type's lowest value, infinities."""
    b = Block(snn, 12, 136, 64, 72, 5, 3200, True, "FN_SILU")
    g = _gen(T)
    x, logits = torch.randn(T, 136, generator=g, device="cuda").to(F16), torch.randn(T, 12, generator=g, device="cuda")
    logits[0] = -float("inf")
    logits[1] = float("nan")
    logits[2, 2:] = -float("inf")
    logits[3] = 0.0
    logits[4] = torch.finfo(F32).min
    logits[5, ::2] = float("nan")
    logits[6] = torch.finfo(F32).min
    logits[6, 7] = 1.0
    y = b.h.forward(x, logits, 4, out_type=snn.OUT_F32)
    assert (y[:2] == 0).all()
    _check(b, x, logits, 4, True, y)
    logits[7, 3] = float("inf")   # that expert alone counts
    again = b.h.forward(x, logits, 4, out_type=snn.OUT_F32)
    only = torch.full_like(logits, -float("inf"))
    only[7, 3] = 0.0
    assert torch.equal(again[7], b.h.forward(x, only, 1, out_type=snn.OUT_F32)[7])
    rest = [t for t in range(T) if t != 7]
    assert torch.equal(again[rest], y[rest])
    nobody = torch.full((T, 12), -float("inf"), device="cuda")
    assert (b.h.forward(x, nobody, 2) == 0).all()


@pytest.mark.parametrize("T", [8, 24])
def test_infinities_and_nan_stay_in_their_tokens(snn, T):  # noqa: F811
    b = Block(snn, 4, 136, 64, 72, 5, 3300, True, "FN_SILU")
    g = _gen(T)
    x, logits = torch.randn(T, 136, generator=g, device="cuda").to(BF16), torch.randn(T, 4, generator=g, device="cuda")
    clean = b.h.forward(x, logits, 2, out_type=snn.OUT_F32)
    x[1, 3], x[T - 1, 100], x[4, 0] = float("nan"), float("inf"), -float("inf")
    y = b.h.forward(x, logits, 2, out_type=snn.OUT_F32)
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[[1, 4, T - 1]] = False
    assert torch.equal(y[keep], clean[keep]) and torch.isnan(y[1]).all() and not torch.isfinite(y[4]).any() and not torch.isfinite(y[T - 1]).any()


@pytest.mark.parametrize("T", [5, 64])
def test_strides(snn, T):  # noqa: F811
    b = Block(snn, 10, 136, 72, 75, 5, 3400, True, "FN_GELU")
    g = _gen(T)
    x = torch.randn(T, 160, generator=g, device="cuda").to(BF16)[:, 8:144]
    logits = torch.randn(T, 15, generator=g, device="cuda")[:, 3:13]
    buffer = torch.full((T, 90), 7.0, dtype=F16, device="cuda")
    out = buffer[:, 5:80]
    assert b.h.forward(x, logits, 3, out=out) is out
    assert torch.equal(out, b.h.forward(x.contiguous(), logits.contiguous(), 3, out_type=snn.OUT_F16))
    assert (buffer[:, :5] == 7).all() and (buffer[:, 80:] == 7).all()
    _check(b, x, logits, 3, True, out)


@pytest.mark.parametrize("T", [1, 8, 9, 64])
@pytest.mark.parametrize("fn,gated", [("FN_SILU", True), ("FN_GELU", False)])
def test_the_calls_that_it_stands_for(snn, T, fn, gated):  # noqa: F811
    """Router, experts, activation, experts and weighted sum with the same handles, in fp32 between them where the calls can: both within the tolerance, and of
    more tokens than the mixture takes."""
    b = Block(snn, 16, 520, 264, 200, 5, 3500, gated, fn)
    g = _gen(T)

    def calls(x, logits):
        r = snn.route(logits, 4)
        up = b.up[0].forward(x, r.offsets, rows=r.rows, out_type=snn.OUT_F32)
        gate = b.gate[0].forward(x, r.offsets, rows=r.rows, out_type=snn.OUT_F32) if gated else None
        h = snn.activate(up, gate=gate, fn=getattr(snn, fn), out_type=snn.OUT_F16)
        return r, h, snn.combine(b.down[0].forward(h, r.offsets, out_type=snn.OUT_F32), r.slots, r.weights)

    x, logits = torch.randn(T, 520, generator=g, device="cuda").to(F16), torch.randn(T, 16, generator=g, device="cuda")
    y = b.h.forward(x, logits, 4, out_type=snn.OUT_F32)
    ref = _check(b, x, logits, 4, True, y)
    r, h, z = calls(x, logits)
    # h in fp16: half a step of each value, in the worst signs
    extra = torch.zeros_like(ref)
    for t, e, w in _choices(logits, 4, True):
        extra[t] += w * b.down[2][e] * (2.0 ** -11 * b.first(x[t:t + 1].double(), e)[0].abs().sum() + 264 * 2.0 ** -25)
    assert ((z.double() - ref).abs() <= extra + _tolerance(b, x, _choices(logits, 4, True), F32, ref)).all()
    more = torch.randn(65, 520, generator=g, device="cuda").to(F16)
    with pytest.raises(snn.SnnError, match="65 tokens") as ei:
        b.h.forward(more, torch.zeros(65, 16, device="cuda"), 4)
    assert ei.value.status == 2
    assert calls(more, torch.randn(65, 16, generator=g, device="cuda"))[2].shape == (65, 200)


def test_scaled_experts_behind_the_router(snn):  # noqa: F811
    """A mixture of 8-bit experts: route, quantise by the router's index, products, activation into 8 bits, products, weighted sum."""
    T, E, k, c_in, hidden, c_out = 90, 6, 2, 272, 144, 100
    g = _gen(11)
    w = [snn.quantise(torch.randn(E * b, a, generator=g, device="cuda")) for a, b in ((c_in, hidden), (c_in, hidden), (hidden, c_out))]
    values = [q.values.float().reshape(E, -1, q.values.shape[1]).to(torch.float8_e4m3fn) for q in w]   # (one scale, 1, for all blocks)
    gate, up, down = (snn.SnnConvScaled(v, torch.full((E, -(-v.shape[1] // 128), -(-v.shape[2] // 128)), 2.0 ** -12, device="cuda")) for v in values)
    x, logits = torch.randn(T, c_in, generator=g, device="cuda").to(BF16), torch.randn(T, E, generator=g, device="cuda")
    r = snn.route(logits, k)
    q = snn.quantise(x, rows=r.rows)
    h = snn.quantise(up.forward(*q, offsets=r.offsets, out_type=snn.OUT_F32), gate=gate.forward(*q, offsets=r.offsets, out_type=snn.OUT_F32), fn=snn.FN_SILU)
    out = snn.combine(down.forward(*h, offsets=r.offsets, out_type=snn.OUT_F32), r.slots, r.weights)
    wide = lambda s, n: s.double().repeat_interleave(128, 1)[:, :n]  # noqa: E731
    a, b = q.values.double() * wide(q.scales, c_in), h.values.double() * wide(h.scales, hidden)
    ref = torch.zeros(T, c_out, dtype=torch.float64, device="cuda")
    offsets, rows = r.offsets.tolist(), r.rows.tolist()
    weight = {(s, t): r.weights[t, j].item() for t in range(T) for j, s in enumerate(r.slots[t].tolist())}
    for e in range(E):
        part = slice(offsets[e], offsets[e + 1])
        v, u = (a[part] @ values[i][e].double().T * 2.0 ** -12 for i in (0, 1))
        # an eighth of a bit of 8: half a step (2^-4) of each value, or of the smallest normal one, by its block's scale
        m = _fn64("FN_SILU", v) * u
        assert ((b[part] - m).abs() <= (2.0 ** -4 + 2.0 ** -10) * m.abs() + 2.0 ** -10 * wide(h.scales[part], hidden)).all()
        y = b[part] @ values[2][e].double().T * 2.0 ** -12
        for i in range(offsets[e], offsets[e + 1]):
            ref[rows[i]] += weight[(i, rows[i])] * y[i - offsets[e]]
    # (fp32 sums of the second projection and of the choices: 144 + 8 additions, relative to the sum of the magnitudes)
    size = ref.abs().max() + (b.abs().sum(1).max() * 448 * 2.0 ** -12)
    assert ((out.double() - ref).abs() <= 160 * 2.0 ** -23 * size).all()


@pytest.mark.parametrize("T", [3, 20])
def test_captured_graphs_and_streams(snn, T):  # noqa: F811
    """Two graphs of one handle, each with a workspace of its own, replayed side by side on other inputs; twice the same bits."""
    b = Block(snn, 16, 264, 136, 96, 5, 3600, True, "FN_SILU")
    g, graphs = _gen(T), []
    for _ in range(2):
        x, logits, y = torch.zeros(T, 264, dtype=BF16, device="cuda"), torch.zeros(T, 16, device="cuda"), torch.empty(T, 96, dtype=F32, device="cuda")
        b.h.forward(x, logits, 4, out=y)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            b.h.forward(x, logits, 4, out=y)
        graphs.append((graph, x, logits, y, torch.cuda.Stream()))
    for _ in range(4):
        for _, x, logits, _, _ in graphs:
            x.copy_(torch.randn(T, 264, generator=g, device="cuda"))
            logits.copy_(torch.randn(T, 16, generator=g, device="cuda"))
        torch.cuda.synchronize()
        for graph, _, _, _, s in graphs:
            with torch.cuda.stream(s):
                for _ in range(5):
                    graph.replay()
        torch.cuda.synchronize()
        for _, x, logits, y, _ in graphs:
            assert torch.equal(y, b.h.forward(x, logits, 4, out_type=snn.OUT_F32))
            _check(b, x, logits, 4, True, y)


def test_two_threads(snn):  # noqa: F811
    b = Block(snn, 16, 264, 136, 96, 5, 3700, True, "FN_SILU")
    g = _gen(4)
    inputs = [(torch.randn(t, 264, generator=g, device="cuda").to(BF16), torch.randn(t, 16, generator=g, device="cuda")) for t in (7, 40)]
    want = [b.h.forward(x, l, 4) for x, l in inputs]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            got = [b.h.forward(*inputs[i], 4) for _ in range(50)]
        s.synchronize()
        wrong.extend(i for y in got if not torch.equal(y, want[i]))
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_what_does_not_fit(snn):  # noqa: F811
    def experts(count, a, b):
        layers, _, _ = _layers(snn, 1, a, b, 3, 3800)
        return snn.SnnConvExperts(layers * count)
    up, down = experts(3, 64, 32), experts(3, 32, 16)
    for bad in (dict(down=experts(3, 64, 16)), dict(down=experts(2, 32, 16)), dict(gate=experts(3, 64, 40)), dict(gate=experts(2, 64, 32)), dict(gate=experts(3, 72, 32)), dict(fn=9)):
        args = dict(up=up, down=down, gate=None, fn=snn.FN_SILU)
        args.update(bad)
        with pytest.raises(snn.SnnError) as ei:
            snn.SnnConvMoe(**args)
        assert ei.value.status == 1
    h = snn.SnnConvMoe(up, down)
    x, logits = torch.zeros(2, 64, dtype=F16, device="cuda"), torch.zeros(2, 3, device="cuda")
    for args in ((x.float(), logits, 1), (x[:, :56], logits, 1), (x, logits[:, :2], 1), (x, logits[:1], 1), (x, logits, 0), (x, logits, 4), (x, logits.double(), 1),
                 (x, logits.cpu(), 1), (x.cpu(), logits, 1)):
        with pytest.raises(snn.SnnError) as ei:
            h.forward(*args)
        assert ei.value.status == 1
    assert h.forward(x[:0], logits[:0], 1).shape == (0, 16)
    down.destroy()
    with pytest.raises(snn.SnnError, match="destroyed"):
        h.forward(x, logits, 1)

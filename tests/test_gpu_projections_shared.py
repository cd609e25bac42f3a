"""Handles of the projections that several callers use at once: streams of one thread, and threads with streams of their own; and experts from layers
of different codebooks, index widths and activation types."""
import threading

import numpy as np
import pytest
import torch

from test_gpu_projections import BF16, F16, F32, _check_route, _gen, _layers, _whole, snn  # noqa: F401

pytestmark = pytest.mark.gpu

C, K, E, TOP, RANK = 512, 384, 4, 3, 16


class Caller:
    """Inputs of one caller's and the one right answer to each of its calls (whole numbers: the sums are exact)."""

    def __init__(self, w, al, a, b, sizes, seed):
        g = _gen(seed)
        R = sum(sizes)
        self.x = _whole(g, 2, R, C).to(BF16)
        self.offsets = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32, device="cuda")
        self.adapter = torch.randint(-1, len(a), (R,), generator=g, device="cuda", dtype=torch.int32)
        self.logits = torch.randn(R, 40, generator=g, device="cuda")
        self.slots = torch.randint(-1, R, (R, TOP), generator=g, device="cuda", dtype=torch.int32)
        self.weights = torch.randint(-2, 3, (R, TOP), generator=g, device="cuda").float()
        x, parts, lo = self.x.double(), [], 0
        for e, n in enumerate(sizes):
            parts.append(((x[lo:lo + n] @ w[e].T).float() * al[e]).to(BF16))
            lo += n
        self.y = torch.cat(parts)
        z = 0.25 * (x @ w[0].T)
        for i in range(len(a)):
            m = self.adapter == i
            z[m] += (x[m] @ a[i].double().T) @ b[i].double().T
        self.z = z.to(F32)
        assert torch.equal(self.z.double(), z)
        self.sum = (((self.slots >= 0) * self.weights).double().unsqueeze(2) * x[self.slots.clamp(min=0).long()]).sum(1).to(F32)

    def check(self, y, z, r, s):
        assert torch.equal(y, self.y)
        assert torch.equal(z, self.z)
        _check_route(r, self.logits, TOP, True)
        assert torch.equal(s, self.sum)


@pytest.fixture(params=["few", "many"])
def handles(snn, request, monkeypatch):  # noqa: F811
    monkeypatch.setenv("SNN_FORCE_ROWS", request.param)
    layers, w, al = _layers(snn, E, C, K, 5, 2400, alpha=0.25)
    g = _gen(31)
    a, b = _whole(g, 1, 2, RANK, C).to(BF16), _whole(g, 1, 2, K, RANK).to(BF16)
    yield snn.SnnConvExperts(layers), snn.SnnConvAdapters(layers[0]), w, al, a, b, torch.ones(2, device="cuda")
    torch.cuda.synchronize()


SIZES = ([100, 0, 150, 50], [3, 287, 0, 10])


def test_two_streams(snn, handles):  # noqa: F811
    """Calls with a stream argument: inputs are there before, and stay until all is done; outputs are each call's own."""
    ex, ad, w, al, a, b, scale = handles
    callers = [Caller(w, al, a, b, sizes, 32 + i) for i, sizes in enumerate(SIZES)]
    streams = [torch.cuda.Stream() for _ in callers]
    torch.cuda.synchronize()
    got = []
    for _ in range(6):
        for s, c in zip(streams, callers):
            got.append((c, ex.forward(c.x, c.offsets, stream=s), ad.forward(c.x, c.adapter, a, b, scale, out_type=snn.OUT_F32, stream=s),
                        snn.route(c.logits, TOP, stream=s), snn.combine(c.x, c.slots, c.weights, out_type=snn.OUT_F32, stream=s)))
    torch.cuda.synchronize()
    for c, *results in got:
        c.check(*results)


def test_two_threads(snn, handles):  # noqa: F811
    """One handle, two host threads, each on its own stream: by the checks in C++ (out given) and those in Python."""
    ex, ad, w, al, a, b, scale = handles
    callers = [Caller(w, al, a, b, sizes, 42 + i) for i, sizes in enumerate(SIZES)]
    torch.cuda.synchronize()
    start, failed = threading.Barrier(len(callers), timeout=60), []

    def run(c):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                start.wait()
                got = []
                for i in range(12):
                    if i % 2:
                        y, z, s = torch.empty_like(c.y), torch.empty_like(c.z), torch.empty_like(c.sum)
                        r = snn.alloc_route(len(c.x), c.logits.shape[1], TOP)
                        ex.forward(c.x, c.offsets, out=y)
                        ad.forward(c.x, c.adapter, a, b, scale, out=z)
                        snn.route(c.logits, TOP, out=r)
                        snn.combine(c.x, c.slots, c.weights, out=s)
                    else:
                        y, z = ex.forward(c.x, c.offsets), ad.forward(c.x, c.adapter, a, b, scale, out_type=snn.OUT_F32)
                        r, s = snn.route(c.logits, TOP), snn.combine(c.x, c.slots, c.weights, out_type=snn.OUT_F32)
                    got.append((y, z, r, s))
                stream.synchronize()
                for results in got:
                    c.check(*results)
        except BaseException as e:   # (told by the test's own thread)
            failed.append(e)

    threads = [threading.Thread(target=run, args=(c,)) for c in callers]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    if failed:
        raise failed[0]


@pytest.mark.parametrize("act", [F16, BF16])
def test_experts_of_different_layers(snn, act, monkeypatch):  # noqa: F811
    """Layers of every index width and of both activation types, one create: the weights are what counts."""
    c_in, c_out = 136, 150
    kinds = [(tau, act_type) for tau in range(1, 9) for act_type in (snn.ACT_BIN, snn.ACT_F16)]
    layers, w, al = [], [], []
    for i, (tau, act_type) in enumerate(kinds):
        one = _layers(snn, 1, c_in, c_out, tau, 2500 + i, act_type=act_type)
        for all_of, new in zip((layers, w, al), one):
            all_of += new
    ex = snn.SnnConvExperts(layers)
    sizes = [3 * i % 11 + (40 if i == 5 else 0) for i in range(len(kinds))]
    x = _whole(_gen(50), 8, sum(sizes), c_in).to(act)
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32, device="cuda")
    for force in ("few", "many"):
        monkeypatch.setenv("SNN_FORCE_ROWS", force)
        y = ex.forward(x, offsets, out_type=snn.OUT_F32)
        lo = 0
        for e, n in enumerate(sizes):
            assert torch.equal(y[lo:lo + n], (x[lo:lo + n].double() @ w[e].T).float() * al[e]), f"expert {e}, {kinds[e]}, {force}"
            lo += n
    for kind, l in zip(kinds, layers):   # (one projection with adapters from each)
        ad, n = snn.SnnConvAdapters(l), sizes[5]
        i = layers.index(l)
        a, b = torch.zeros(1, 8, c_in, dtype=act, device="cuda"), torch.zeros(1, c_out, 8, dtype=act, device="cuda")
        z = ad.forward(x[:n], torch.zeros(n, dtype=torch.int32, device="cuda"), a, b, torch.ones(1, device="cuda"), out_type=snn.OUT_F32)
        assert torch.equal(z, (x[:n].double() @ w[i].T).float() * al[i]), kind

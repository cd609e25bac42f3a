"""The projections where offsets and counts pass 32 bits, the calls that are refused for their size, and calls on the branches of one
captured graph."""
import pytest
import torch

from test_gpu_projections import BF16, F16, F32, _check_route, _gen, _layers, _whole, snn  # noqa: F401

pytestmark = pytest.mark.gpu

R, LD = 70001, 32768   # R * LD is above 2^31


def _free(gigabytes):
    if torch.cuda.mem_get_info()[0] < gigabytes << 30:
        pytest.skip(f"less than {gigabytes} GB free")


def _wide(dtype, fill=None):
    t = torch.empty(R, LD, dtype=dtype, device="cuda")
    return t if fill is None else t.fill_(fill)


@pytest.mark.parametrize("force", ["few", "many"])
def test_rows_far_apart(snn, force, monkeypatch):
    _free(16)
    monkeypatch.setenv("SNN_FORCE_ROWS", force)
    c_in, c_out, n, rank = 64, 72, 3, 16
    g = _gen(40)
    layers, w, _ = _layers(snn, 3, c_in, c_out, 5, 1800, alpha=0.25)
    ex, ad = snn.SnnConvExperts(layers), snn.SnnConvAdapters(layers[0])
    values = _whole(g, 4, R, c_in)
    x = _wide(BF16)[:, :c_in]
    x.copy_(values)
    whole_out = _wide(BF16, 3.0)
    out = whole_out[:, 8:8 + c_out]
    cuts = [0, 30000, 30007, R]
    offsets = torch.tensor(cuts, dtype=torch.int32, device="cuda")

    def check(from_rows):
        for e in range(3):
            part = slice(cuts[e], cuts[e + 1])
            assert torch.equal(out[part], (0.25 * (from_rows[part] @ w[e].T)).to(BF16)), f"expert {e}"
        assert (whole_out[:, :8] == 3).all() and (whole_out[-5:, 8 + c_out:] == 3).all()

    ex.forward(x, offsets, out=out)
    check(values)
    index = torch.randperm(R, generator=g, device="cuda")
    ex.forward(x, offsets, rows=index.to(torch.int32), out=out)
    check(values[index])

    a, b = _whole(g, 1, n, rank, c_in).to(BF16), _whole(g, 1, n, c_out, rank).to(BF16)
    adapter = (torch.arange(R, device="cuda") // 9000 % (n + 1)).to(torch.int32)
    ad.forward(x, adapter, a, b, torch.ones(n, device="cuda"), out=out)
    ref = 0.25 * (values @ w[0].T)
    for i in range(n):
        ref[adapter == i] += (values[adapter == i] @ a[i].double().T) @ b[i].double().T
    assert torch.equal(out, ref.float().to(BF16))


def test_logits_and_sums_far_apart(snn):
    _free(24)
    g = _gen(41)
    E, k, c = 24, 3, 40
    logits = _wide(F16)[:, 8:8 + E]
    logits.copy_(torch.rand(R, E, generator=g, device="cuda").argsort(1))   # (no two equal in a row)
    r = snn.route(logits, k)
    ids = torch.sort(logits.float(), dim=1, descending=True).indices[:, :k]
    assert torch.equal(r.ids, ids.to(torch.int32))
    order = torch.sort(ids.reshape(-1), stable=True).indices
    assert torch.equal(r.rows, (order // k).to(torch.int32))
    for first in (0, 1):   # whole eights, and columns that no vector fits
        y, out = _wide(F16)[:, first:first + c], _wide(F16)[:, first:first + c]
        values = _whole(g, 8, R, c)
        y.copy_(values)
        slots = torch.randint(-1, R, (R, k), generator=g, device="cuda", dtype=torch.int32)
        weights = torch.randint(-2, 3, (R, k), generator=g, device="cuda").float()
        snn.combine(y, slots, weights, out=out)
        ref = ((slots >= 0).double() * weights.double()).unsqueeze(2) * values[slots.clamp(min=0).long()]
        assert torch.equal(out, ref.sum(1).to(F16))


def test_route_of_so_many_tokens_that_the_rows_behind_the_last_pass_32_bits(snn):
    """What follows the last row is written by all CTAs, 512 places each at a time: here behind 2^31."""
    _free(12)
    T, none = 240_000_000, 1000
    logits = torch.zeros(T, 1, dtype=F16, device="cuda")
    logits[T - none:] = float("-inf")
    r = snn.route(logits, 1)
    n = T - none
    assert r.offsets.tolist() == [0, n]
    count = torch.arange(n, dtype=torch.int32, device="cuda")
    assert torch.equal(r.rows[:n], count) and torch.equal(r.slots[:n, 0], count)
    assert (r.rows[n:] == -1).all() and (r.slots[n:] == -1).all() and (r.ids[n:] == -1).all() and (r.ids[:n] == 0).all()
    assert (r.weights[:n] == 1).all() and (r.weights[n:] == 0).all()


def test_sizes_that_are_refused(snn):
    """Before anything is launched: the pointers are good for far less."""
    layers, _, _ = _layers(snn, 2, 64, 256, 5, 1850)
    ex, ad = snn.SnnConvExperts(layers), snn.SnnConvAdapters(layers[0])
    lib = snn.load_library()
    t = torch.zeros(4096, device="cuda")
    p = t.data_ptr()
    before = snn.kernel_launches()
    for rows in ((1 << 30) + 1, (1 << 31) - 1):
        st = lib.snn_conv_experts_forward(ex._h, p, snn.ACT_F16, 16, 64, None, p, rows, p, snn.OUT_F32, 256, None)
        assert st == 2 and b"split the call" in lib.snn_last_error()
        st = lib.snn_conv_adapters_forward(ad._h, p, snn.ACT_F16, rows, 64, p, p, p, p, 1, 8, p, p, snn.OUT_F32, 256, None)
        assert st == 2 and b"split the call" in lib.snn_last_error()
    assert snn.kernel_launches() == before


def test_branches_of_one_graph(snn):
    """Two branches of a captured graph run the same handles side by side, each with what it writes of its own, and meet in a third call;
    the graph is replayed on new inputs."""
    T, d, E, k = 260, 256, 6, 2
    layers, w, al = _layers(snn, E, d, d, 5, 1900)
    ex, ad = snn.SnnConvExperts(layers), snn.SnnConvAdapters(layers[0])
    g = _gen(42)
    a, b = _whole(g, 1, 2, 8, d).to(BF16), _whole(g, 1, 2, d, 8).to(BF16)
    scale = torch.ones(2, device="cuda")
    adapter = (torch.arange(T, device="cuda") // 50 % 3).to(torch.int32)
    xs = [torch.zeros(T, d, dtype=BF16, device="cuda") for _ in range(2)]
    logits = [torch.zeros(T, E, device="cuda") for _ in range(2)]

    def branch(x, l):
        h = ad.forward(x, adapter, a, b, scale)
        r = snn.route(l, k)
        return r, h, snn.combine(ex.forward(x, r.offsets, rows=r.rows), r.slots, r.weights, out_type=snn.OUT_F32)

    def run(side):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        with torch.cuda.stream(side):
            other = branch(xs[1], logits[1])
        one = branch(xs[0], logits[0])
        main.wait_stream(side)
        both = snn.combine(torch.cat([one[2], other[2]]), torch.arange(2 * T, device="cuda", dtype=torch.int32).reshape(2, T).T.contiguous(),
                           torch.ones(T, 2, device="cuda"))
        return one, other, both

    def draw(seed):
        gg = _gen(seed)
        for x, l in zip(xs, logits):
            x.copy_(_whole(gg, 2, T, d))
            l.copy_(torch.randn(T, E, generator=gg, device="cuda"))

    side = torch.cuda.Stream()
    draw(1)
    run(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run(side)
    for seed in (2, 3):
        draw(seed)
        graph.replay()
        torch.cuda.synchronize()
        for i in range(2):
            alone = branch(xs[i], logits[i])
            _check_route(captured[i][0], logits[i], k, True)
            assert torch.equal(captured[i][1], alone[1]) and torch.equal(captured[i][2], alone[2])
        assert torch.equal(captured[2], captured[0][2] + captured[1][2])


@pytest.mark.parametrize("T", [128, 6143, 6144, 6145, 9999])
@pytest.mark.parametrize("E,k", [(1, 1), (3, 2), (37, 4), (130, 8), (1023, 3)])
def test_counts_of_many_groups_of_tokens(snn, T, E, k):
    """Up to 96 groups of 64 tokens every group adds up the others' counts, four experts' in a word; beyond, a launch of their own does."""
    g = _gen(T + E)
    logits = torch.rand(T, E, generator=g, device="cuda").argsort(1).float()   # (no two equal in a row)
    logits[torch.rand(T, generator=g, device="cuda") < 0.1] = float("-inf")    # (nobody for a tenth of the tokens)
    r = snn.route(logits, k)
    able = torch.isfinite(logits[:, 0])
    ids = torch.sort(logits, dim=1, descending=True).indices[:, :k]
    assert torch.equal(r.ids, torch.where(able[:, None], ids, -1).to(torch.int32))
    key = torch.where(able[:, None], ids, E).reshape(-1)
    order, n = torch.sort(key, stable=True).indices, int(able.sum()) * k
    assert torch.equal(r.rows[:n], (order[:n] // k).to(torch.int32)) and (r.rows[n:] == -1).all()
    assert torch.equal(r.offsets[1:], torch.cumsum(torch.bincount(key, minlength=E + 1)[:E], 0).to(torch.int32)) and r.offsets[0] == 0
    slots = torch.full((T * k,), -1, device="cuda")
    slots[order[:n]] = torch.arange(n, device="cuda")
    assert torch.equal(r.slots.reshape(-1), slots.to(torch.int32))

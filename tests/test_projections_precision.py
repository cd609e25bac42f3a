"""A x of the adapters is held and added as the fp32 value that it is: whole numbers of 22 to 24 bits, each output with one of them, compared bit by
bit.  (In the other cases of whole numbers A x stays below 130, which 8 bits hold, and the tolerance for normal values allows for c_in roundings
of A x, more than holding it in few bits would cost.)"""
import pytest
import torch

from test_gpu_projections import BF16, F16, _layers, snn  # noqa: F401

# rows, c_in, c_out, adapters, rank, rows of a run
CASES = [
    (1, 64, 40, 1, 8, 1),
    (9, 512, 131, 3, 16, 1),
    (40, 264, 300, 16, 24, 1),
    (70, 1024, 129, 4, 64, 9),
    (200, 128, 260, 150, 16, 1),    # more adapters in a tile than the matrix instructions add
    (330, 72, 256, 5, 8, 1),        # four adapters to a pass
    (420, 520, 140, 7, 16, 31),
    (600, 1024, 384, 3, 128, 250),
]


def _draw(R, c_in, c_out, n, rank, run):
    """x, A, B, scale and adapter as doubles and whole numbers, all of them values of fp16 and bf16.  A x is 2560 * 2048, of either sign, and a sum of
    c_in - 1 products of numbers up to 8: between 2^22 and 2^23 and below 2^23 in every order and part of it.  B has one 1 or -1 for each
    channel.  With scales 1/2 to 2 and |S| <= 2560 + 8 c_in everything stays below 2^24 of its unit (1, or 1/2): fp32 sums are exact."""
    g = torch.Generator().manual_seed(R + c_in)

    def sign(*shape):
        return 2.0 * torch.randint(0, 2, shape, generator=g).double() - 1

    x, a = torch.randint(-8, 9, (R, c_in), generator=g).double(), torch.randint(-8, 9, (n, rank, c_in), generator=g).double()
    x[:, 0], a[:, :, 0] = 2560 * sign(R), 2048 * sign(n, rank)
    b = torch.zeros(n, c_out, rank, dtype=torch.float64)
    b.scatter_(2, torch.randint(0, rank, (n, c_out, 1), generator=g), sign(n, c_out, 1))
    scale = sign(n) * 2.0 ** torch.randint(-1, 2, (n,), generator=g).double()
    pick = torch.randint(-1, n + 1, ((R + run - 1) // run,), generator=g)
    pick[0] = n - 1
    return x, a, b, scale, pick.repeat_interleave(run)[:R]


def _terms(x, a, b, scale, adapter, hold=lambda h: h):
    """scale * B (A x) in 64 bits, scale * (A x) passed through `hold`."""
    out = torch.zeros(len(x), b.shape[1], dtype=torch.float64, device=x.device)
    for i in range(len(a)):
        m = adapter == i
        out[m] = hold(scale[i] * (x[m] @ a[i].T)) @ b[i].T
    return out


def _cut(bits):
    """To the leading bits: what is left of a value when parts of it are dropped."""
    def hold(h):
        m, e = torch.frexp(h)
        return torch.ldexp(torch.trunc(m * 2.0 ** bits) / 2.0 ** bits, e)
    return hold


def _rounded(bits):
    def hold(h):
        m, e = torch.frexp(h)
        return torch.ldexp(torch.round(m * 2.0 ** bits) / 2.0 ** bits, e)
    return hold


@pytest.mark.parametrize("case", CASES)
def test_fewer_bits_would_show(case):
    """On the host: A x as one or two of its three parts of 11 bits, or rounded to bf16, tf32, or 22 bits, changes the outputs."""
    x, a, b, scale, adapter = _draw(*case)
    for t in (x, a, b):
        assert torch.equal(t.to(BF16).double(), t) and torch.equal(t.to(F16).double(), t)
    ref, has = _terms(x, a, b, scale, adapter), (adapter >= 0) & (adapter < len(a))
    h = torch.cat([(x[adapter == i] @ a[i].T).reshape(-1) for i in range(len(a))])
    assert (h.abs() > 2 ** 22).all() and (h.abs() < 2 ** 23).all() and has.any()
    assert torch.equal(_terms(x, a, b, scale, adapter, _cut(33)), ref)
    for hold, share in ((_cut(11), 0.9), (_rounded(8), 0.9), (_rounded(11), 0.9), (_cut(22), 0.25), (_rounded(22), 0.25)):
        assert (_terms(x, a, b, scale, adapter, hold) != ref)[has].double().mean() >= share


@pytest.mark.gpu
@pytest.mark.parametrize("act", [F16, BF16])
@pytest.mark.parametrize("force", ["few", "many"])
@pytest.mark.parametrize("case", CASES)
def test_all_bits_of_the_first_factor(snn, monkeypatch, case, force, act):  # noqa: F811
    monkeypatch.setenv("SNN_FORCE_ROWS", force)
    _, c_in, c_out, *_ = case
    layers, w, _ = _layers(snn, 1, c_in, c_out, 5, 2300, alpha=1.0)
    x, a, b, scale, adapter = (t.cuda() for t in _draw(*case))
    y = snn.SnnConvAdapters(layers[0]).forward(x.to(act), adapter.to(torch.int32), a.to(act), b.to(act), scale.float(), out_type=snn.OUT_F32)
    ref = x @ w[0].T + _terms(x, a, b, scale, adapter)
    assert torch.equal(ref.float().double(), ref) and (ref.abs() < 2 ** 24).all()
    assert torch.equal(y, ref.float())

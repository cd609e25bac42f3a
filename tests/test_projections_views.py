"""Tensors whose memory holds the negated values (torch keeps a bit for it: the imaginary part of a conjugated tensor) are refused: the library
reads memory."""

import pytest
import torch

import paper_2110_09195_b200 as snn
from test_projections import I, X, _experts, no_library  # noqa: F401


def _negated(t):
    return torch._neg_view(t)


def test_what_torch_does():
    z = torch.complex(torch.ones(3, 1), torch.ones(3, 1))
    y = z.conj().imag
    assert y.is_neg() and (y == -1).all() and y.shape[1] == 1   # (one column: rows that are dense)


@pytest.mark.parametrize("x,out", [(_negated(torch.zeros(4, 16, **X)), None), (torch.zeros(4, 16, **X), _negated(torch.zeros(4, 5, **X)))])
def test_experts_refuse_negated_tensors(no_library, x, out):  # noqa: F811
    h = _experts()
    with pytest.raises(snn.SnnError) as ei:
        h.forward(x, torch.zeros(4, **I), out=out)
    assert ei.value.status == 1 and "negated" in str(ei.value)


@pytest.mark.parametrize("name", ["x", "a", "b", "scale", "adapter"])
def test_adapters_refuse_negated_tensors(no_library, name):  # noqa: F811
    h = _experts(snn.SnnConvAdapters)
    args = dict(x=torch.zeros(4, 16, **X), adapter=torch.zeros(4, **I), a=torch.zeros(2, 8, 16, **X), b=torch.zeros(2, 5, 8, **X), scale=torch.zeros(2))
    args[name] = _negated(args[name])
    with pytest.raises(snn.SnnError) as ei:
        h.forward(**args)
    assert ei.value.status == 1 and "negated" in str(ei.value)


@pytest.mark.gpu
def test_route_and_combine_refuse_negated_tensors():
    z = torch.complex(torch.ones(3, 1), torch.full((3, 1), float("inf"))).cuda()
    y = z.conj().imag
    with pytest.raises(snn.SnnError, match="negated"):
        snn.route(y, 1)
    with pytest.raises(snn.SnnError, match="negated"):
        snn.combine(y, torch.zeros(2, 1, device="cuda", **I), torch.ones(2, 1, device="cuda"))
    out = torch.empty(2, 1, device="cuda")
    with pytest.raises(snn.SnnError, match="negated"):
        snn.combine(y.resolve_neg(), torch.zeros(2, 1, device="cuda", **I), _negated(torch.ones(2, 1, device="cuda")), out=out)
    assert torch.equal(snn.combine(y.resolve_neg(), torch.zeros(2, 1, device="cuda", **I), torch.ones(2, 1, device="cuda"), out=out),
                       torch.full((2, 1), -float("inf"), device="cuda"))

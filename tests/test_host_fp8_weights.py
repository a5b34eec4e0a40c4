"""Fp8Weight.quantise on the tensors that programs hold weights in (on the CPU; the check that operands are on a GPU is left out)."""
import pytest
import torch

from paper_2304_11745_amd import tokens as T


@pytest.fixture()
def made(monkeypatch):
    monkeypatch.setattr(T.Fp8Weight, "__init__", lambda self, codes, scales: self.__dict__.update(codes=codes, scales=scales, out=codes.shape[0], cin=codes.shape[1]))


def test_a_parameter_leaves_no_graph_behind(made):
    """A graph would hold the parameter's copies in 32 bits, four times the codes, as long as the codes live."""
    p = torch.nn.Parameter(torch.randn(200, 144, generator=torch.Generator().manual_seed(1)))
    q, plain = T.Fp8Weight.quantise(p), T.Fp8Weight.quantise(p.detach())
    for t in (q.codes, q.scales, q.values()):
        assert not t.requires_grad and t.grad_fn is None
    assert torch.equal(q.codes.view(torch.uint8), plain.codes.view(torch.uint8)) and torch.equal(q.scales, plain.scales)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float64])
def test_other_types_and_strides(made, dtype):
    w = torch.randn(144, 200, generator=torch.Generator().manual_seed(2)).to(dtype)
    a, b = T.Fp8Weight.quantise(w.t()), T.Fp8Weight.quantise(w.float().t().contiguous())
    assert a.codes.is_contiguous() and a.scales.is_contiguous()
    assert torch.equal(a.codes.view(torch.uint8), b.codes.view(torch.uint8)) and torch.equal(a.scales, b.scales)

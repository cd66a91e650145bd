"""What autograd is told of the sequence operators and of AdamW."""
import pytest
import torch

from paper_2606_21101_amd.optim import AdamW
from paper_2606_21101_amd.sequence import GatedRecurrence, SequenceEmbedding

pytestmark = pytest.mark.gpu


def test_second_derivatives_are_refused():
    """The gradients are no functions that autograd could differentiate: an error, not a missing term."""
    table = torch.randn((10, 8), device="cuda", requires_grad=True)
    ids = torch.tensor([1, 2, 1], dtype=torch.int32, device="cuda")
    (grad,) = torch.autograd.grad(SequenceEmbedding(table)(ids).square().sum(), table, create_graph=True)
    with pytest.raises(RuntimeError):
        grad.sum().backward()
    x = torch.randn((6, 8), device="cuda", requires_grad=True)
    gate = torch.randn((6, 8), device="cuda", requires_grad=True)
    h, _ = GatedRecurrence(8)(x, gate, torch.tensor([0, 6], dtype=torch.int32, device="cuda"))
    (grad,) = torch.autograd.grad(h.square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        grad.sum().backward()

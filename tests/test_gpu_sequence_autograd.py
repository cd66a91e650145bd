"""What autograd is told of the sequence operators and of AdamW, and that passes leave their inputs as they are."""
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


def test_a_step_between_a_graphs_forward_and_backward_is_seen():
    """Weights that a step changed are not taken for those of the forward pass, as with torch's in-place operations."""
    w = torch.randn((4, 4), device="cuda", requires_grad=True)
    x = torch.randn((4, 4), device="cuda", requires_grad=True)
    y = (x @ w).sum()
    opt = AdamW([w])
    opt.step([torch.ones_like(w)])
    with pytest.raises(RuntimeError):
        y.backward()
    (x @ w).sum().backward()
    # four fp32 terms below 4 in any order: each of three sums rounds by at most 2^-21 of 16
    assert float((x.grad - w.detach().sum(1)).abs().max()) <= 3 * 16 * 2.0 ** -24 * 2


def test_weights_made_without_autograd_are_stepped():
    with torch.inference_mode():
        w = torch.zeros(4, device="cuda", requires_grad=True)
    AdamW([w], lr=0.5, weight_decay=0.0, eps=0.0).step([torch.ones(4, device="cuda")])
    # the first step of a constant gradient is lr, but for a few roundings of m, v and their corrections
    assert float((w.detach() + 0.5).abs().max()) <= 0.5 * 16 * 2.0 ** -24


def test_gradients_of_other_dtypes_in_turn():
    """The states go on from step to step, whatever type each step's gradients have."""
    torch.manual_seed(0)
    p = torch.randn(300, device="cuda")
    q = p.clone()
    a, b = AdamW([p]), AdamW([q])
    for k in range(4):
        g = torch.randn(300, device="cuda").to(torch.bfloat16)
        a.step([g])
        b.step([g if k % 2 else g.float()])
    assert torch.equal(p, q) and torch.equal(a.m[0], b.m[0]) and len(b._made) == 2


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim", [50, 64])
@pytest.mark.parametrize("max_len", [16, 0])
def test_passes_leave_their_inputs_and_give_equal_bits(dtype, dim, max_len):
    """Three training passes that nothing waits between, the second over other histories: the third is as the first."""
    torch.manual_seed(dim)
    op = GatedRecurrence(dim, max_len=max_len)

    def inputs(lens):
        off = torch.zeros(len(lens) + 1, dtype=torch.int32, device="cuda")
        off[1:] = lens.cumsum(0)
        n = int(off[-1])
        x, gate, dh = (torch.randn((n, dim), device="cuda").to(dtype) for _ in range(3))
        return [x, gate, off, torch.randn((len(lens), dim), device="cuda"), dh, torch.randn((len(lens), dim), device="cuda")]

    def work(x, gate, off, h0, dh, dl):
        h, last, saved = op.forward(x, gate, off, h0, save=True)
        return [h, last, *op.backward(saved, dh, dl)]

    lens = torch.randint(0, 17, (3000,), device="cuda")
    mine, other = inputs(lens), inputs(lens.flip(0))
    kept = [t.clone() for t in mine]
    first = work(*mine)
    work(*other)
    for a, b in zip(first, work(*mine)):
        assert torch.equal(a, b)
    for a, b in zip(mine, kept):
        assert torch.equal(a, b)

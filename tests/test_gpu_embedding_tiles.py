"""The gradient's sort at its tiles' and digits' limits: sums of small whole numbers, which are exact in fp32."""
import pytest
import torch

from paper_2606_21101_amd.sequence import SequenceEmbedding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [4096, 4097, 8191, 16385, 32768, 33793, 66000, 800_001])
@pytest.mark.parametrize("rows", [1, 2, 3, 7, 300, 1023, 1024, 70_000, 1_100_000])
def test_whole_sums(tokens, rows):
    g = torch.Generator(device="cuda").manual_seed(tokens + rows)
    ids = (torch.rand(tokens, device="cuda", generator=g).square() * rows).to(torch.int32).clamp_(max=rows - 1)
    dout = torch.randint(-4, 5, (tokens, 5), device="cuda", generator=g).to(torch.float32)
    op = SequenceEmbedding(torch.empty((rows, 5), device="cuda"), padding_id=rows // 2 if rows > 2 else -1)
    want = torch.zeros((rows, 5), dtype=torch.float64, device="cuda").index_add_(0, ids.long(), dout.double())
    if rows > 2:
        want[rows // 2] = 0.0
    grad = op.backward(ids, dout, grad=torch.full((rows, 5), 9.0, device="cuda"))
    assert float(want.abs().max()) < 2 ** 24 and torch.equal(grad.double(), want)

"""Sequences and AdamW where offsets pass 32 bits, and what the torch classes refuse."""
import numpy as np
import pytest
import torch

import seq_reference as ref
from paper_2606_21101_amd import dpi
from paper_2606_21101_amd.optim import AdamW
from paper_2606_21101_amd.sequence import GatedRecurrence, SequenceEmbedding

pytestmark = pytest.mark.gpu


def test_embedding_of_a_table_past_32_bits():
    """36 M rows of 64 fp32 (2.3e9 elements): rows at both ends, and the gradient's rows between them are zeros."""
    rows = 36_000_000
    table = torch.zeros((rows, 64), device="cuda")
    at = torch.tensor([0, 1, rows // 2, rows - 2, rows - 1], device="cuda")
    table[at] = torch.arange(1, 6, device="cuda", dtype=torch.float32)[:, None].expand(5, 64)
    op = SequenceEmbedding(table, scale=2.0)
    order = torch.tensor([4, 0, 3, 1, 2, 4, 4], device="cuda")
    ids = at[order].to(torch.int32)
    assert op.forward(ids)[:, 63].tolist() == [10.0, 2.0, 8.0, 4.0, 6.0, 10.0, 10.0]
    many = ids.repeat(2000)                       # the sort of many workgroups
    for tokens in (ids, many):
        grad = op.backward(tokens, torch.ones((len(tokens), 64), device="cuda"), grad=table)
        k = len(tokens) // 7
        assert grad[at, 5].tolist() == [2.0 * k, 2.0 * k, 2.0 * k, 2.0 * k, 6.0 * k]
        assert float(grad.abs().sum(0, dtype=torch.float64)[7]) == 14.0 * k


def test_more_tokens_than_one_launch_has_rows_for():
    """2^27 + 5 tokens of 33 fp16: rows on both sides of the launches' border, and counts as the gradient of ones."""
    n, rows, dim = 2 ** 27 + 5, 10, 33
    table = torch.arange(rows * dim, device="cuda").reshape(rows, dim).to(torch.float16)
    ids = (torch.arange(n, device="cuda") % rows).to(torch.int32)
    op = SequenceEmbedding(table, padding_id=3)
    y = op.forward(ids)
    for t in (0, 2 ** 27 - 1, 2 ** 27, 2 ** 27 + 1, n - 1):
        assert torch.equal(y[t], table[t % rows] if t % rows != 3 else torch.zeros_like(table[0])), t
    grad = op.backward(ids, y.fill_(1.0), grad=torch.empty((rows, dim), device="cuda"))
    want = torch.bincount(ids, minlength=rows).float()          # below 2^24: exact
    want[3] = 0.0
    assert torch.equal(grad, want[:, None].expand(rows, dim))


def test_more_single_tokens_than_one_launch_has():
    """2^17 + 2 rows of 65,536 channels; all slots but the first and the last two name no state."""
    n, dim = 2 ** 17 + 2, dpi.DPI_MAX_DIM
    x = torch.full((n, dim), 2.0, dtype=torch.float16, device="cuda")
    gate = torch.zeros((n, dim), dtype=torch.float16, device="cuda")
    slots = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    slots[0], slots[n - 2], slots[n - 1] = 1, 0, 2
    state = torch.tensor([[0.0], [4.0], [8.0]], device="cuda").expand(3, dim).contiguous()
    y = GatedRecurrence(dim).step(x, gate, state, slots)
    assert [float(y[b].float().min()) for b in (0, 1, n - 3, n - 2, n - 1)] == [3.0, 0.0, 0.0, 1.0, 5.0]
    assert state.min(dim=1).values.tolist() == [1.0, 3.0, 5.0] == state.max(dim=1).values.tolist()


def test_recurrence_past_32_bits():
    """34 M tokens of 64 fp16 (2.2e9 elements) in three sequences, the last of 700 tokens: as by itself."""
    n, last = 34_000_000, 700
    x = torch.empty((n, 64), dtype=torch.float16, device="cuda").normal_()
    g = torch.empty((n, 64), dtype=torch.float16, device="cuda").normal_(1.0, 1.0)
    off = torch.tensor([0, 5, n - last, n], dtype=torch.int32, device="cuda")
    op = GatedRecurrence(64)
    h, ends, saved = op.forward(x, g, off, save=True)
    alone = torch.tensor([0, last], dtype=torch.int32, device="cuda")
    h1, end1, saved1 = op.forward(x[-last:], g[-last:], alone, save=True)
    assert float((ends[2] - end1[0]).abs().max()) < 1e-4
    assert float((h[-last:].float() - h1.float()).abs().max()) < 4e-3      # two roundings of values below 4
    dx, dg, d0 = op.backward(saved, None, torch.ones((3, 64), device="cuda"), dx=h)
    dx1, dg1, d1 = op.backward(saved1, None, torch.ones((1, 64), device="cuda"))
    assert float((d0[2] - d1[0]).abs().max()) < 1e-5
    assert torch.allclose(dx[-last:].float(), dx1.float(), rtol=2e-3, atol=1e-6)
    assert torch.allclose(dg[-last:].float(), dg1.float(), rtol=2e-3, atol=1e-4)


def test_adamw_of_a_tensor_past_32_bits():
    """2^32 + 1000 elements with 8-bit states: the last ones as the definition has them, index and all."""
    n = 2 ** 32 + 1000
    p, g = (torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    tail = torch.from_numpy(np.random.default_rng(0).standard_normal(1000).astype(np.float32)).to(torch.bfloat16)
    g[-1000:] = tail.cuda()
    opt = AdamW([p], state_bits=8, seed=5)
    opt.step([g])
    f, first = np.float32, 2 ** 32
    r = ref.mix((((np.arange(first, n, dtype=np.uint64) & np.uint64(ref.M32)) * np.uint64(0x9E3779B1)
                  + np.uint64(1) + ref.mix((5 + 0x9E3779B1) & ref.M32)) & np.uint64(ref.M32)))
    gf = tail.float().numpy()
    for codes, scale, z, rnd, small in (
            (opt.m[0], opt.m_scale[0], gf * f(1 - 0.9), ((r & np.uint64(0xFFFF)) << np.uint64(4)).astype(np.int64), False),
            (opt.v[0], opt.v_scale[0], (gf * gf) * f(1 - 0.999), ((r >> np.uint64(16)) << np.uint64(4)).astype(np.int64), True)):
        want, want_scale = ref.store8(z, rnd, small)
        assert np.array_equal(codes[-1000:].view(torch.uint8).cpu().numpy(), want)
        assert np.array_equal(scale[-4:].cpu().numpy(), want_scale)
    assert not bool(p[:-1000].any())


def refused(call, *args, **kw):
    with pytest.raises(dpi.DpiError) as e:
        call(*args, **kw)
    assert e.value.status in (dpi.DPI_ERR_INVALID_ARG, dpi.DPI_ERR_UNSUPPORTED)


def test_embedding_refusals():
    table = torch.zeros((10, 8), device="cuda")
    op = SequenceEmbedding(table)
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    refused(SequenceEmbedding, table[:, :4])
    refused(SequenceEmbedding, table.double())
    refused(SequenceEmbedding, table, out_dtype=torch.float64)
    refused(op.forward, ids.long())
    refused(op.forward, ids[::2])
    refused(op.forward, ids.cpu())
    refused(op.forward, ids, out=torch.zeros((4, 7), device="cuda"))
    refused(op.forward, ids, out=torch.zeros((4, 8), dtype=torch.float16, device="cuda"))
    refused(op.forward, ids, out=torch.zeros((8, 4), device="cuda").t())
    refused(op.backward, ids, torch.zeros((3, 8), device="cuda"))
    refused(op.backward, ids, torch.zeros((4, 8), device="cuda"), grad=torch.zeros((9, 8), device="cuda"))


def test_recurrence_refusals():
    x = torch.zeros((6, 8), device="cuda")
    off = torch.tensor([0, 6], dtype=torch.int32, device="cuda")
    op = GatedRecurrence(8)
    refused(op.forward, x, x.half(), off)
    refused(op.forward, x, x[:5], off)
    refused(op.forward, x, x, off.long())
    refused(op.forward, x, x, off[:0])
    refused(op.forward, x, x, off, torch.zeros((2, 8), device="cuda"))
    refused(op.forward, x, x, off, torch.zeros((1, 8), dtype=torch.float16, device="cuda"))
    refused(op.forward, x, x, off.cpu())
    refused(GatedRecurrence(9).forward, x, x, off)
    refused(op.forward, torch.zeros((6, 1 << 18), device="cuda")[:, :8], x, off)      # a stride too wide
    saved = op.forward(x, x, off, save=True)[2]
    refused(op.backward, saved, x.half())
    refused(op.backward, saved, x, torch.zeros((2, 8), device="cuda"))
    store = torch.zeros((4, 8), device="cuda")
    refused(op.step, x, x, store)                                                     # fewer states than rows
    refused(op.step, x, x, store.half(), torch.arange(6, dtype=torch.int32, device="cuda"))
    refused(op.step, x, x, store, torch.arange(5, dtype=torch.int32, device="cuda"))


def test_adamw_refusals():
    p = torch.zeros(300, device="cuda")
    refused(AdamW, [])
    refused(AdamW, [p], state_bits=16)
    refused(AdamW, [p.double()])
    refused(AdamW, [torch.zeros((4, 4), device="cuda").t()])
    refused(AdamW, [p], m=[torch.zeros(299, device="cuda")])
    refused(AdamW, [p], masters=[p.half()])
    refused(AdamW, [p], state_bits=8, m_scale=[torch.zeros(1, device="cuda")])
    opt = AdamW([p])
    refused(opt.step, [])
    refused(opt.step, [torch.zeros(301, device="cuda")])
    refused(opt.step, [torch.zeros(600, device="cuda")[::2]])
    refused(opt.step, [torch.zeros(300, dtype=torch.float64, device="cuda")])
    refused(opt.step, [torch.zeros(300)])
    for kw in (dict(step=0), dict(lr=-1.0), dict(lr=float("nan")), dict(grad_scale=float("inf"))):
        refused(opt.step, [torch.zeros(300, device="cuda")], **kw)
    assert opt.step_count == 0 and not bool(p.any())

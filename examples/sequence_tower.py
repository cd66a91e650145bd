"""A behaviour-sequence tower trained and served: which item does a user look at next?

Synthetic users browse items of one topic at a time.  A tower reads the packed
histories -- ids to scaled rows (SequenceEmbedding), a projection to values and
gates, a gated recurrence over each history (GatedRecurrence) -- and its last
state scores a candidate item; context fields go through the fused lookup.  All
weights are stepped by one AdamW.  Afterwards users' states lie in a store, and
each new event moves one of them on by a single token.

  python examples/sequence_tower.py [--steps 150] [--state-bits 8]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_21101_amd.lookup import FusedLookup  # noqa: E402
from paper_2606_21101_amd.optim import AdamW  # noqa: E402
from paper_2606_21101_amd.sequence import GatedRecurrence, SequenceEmbedding  # noqa: E402

TOPICS, ITEMS_PER_TOPIC, PADDING = 64, 32, 0
ITEMS = 1 + TOPICS * ITEMS_PER_TOPIC
CONTEXT_ROWS, CONTEXT_DIM = (100, 24, 7), 16


class Tower:
    def __init__(self, dim: int, max_len: int, dtype: torch.dtype, gen: torch.Generator):
        def weight(*shape, sigma):
            return (torch.randn(shape, generator=gen, device="cuda") * sigma).to(dtype).requires_grad_()
        self.dim, self.dtype = dim, dtype
        self.items = weight(ITEMS, dim, sigma=0.02)
        self.project = weight(2 * dim, dim, sigma=dim ** -0.5)
        self.bias = torch.cat([torch.zeros(dim), torch.full((dim,), 1.0)]).to("cuda", dtype).requires_grad_()
        self.context_weight = weight(len(CONTEXT_ROWS) * CONTEXT_DIM, sigma=0.1)
        self.rows = SequenceEmbedding(self.items, scale=dim ** 0.5, padding_id=PADDING)
        self.recurrence = GatedRecurrence(dim, max_len=max_len)
        tables = [torch.randn((n, CONTEXT_DIM), generator=gen, device="cuda") * 0.1 for n in CONTEXT_ROWS]
        self.context = FusedLookup(tables)   # fixed context features

    def weights(self):
        return [self.items, self.project, self.bias, self.context_weight]

    def gates(self, ids):
        """Values and gates of tokens: the halves of one projection."""
        both = F.linear(self.rows(ids), self.project, self.bias)
        return both[:, : self.dim], both[:, self.dim:]

    def states(self, ids, offsets):
        return self.recurrence(*self.gates(ids), offsets)[1]

    def score(self, state, candidates, context_ids):
        block = self.context(context_ids, None, len(candidates))
        return (state * self.rows(candidates).float()).sum(1) + block @ self.context_weight.float()


def batch(users: int, max_len: int, gen: torch.Generator):
    """Histories, candidates (half of them of the history's topic), labels, context ids."""
    lens = torch.randint(0, max_len + 1, (users,), generator=gen, device="cuda")
    offsets = F.pad(torch.cumsum(lens, 0), (1, 0)).to(torch.int32)
    n = int(offsets[-1])
    topic = torch.randint(0, TOPICS, (users,), generator=gen, device="cuda")
    label = torch.randint(0, 2, (users,), generator=gen, device="cuda")
    other = (topic + torch.randint(1, TOPICS, (users,), generator=gen, device="cuda")) % TOPICS

    def items(topics):
        return 1 + topics * ITEMS_PER_TOPIC + torch.randint(0, ITEMS_PER_TOPIC, topics.shape, generator=gen, device="cuda")
    ids = items(torch.repeat_interleave(topic, lens))
    ids[torch.rand(n, generator=gen, device="cuda") < 0.05] = PADDING
    candidates = items(torch.where(label == 1, topic, other))
    context = torch.cat([torch.randint(0, r, (users,), generator=gen, device="cuda") for r in CONTEXT_ROWS])
    return ids.to(torch.int32), offsets, candidates.to(torch.int32), label.float(), context.to(torch.int32)


def train(tower: Tower, steps: int, users: int, max_len: int, state_bits: int, gen: torch.Generator):
    opt = AdamW(tower.weights(), masters=tower.dtype != torch.float32, state_bits=state_bits, lr=3e-3, seed=7)
    losses = []
    for _ in range(steps):
        ids, offsets, candidates, label, context = batch(users, max_len, gen)
        loss = F.binary_cross_entropy_with_logits(tower.score(tower.states(ids, offsets), candidates, context), label)
        loss.backward()
        opt.step()
        for w in tower.weights():
            w.grad = None
        losses.append(loss.detach())
    return [float(x) for x in losses]


@torch.no_grad()
def serve(tower: Tower, users: int, max_len: int, gen: torch.Generator):
    """States of `users` histories read at once, and token by token into a store: the largest difference."""
    ids, offsets, *_ = batch(users, max_len, gen)
    whole = tower.states(ids, offsets)
    store = torch.zeros((2 * users, tower.dim), device="cuda")
    slot = torch.randperm(2 * users, generator=gen, device="cuda")[:users].to(torch.int32)
    begin, lens = offsets[:-1].long(), torch.diff(offsets).long()
    for t in range(int(lens.max())):
        alive = torch.nonzero(lens > t)[:, 0]
        x, gate = tower.gates(ids[begin[alive] + t].contiguous())
        tower.recurrence.step(x, gate, store, slot[alive].contiguous())
    return float((store[slot.long()] - whole).abs().max())


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=150)
    ap.add_argument("--users", type=int, default=2048)
    ap.add_argument("--max-len", type=int, default=60)
    ap.add_argument("--dim", type=int, default=64)
    ap.add_argument("--state-bits", type=int, choices=(8, 32), default=32)
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="bf16")
    args = ap.parse_args(argv)
    gen = torch.Generator(device="cuda").manual_seed(0)
    tower = Tower(args.dim, args.max_len, torch.bfloat16 if args.dtype == "bf16" else torch.float32, gen)
    losses = train(tower, args.steps, args.users, args.max_len, args.state_bits, gen)
    apart = serve(tower, 256, args.max_len, gen)
    print(f"loss {losses[0]:.4f} -> {sum(losses[-10:]) / len(losses[-10:]):.4f} in {args.steps} steps; "
          f"states served token by token differ by at most {apart:.2e}")
    return losses, apart


if __name__ == "__main__":
    main()

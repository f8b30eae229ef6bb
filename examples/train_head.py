"""A query head trained against a collection, and served beside its index.

The collection's vectors are fixed; a head of two layers maps an encoder's hidden
rows to query vectors.  Each step scores a batch against every item of the
collection (softmax cross entropy, no logits kept), keeps the layers' inputs in 8
bits for the backward pass, and updates the head.  Afterwards the head's weights
are packed in 4 bits, single queries go through it, and their vectors read exact
ranks from the index of the collection.

    python examples/train_head.py [--items 20000] [--steps 150]

Hidden rows are synthetic: a fixed random layer over the item that answers the
query, with noise, so that an untrained head finds next to nothing.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_07152_gb300 as pvs  # noqa: E402
import synth  # noqa: E402

SCALE = 20.0          # 1 / temperature of the softmax
GROUP = 64            # weights that share a 4-bit scale


class Head:
    """hidden [B, H] -> GELU layer [B, M] -> vectors [B, D], weights float32 with
    bfloat16 copies for the products."""

    def __init__(self, hidden: int, middle: int, dim: int, seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.w1 = torch.randn(middle, hidden, generator=g, device="cuda") / hidden ** 0.5
        self.w2 = torch.randn(dim, middle, generator=g, device="cuda") / middle ** 0.5
        self.adam = torch.optim.Adam([self.w1, self.w2], lr=2e-3)

    def step(self, hidden, items, targets, bias):
        """One training step; returns the mean loss (a tensor, nothing waits)."""
        w1, w2 = self.w1.bfloat16(), self.w2.bfloat16()
        # forward: what the backward pass needs of each layer stays as 8-bit rows
        in1, s_in1, _ = pvs.pvs_ckpt_store(hidden)
        pre, s_pre, act = pvs.pvs_ckpt_store(hidden @ w1.T, act=pvs.PVS_ACT_GELU)
        in2, s_in2, _ = pvs.pvs_ckpt_store(act)
        vectors = act @ w2.T
        del act
        loss, stats = pvs.pvs_xent_forward(vectors, items, targets, bias=bias, scale=SCALE)
        # backward
        grad = torch.full_like(loss, 1.0 / loss.numel())
        dvec, _ = pvs.pvs_xent_backward(vectors, items, targets, stats, grad, bias=bias,
                                        scale=SCALE, need_w=False)
        self.w2.grad = pvs.pvs_ckpt_grad_weight(dvec, in2, s_in2).float()
        dpre = pvs.pvs_ckpt_act_backward(dvec @ w2, pre, s_pre, pvs.PVS_ACT_GELU)
        self.w1.grad = pvs.pvs_ckpt_grad_weight(dpre, in1, s_in1).float()
        self.adam.step()
        return loss.mean()

    def pack(self):
        return pvs.pvs_wq_pack(self.w1, GROUP), pvs.pvs_wq_pack(self.w2, GROUP)


def query_vector(packed, hidden):
    """One hidden row [1, H] float32 through the packed head."""
    (c1, s1), (c2, s2) = packed
    pre = pvs.pvs_wq_matvec(hidden, c1, s1, GROUP)
    _, _, act = pvs.pvs_ckpt_store(pre, act=pvs.PVS_ACT_GELU)
    return pvs.pvs_wq_matvec(act, c2, s2, GROUP)[0]


def first_ranks(index, vector, n: int = 10):
    cursor = pvs.pvs_cursor_open(index, vector)
    try:
        ids, _, _ = pvs.pvs_next(cursor, n)
    finally:
        pvs.pvs_cursor_close(cursor)
    return ids


def found(index, packed, hidden, targets, n: int = 10):
    """The share of queries whose item is among the first n ranks."""
    hits = sum(int(t) in first_ranks(index, query_vector(packed, hidden[i:i + 1]), n)
               for i, t in enumerate(targets.tolist()))
    return hits / targets.numel()


def run(items_n: int = 20_000, dim: int = 128, hidden: int = 256, middle: int = 384,
        batch: int = 512, steps: int = 150, queries: int = 100, seed: int = 0, log=None):
    items = synth.unit_normal(items_n, dim, seed=seed, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    encoder = torch.randn(hidden, dim, generator=g, device="cuda")
    deleted = torch.rand(items_n, generator=g, device="cuda") < 0.02
    bias = torch.zeros(items_n, device="cuda").masked_fill_(deleted, float("-inf"))
    live = torch.nonzero(~deleted)[:, 0]

    def sample(n):
        y = live[torch.randint(0, live.numel(), (n,), generator=g, device="cuda")]
        h = items[y] @ encoder.T + 0.2 * torch.randn(n, hidden, generator=g, device="cuda")
        return torch.tanh(h), y

    index = pvs.pvs_build(items)
    pvs.pvs_tombstone(index, torch.nonzero(deleted)[:, 0].cpu().numpy())
    try:
        head = Head(hidden, middle, dim, seed + 2)
        test_hidden, test_y = sample(queries)
        before = found(index, head.pack(), test_hidden, test_y)
        vectors = items.bfloat16()
        losses = []
        for i in range(steps):
            h, y = sample(batch)
            losses.append(head.step(h.bfloat16(), vectors, y, bias))
            if log and (i + 1) % 50 == 0:
                log(f"step {i + 1}: loss {losses[-1].item():.3g}")
        after = found(index, head.pack(), test_hidden, test_y)
        pvs.pvs_head_status()
    finally:
        pvs.pvs_index_free(index)
    return dict(first_loss=losses[0].item(), last_loss=losses[-1].item(), before=before, after=after)


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--items", type=int, default=20_000)
    p.add_argument("--steps", type=int, default=150)
    a = p.parse_args()
    r = run(items_n=a.items, steps=a.steps, log=print)
    print(f"loss {r['first_loss']:.3g} -> {r['last_loss']:.3g}; item among the first 10 ranks of a "
          f"4-bit head's query: {r['before']:.0%} -> {r['after']:.0%}")


if __name__ == "__main__":
    main()

"""A query head over token embeddings, distilled from a teacher and served in 4-bit floats.

Queries are short lists of token ids.  A table turns tokens into rows, a query is the sum of
its rows over the root of their number, and one layer makes its vector.  Instead of one right item, each query has a teacher's
scores of a few items (a slower model's list); a step lowers the divergence of the head's softmax
over the whole collection from it.  Afterwards the layer is packed in microscaled 4-bit floats, a
batch of queries goes through it at once, and their vectors read exact ranks from the index.

    python examples/distill_head.py [--items 20000] [--steps 150]

The teacher is synthetic: the exact scores of a fixed table and layer, which the head has to find.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_07152_gb300 as pvs  # noqa: E402
import synth  # noqa: E402

SCALE = 20.0          # 1 / temperature of the head's softmax, and of the teacher's
GROUP = 16            # weights that share a 4-bit scale
EMPTY = -100          # a token or a slot of a list that is not there


class Head:
    """tokens [B, L] -> rows of `table` [V, H] -> their sum L^-1/2 -> `w` [D, H] -> vectors [B, D]."""

    def __init__(self, vocabulary: int, hidden: int, dim: int, seed: int = 0, lr: float = 2e-2):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.table = torch.randn(vocabulary, hidden, generator=g, device="cuda")
        self.w = torch.randn(dim, hidden, generator=g, device="cuda") / hidden ** 0.5
        self.adam = torch.optim.Adam([self.table, self.w], lr=lr)

    def pooled(self, tokens):
        """The sum [B, H] of the tokens' rows times L^-1/2 (an empty token counts as zeros)."""
        b, n = tokens.shape
        rows = pvs.pvs_embed_forward(self.table, tokens.reshape(-1), scale=n ** -0.5, ignore_index=EMPTY)
        return rows.view(b, n, -1).sum(dim=1)

    def gradients(self, tokens, items, ids, scores, bias=None):
        """The mean loss and its gradients (dtable, dw)."""
        b, n = tokens.shape
        x = self.pooled(tokens)
        vectors = x @ self.w.T
        loss, stats, hits = pvs.pvs_distill_forward(vectors, items, ids, scores, bias=bias, scale=SCALE,
                                                    teacher_scale=SCALE, ignore_index=EMPTY)
        grad = torch.full_like(loss, 1.0 / b)
        dvec, _ = pvs.pvs_distill_backward(vectors, items, ids, stats, hits, grad, bias=bias, scale=SCALE,
                                           ignore_index=EMPTY, need_w=False)
        dw = dvec.T @ x
        drows = (dvec @ self.w)[:, None, :].expand(b, n, -1).reshape(b * n, -1)
        dtable = pvs.pvs_embed_backward(drows, tokens.reshape(-1), self.table.shape[0], scale=n ** -0.5,
                                        ignore_index=EMPTY)
        return loss.mean(), dtable, dw

    def step(self, *batch, **kw):
        loss, self.table.grad, self.w.grad = self.gradients(*batch, **kw)
        self.adam.step()
        return loss

    def vectors(self, tokens, packed=None):
        """Unit vectors of a batch of queries, with the layer in float32 or packed."""
        x = self.pooled(tokens)
        v = x @ self.w.T if packed is None else pvs.pvs_mx_matmul(x, *packed, GROUP)
        return v / v.norm(dim=1, keepdim=True)


def shared(index, vectors, ids, n: int = 10):
    """The share of the teacher's items (the first n of each list) among the first n exact ranks."""
    hits = 0
    for v, want in zip(vectors, ids[:, :n].tolist()):
        cursor = pvs.pvs_cursor_open(index, v.contiguous())
        try:
            got, _, _ = pvs.pvs_next(cursor, n)
        finally:
            pvs.pvs_cursor_close(cursor)
        hits += len(set(got.tolist()) & set(want))
    return hits / (n * len(vectors))


def run(items_n: int = 20_000, dim: int = 64, hidden: int = 128, vocabulary: int = 2000, length: int = 6,
        top: int = 32, batch: int = 512, steps: int = 150, queries: int = 60, seed: int = 0, log=None):
    items = synth.unit_normal(items_n, dim, seed=seed, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    table = torch.randn(vocabulary, dim, generator=g, device="cuda")

    def sample(n):
        # frequent tokens first; some queries are shorter
        u = torch.rand(n, length, generator=g, device="cuda")
        tokens = torch.pow(float(vocabulary), u).long().clamp(max=vocabulary) - 1
        short = torch.rand(n, length, generator=g, device="cuda") < 0.2
        short[:, 0] = False
        v = table[tokens].masked_fill_(short[..., None], 0.0).sum(dim=1)
        v = v / v.norm(dim=1, keepdim=True)
        scores, ids = (v @ items.T).topk(top, dim=1)
        return tokens.masked_fill_(short, EMPTY), ids, scores

    index = pvs.pvs_build(items)
    try:
        head = Head(vocabulary, hidden, dim, seed + 2)
        test_tokens, test_ids, _ = sample(queries)
        before = shared(index, head.vectors(test_tokens), test_ids)
        losses = []
        for i in range(steps):
            tokens, ids, scores = sample(batch)
            losses.append(head.step(tokens, items, ids, scores))
            if log and (i + 1) % 50 == 0:
                log(f"step {i + 1}: loss {losses[-1].item():.3g}")
        after = shared(index, head.vectors(test_tokens), test_ids)
        packed = pvs.pvs_mx_pack(head.w, GROUP)
        served = shared(index, head.vectors(test_tokens, packed), test_ids)
        pvs.pvs_head_status()
    finally:
        pvs.pvs_index_free(index)
    return dict(first_loss=losses[0].item(), last_loss=losses[-1].item(), before=before, after=after, served=served)


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--items", type=int, default=20_000)
    p.add_argument("--steps", type=int, default=150)
    a = p.parse_args()
    r = run(items_n=a.items, steps=a.steps, log=print)
    print(f"loss {r['first_loss']:.3g} -> {r['last_loss']:.3g}; of the teacher's first 10 items, among the first "
          f"10 ranks: {r['before']:.0%} -> {r['after']:.0%}, with 4-bit weights and rows {r['served']:.0%}")


if __name__ == "__main__":
    main()

"""From ratings to lists of items: factors by ALS, a next-item model over the histories, beam search.

A user's ratings, in the order of time, are tokens: the items' factors (learned by ALS) projected to
queries, keys and values, normed and rotated by the ratings' time bins, and read by linear attention
with a decay for each head. The model is trained to name each next item of the history, and then
answers every user with lists of items: the history is read once, and each further item is one step
of the recurrent form whose state comes from the beam it extends.

    python examples/next_items.py [--users 500] [--items 1000] [--steps 20]

Everything runs on one GPU with synthetic ratings.
"""
from __future__ import annotations

import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import numpy as np
import torch
import torch.nn.functional as F

import workload
from paper_1108_2580_amd import (ALS, beam_select, decay_attention, decay_attention_step, norm_rotate,
                                 rotary_tables)

DEV = "cuda:0"
HEADS, KEY_HEADS, WIDTH, BINS = 4, 2, 32, 64


class NextItems(torch.nn.Module):
    """One layer over item factors; the items' factors are also the output's weights."""

    def __init__(self, factors, seed):
        super().__init__()
        D = factors.shape[1]
        g = torch.Generator().manual_seed(seed)
        rows = (HEADS + 2 * KEY_HEADS) * WIDTH
        self.project = torch.nn.Parameter(torch.randn(rows, D, generator=g).to(DEV) * D ** -0.5)
        self.join = torch.nn.Parameter(torch.randn(D, HEADS * WIDTH, generator=g).to(DEV) *
                                       (HEADS * WIDTH) ** -0.5)
        self.q_weight = torch.nn.Parameter(torch.ones(WIDTH, device=DEV))
        self.k_weight = torch.nn.Parameter(torch.ones(WIDTH, device=DEV))
        self.items = torch.nn.Parameter(factors.clone())
        # windows of about 4 to 32 ratings
        self.register_buffer("log_decay", -torch.exp2(-2.0 - torch.arange(HEADS, device=DEV).float()))
        self.cos, self.sin = rotary_tables(BINS, WIDTH, device=DEV)

    def tokens(self, item, position):
        """(queries, keys, values) of tokens, heads and widths apart, all views of one projection."""
        x = (F.embedding(item, self.items) @ self.project.t()).unflatten(1, (-1, WIDTH))
        q, k, v = x.split((HEADS, KEY_HEADS, KEY_HEADS), 1)
        q, k = norm_rotate(q, k, self.q_weight, self.k_weight, self.cos, self.sin, position)
        return q, k, v

    def logits(self, out):
        return (out.flatten(1) @ self.join.t()) @ self.items.t()

    def forward(self, item, position, row_ptr):
        q, k, v = self.tokens(item, position)
        return self.logits(decay_attention(q, k, v, self.log_decay, row_ptr))


@torch.no_grad()
def answer(model, item, position, row_ptr, beams, length, end):
    """The best lists of `length` items for every row: (items [rows, beams, length], scores)."""
    q, k, v = model.tokens(item, position)
    out, state = decay_attention(q, k, v, model.log_decay, row_ptr, return_state=True)
    B = row_ptr.numel() - 1
    last = (row_ptr[1:] - 1).clamp(min=0)
    # an empty history says nothing: all items alike
    empty = (row_ptr[1:] == row_ptr[:-1])[:, None, None]
    logits = model.logits(out[last].masked_fill(empty, 0.0))
    scores = torch.zeros(B, 1, device=DEV)
    parents, token, scores, done = beam_select(logits[:, None], scores, None, end, width=beams)
    lists = token[..., None]
    first = torch.arange(B, device=DEV, dtype=torch.int32)[:, None]
    source = (first + parents).flatten()  # rows of `state`: one a user, then one a beam
    at = position[last.long()].repeat_interleave(beams)
    for _ in range(length - 1):
        q, k, v = model.tokens(token.flatten().clamp(min=0), at)
        out, state = decay_attention_step(q, k, v, model.log_decay, state, source=source)
        parents, token, scores, done = beam_select(model.logits(out).view(B, beams, -1), scores, done, end)
        lists = torch.cat([lists.gather(1, parents.long()[..., None].expand_as(lists)), token[..., None]], 2)
        source = (first * beams + parents).flatten()
    return lists, scores


def main(users=500, items=1000, steps=20, beams=4, length=5, seed=7):
    rng = np.random.default_rng(seed)
    degrees = rng.integers(0, 60, size=users)
    ptr, col, val = workload.make_custom(users, items, degrees, seed=seed)
    # learn the items' factors
    D = 20
    U, V = (torch.from_numpy(x).to(DEV) for x in workload.init_factors(users, items, D, seed))
    with ALS(users, items, ptr, col, val, D) as als:
        for _ in range(3):
            als.half_sweep("items", U, 0.065, V)
            rmse = als.half_sweep("users", V, 0.065, U, rmse=True)
    print(f"ALS: {users} users, {items} items, {col.size} ratings, RMSE {rmse:.3f}", flush=True)
    # the ratings of each user in the order of time
    bins = np.concatenate([np.sort(rng.integers(0, BINS, n)) for n in degrees] or [[]]).astype(np.int32)
    order = np.concatenate([ptr[b] + rng.permutation(n) for b, n in enumerate(degrees)] or [[]])
    item = torch.from_numpy(col[order.astype(np.int64)].astype(np.int64)).to(DEV)
    position = torch.from_numpy(bins).to(DEV)
    row_ptr = torch.from_numpy(np.ascontiguousarray(ptr)).to(DEV)
    # each token's target is the next item of its row
    row = torch.repeat_interleave(torch.arange(users, device=DEV), row_ptr[1:] - row_ptr[:-1])
    has_next = torch.zeros(item.numel(), dtype=torch.bool, device=DEV)
    has_next[:-1] = row[1:] == row[:-1]
    target = torch.roll(item, -1)[has_next]

    scale = V / V.norm(dim=1, keepdim=True).clamp(min=1e-6)
    model = NextItems(scale, seed)
    step = torch.optim.AdamW(model.parameters(), lr=3e-2)
    losses = []
    for i in range(steps):
        logits = model(item, position, row_ptr)
        loss = F.cross_entropy(logits[has_next], target)
        step.zero_grad()
        loss.backward()
        step.step()
        losses.append(float(loss.detach()))
        print(f"step {i}: loss {losses[-1]:.4f}", flush=True)
    lists, scores = answer(model, item, position, row_ptr, beams, length, end=0)
    print(f"first user's lists: {lists[0].tolist()} scores {[round(s, 3) for s in scores[0].tolist()]}",
          flush=True)
    return model, (item, position, row_ptr), losses, lists, scores


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--users", type=int, default=500)
    ap.add_argument("--items", type=int, default=1000)
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    main(a.users, a.items, a.steps)

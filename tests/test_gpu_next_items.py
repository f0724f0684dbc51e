"""The example's whole path: ALS factors, training through the operators, lists by beam search. The
lists are compared with the same search by plain torch over whole histories, without states."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def plain_logits(model, item, position):
    """The model on one history in fp64: logits after its last token."""
    from examples.next_items import HEADS, KEY_HEADS, WIDTH

    p = {k: v.double() for k, v in model.state_dict().items()}
    x = (p["items"][item] @ p["project"].t()).unflatten(1, (-1, WIDTH))
    q, k, v = x.split((HEADS, KEY_HEADS, KEY_HEADS), 1)
    cos, sin = (t.double()[position.long()][:, None] for t in (model.cos, model.sin))

    def normed(x, w):
        y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w
        a, b = y.chunk(2, -1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    q, k = normed(q, p["q_weight"]), normed(k, p["k_weight"])
    k, v = (t.repeat_interleave(HEADS // KEY_HEADS, 1) for t in (k, v))
    gap = torch.arange(item.numel() - 1, -1, -1, device=item.device).double()
    weight = torch.exp(p["log_decay"][None] * gap[:, None]) * (q[-1][None] * k).sum(-1) * WIDTH ** -0.5
    out = (weight[..., None] * v).sum(0)
    return (out.flatten() @ p["join"].t()) @ p["items"].t()


def plain_lists(model, item, position, beams, length, end):
    beam = [(0.0, [], False)]
    for i in range(length):
        cand = []
        for w, (score, tail, done) in enumerate(beam):
            if done:
                cand.append((-score, w, end))
                continue
            at = torch.cat([position, position[-1:].expand(len(tail))])
            s = score + torch.log_softmax(plain_logits(model, torch.cat([item, item.new_tensor(tail)]), at), -1)
            top = torch.sort(s, descending=True, stable=True)
            cand += [(-float(x), w, int(t)) for x, t in zip(top.values[:beams], top.indices[:beams])]
        cand = sorted(cand)[:beams]
        beam = [(-s, beam[w][1] + [t], beam[w][2] or t == end) for s, w, t in cand]
    return [t for _, t, _ in beam], [s for s, _, _ in beam]


def test_example_trains_and_answers():
    sys.path.insert(0, ROOT)
    from examples.next_items import main

    model, (item, position, row_ptr), losses, lists, scores = main(users=60, items=150, steps=12)
    assert losses[-1] < losses[0]
    ptr = row_ptr.tolist()
    rows = [b for b in range(60) if ptr[b + 1] - ptr[b] > 3][:6]
    for b in rows:
        want, want_scores = plain_lists(model, item[ptr[b]:ptr[b + 1]], position[ptr[b]:ptr[b + 1]], 4, 5, 0)
        got = scores[b].tolist()
        print(f"row {b}: {lists[b].tolist()} {got}", flush=True)
        # five log-probabilities of fp32 logits of a few units each
        assert all(abs(x - y) <= 1e-3 for x, y in zip(got, want_scores))
        gaps = [want_scores[i] - want_scores[i + 1] for i in range(3)]
        if min(gaps) > 1e-3:  # else two lists may change places
            assert lists[b].tolist()[:3] == want[:3]

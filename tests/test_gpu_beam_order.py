"""The order of candidates whose scores are equal in 64 bits though their logits differ, as beside a logit of
1e20 or under a score of -1e30: by beam, then by logit, then by item. Cases that gather more candidates
than are ranked at once, and more slices than one round of the merge's threads."""
import math

import pytest

from .test_gpu_sequence import beam_reference, dev, log

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
LARGEST = torch.finfo(torch.float32).max


def ordered_reference(logits, scores, width):
    """[(beam, item)] of each list, by descending score in fp64, beam, descending logit, item. Where the
    largest logit or the score is far above the others, log-sum-exp is what they alone leave."""
    x = logits.double().cpu().nan_to_num(nan=-math.inf, posinf=LARGEST, neginf=-math.inf)
    out = []
    for rows, c in zip(x, scores.double().tolist()):
        cand = []
        for w, row in enumerate(rows):
            top = float(row.max())
            s = (row - top) + (c[w] - math.log(float(torch.exp(row - top).sum())))
            best = torch.sort(row, descending=True, stable=True).indices[:width].tolist()
            cand += [(-float(s[t]), w, -float(row[t]), t) for t in best if row[t] > -math.inf]
        out.append([(w, t) for _, w, _, t in sorted(cand)[:width]])
    return out


def check(logits, scores, width):
    import paper_1108_2580_amd as p

    parents, tokens, *_ = p.beam_select(dev(logits), dev(scores), width=width)
    got = [list(zip(a, b)) for a, b in zip(parents.tolist(), tokens.tolist())]
    want = ordered_reference(logits, scores, width)
    log(f"{tuple(logits.shape)} -> {width}: {got[0][:4]} ...")
    assert got == want


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [30, 5000, 20000])
@pytest.mark.parametrize("high", [1e20, math.inf])
def test_beside_a_logit_that_absorbs_the_others(high, V, dtype):
    g = torch.Generator().manual_seed(V)
    logits = torch.randn(2, 1, V, generator=g).to(dtype)
    logits[:, :, V // 3] = high
    check(logits, torch.zeros(2, 1), 4)


@pytest.mark.parametrize("W,width,V", [(2, 4, 100), (3, 5, 9000), (8, 8, 20000), (32, 32, 20000)])
def test_under_a_score_that_absorbs_the_logits(W, width, V):
    """Of 8 beams of 5 slices, 8 each, all 320 candidates are gathered: they are chosen one at a time."""
    g = torch.Generator().manual_seed(W)
    check(torch.randn(2, W, V, generator=g), torch.full((2, W), -1e30), width)


def test_more_equal_candidates_than_are_ranked_at_once():
    import paper_1108_2580_amd as p

    W, V = 8, 20000
    parents, tokens, *_ = p.beam_select(torch.zeros(1, W, V, device="cuda:0"), torch.zeros(1, W, device="cuda:0"))
    assert parents.tolist() == [[0] * W] and tokens.tolist() == [list(range(W))]
    # few levels in every slice, the same in all beams
    g = torch.Generator().manual_seed(3)
    level = torch.randint(-3, 3, (1, 1, V), generator=g).float().expand(1, W, V).contiguous()
    scores = torch.zeros(1, W)
    want = beam_reference(level, scores, None, -1, W)
    got = p.beam_select(dev(level), dev(scores))
    assert torch.equal(got[0].cpu(), want[0]) and torch.equal(got[1].cpu(), want[1])


def test_more_slices_than_threads_fetch_at_first():
    """32 beams of 153 slices: 4896 sorted lists, of which the merge's threads fetch 4096 ahead."""
    import paper_1108_2580_amd as p

    g = torch.Generator().manual_seed(4)
    logits = torch.randn(1, 32, 624_961, generator=g)
    scores = -torch.rand(1, 32, generator=g) * 0.1
    want = beam_reference(logits, scores, None, -1, 32)
    got = p.beam_select(dev(logits), dev(scores))
    assert torch.equal(got[0].cpu(), want[0]) and torch.equal(got[1].cpu(), want[1])

"""dbias of the attention over gaps of time takes nothing from pairs that a mask leaves out: a query whose scores
are no numbers reaches the buckets of its own row's gaps, and none of those between it and rows that only lie
beside it."""
import math

import pytest

from .test_gpu_gap_attention import bounds_of, inputs, log, reference, run
from .test_gpu_sequence import dev, within

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,last", [(16, 500), (64, 3000), (128, 3000), (64, 100_000)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_lost_query_reaches_its_own_buckets_alone(bad, D, last, dtype):
    """Rows of one time each: all their own gaps are in bucket 0, those to the other rows' tokens are not (the
    rows' times go up and down, so that such gaps have either sign). Only the row in the middle of the tile, whose
    gaps go over many buckets, gives the other buckets anything."""
    import paper_1108_2580_amd as p

    lens, H = [20, 90, 37, 60], 2
    starts = [sum(lens[:i]) for i in range(5)]
    for which in ("q", "k"):
        for row in (0, 2, 3):
            q, k, v, bias, bounds, pos, ptr, do = inputs(lens, H, 1, D, 24, dtype, 71, last)
            a, b = starts[row], starts[row + 1]
            for r, time in ((0, 5 * last), (2, 7 * last), (3, 4 * last)):
                pos[starts[r]:starts[r + 1]] = time
            want = reference(q, k, v, bias, bounds, pos, ptr, 0.2, do)
            q, k = q.clone(), k.clone()
            # every other feature: scores of infinities are infinite or NaN, and so is each row's sum
            (q if which == "q" else k)[a + 5, :, ::2] = bad
            got = run(p, q, k, v, bias, bounds, pos, ptr, do, 0.2)
            log(f"{bad} in {which}, row {row}, width {D}, last bound {last}, {dtype}")
            limit = bounds_of(want, "dbias", D, dtype, H)
            within(got["dbias"][:, 1:], want["dbias"][:, 1:], limit[:, 1:], "dbias")
            if math.isnan(bad):
                assert torch.isnan(got["dbias"][:, 0]).all()
                lost = torch.zeros(sum(lens), dtype=torch.bool)
                lost[a + 5:a + 6 if which == "q" else b] = True
                assert torch.equal(torch.isnan(got["dq"]).all(-1).all(-1).cpu(), lost)
                assert torch.equal(torch.isnan(got["dq"]).any(-1).any(-1).cpu(), lost)


def test_a_lost_bucket_leaves_the_others():
    """A bias of NaN: its own bucket and those that the rows' queries with such a gap read are NaN, and no other."""
    import paper_1108_2580_amd as p

    q, k, v, bias, _, _, ptr, do = inputs([30, 34], 2, 2, 32, 6, "f32", 72)
    bounds = torch.tensor([1, 10, 20, 30, 40], dtype=torch.int32)
    # the first row's gaps are in buckets 0 and 3, the second's in 0, 1 and 2; from the first row to the second's: 3 to 5
    pos = torch.cat([torch.tensor([100] * 15 + [125] * 15), torch.tensor([60] * 10 + [64] * 12 + [75] * 12)]).int()
    want = reference(q, k, v, bias, bounds, pos, ptr, 0.2, do)
    bias[1, 3] = math.nan
    got = run(p, q, k, v, bias, bounds, dev(pos), ptr, do, 0.2)
    nan = torch.isnan(got["dbias"].cpu())
    assert nan[1].tolist() == [True, False, False, True, False, False] and not nan[0].any()
    limit = bounds_of(want, "dbias", 32, "f32")
    within(got["dbias"][0], want["dbias"][0], limit[0], "dbias")
    within(got["dbias"][1, [1, 2, 4, 5]], want["dbias"][1, [1, 2, 4, 5]], limit[1, [1, 2, 4, 5]], "dbias")

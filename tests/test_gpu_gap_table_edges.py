"""Bounds around the end of the table of gaps (the last bound of 7679 is the last that a table holds, 7680 is
searched for): the same values on both sides, right ones at gaps next to the bounds."""
import pytest

from .test_gpu_gap_attention import check, check_step, inputs, log, reference, run, step_inputs, step_reference
from .test_gpu_sequence import dev

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
LAST = 7679  # include/als.h


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("last", [LAST - 1, LAST, LAST + 1, 8191, 8192])
def test_gaps_next_to_the_last_bounds(last, D, dtype):
    import paper_1108_2580_amd as p

    log(f"last bound {last}, width {D}, {dtype}")
    q, k, v, bias, _, _, ptr, do = inputs([60, 90], 2, 1, D, 6, dtype, 81)
    bounds = torch.tensor([1, 2, 4000, last - 1, last], dtype=torch.int32)
    near = torch.tensor([0, 1, 2, 3999, 4000, 4001, last - 2, last - 1, last, last + 1, last + 2, 2 * last, 9000])
    pos = torch.cat([near[torch.arange(n) % near.numel()].sort().values for n in (60, 90)]).int()
    args = (q, k, v, bias, bounds, dev(pos), ptr)
    got = run(p, *args, do, 0.2)
    check(reference(*args, 0.2, do), got, D, dtype, 2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_step_next_to_the_last_bounds(dtype):
    import paper_1108_2580_amd as p

    for last in (LAST, LAST + 1):
        q, k, v, bias, bounds, q_pos, pos, ptr, kp, vp, p_pos, path = step_inputs([70, 30], 4, 3, 4, 2, 40, 6, dtype, 82)
        bounds = torch.tensor([1, 2, 4000, last - 1, last], dtype=torch.int32)
        pos = dev((torch.arange(100) % 5 + 1).int())
        q_pos[:] = last + 3  # gaps from last - 2 to last + 2
        p_pos[:] = last + 3 - torch.arange(p_pos.numel(), device="cuda:0", dtype=torch.int32).view_as(p_pos) % 3
        args = (q, k, v, bias, bounds, q_pos, pos, ptr, kp, vp, p_pos, path)
        check_step(p.gap_attention_step(*args, scale=0.2), step_reference(*args, 0.2), 40, dtype)

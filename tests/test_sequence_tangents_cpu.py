"""Tangents of forward-mode derivatives are refused, not dropped: the operators have none to give. The check comes
before any of the tensors' places, so these run without a GPU."""
import pytest

from paper_1108_2580_amd import sequence as s

torch = pytest.importorskip("torch")
fwad = torch.autograd.forward_ad


def calls():
    """(name, function, arguments, which of them may carry derivatives)"""
    x, w, table = torch.ones(4, 2, 8), torch.ones(8), torch.ones(9, 4)
    pos, ptr = torch.zeros(4, dtype=torch.int32), torch.tensor([0, 4])
    bounds = torch.tensor([1, 2], dtype=torch.int32)
    yield s.norm_rotate, [x, x, w, w, table, table, pos], range(6)
    yield s.decay_attention, [x, x, x, torch.zeros(2), ptr], range(4)
    yield s.decay_attention, [x, x, x, torch.zeros(2), ptr, None, torch.zeros(1, 2, 8, 8)], [6]
    yield s.gap_attention, [x, x, x, torch.zeros(2, 3), bounds, pos, ptr], range(4)


@pytest.mark.parametrize("case", range(4))
def test_a_tangent_is_refused(case):
    call, args, which = list(calls())[case]
    for i in which:
        for leaf in (False, True):  # with a gradient of the other kind as well
            with fwad.dual_level():
                given = list(args)
                given[i] = fwad.make_dual(given[i].clone().requires_grad_(leaf), torch.ones_like(given[i]))
                for grads in (torch.enable_grad(), torch.no_grad()):
                    with grads, pytest.raises(ValueError, match="tangent"):
                        call(*given)


@pytest.mark.parametrize("case", range(4))
def test_tensors_without_one_are_not(case):
    call, args, _ = list(calls())[case]
    with fwad.dual_level(), pytest.raises(TypeError, match="q must be a CUDA"):
        call(*args)

"""clear_unheld of the attentions' shapes is 0 or 1, refused otherwise before any device call. Pointers are made up
and never followed."""
import pytest

from paper_1108_2580_amd import lib
from paper_1108_2580_amd.sequence import _Attention, _Heads

from .test_gap_attention_cpu import A, B, C, D, E, F, W, back, gaps, read, refused, step, path


@pytest.mark.parametrize("value", [-1, 2, 1 << 30])
def test_refusals(value):
    for call in (read, back):
        refused(call(gaps(clear_unheld=value)), "clear_unheld")
    refused(step(gaps(clear_unheld=value), path()), "clear_unheld")
    shape = _Attention(5000, 3, A, B, 4, 2, 64, 64, 0.1, value)
    q, k = _Heads(C, 256, 64), _Heads(D, 128, 64)
    refused(lib.als_decay_attention(shape, 1, q, k, k, None, E, None, W, 1 << 40, None), "clear_unheld")
    refused(lib.als_decay_attention_backward(shape, 1, q, q, k, k, None, None, E, F, W, None, W, 1 << 40, None),
            "clear_unheld")

"""The attention workspaces' sizes: states are needed only between the segments of long rows, so that a batch of
many short rows takes a place for each and no state."""
import pytest

from paper_1108_2580_amd import lib
from paper_1108_2580_amd.sequence import _Attention


def sizes(n_tokens, n_rows, heads, width):
    s = _Attention(n_tokens, n_rows, 1 << 20, 1 << 20, heads, heads, width, width, 1.0)
    return lib.als_decay_attention_workspace(s), lib.als_decay_attention_backward_workspace(s)


@pytest.mark.parametrize("rows,each", [(100_000, 5), (100_000, 20), (1_000_990, 5), (1_000_990, 262)])
@pytest.mark.parametrize("heads,width", [(8, 64), (8, 128)])
def test_short_rows_take_no_states(rows, each, heads, width):
    tokens = rows * each
    few, many = sizes(tokens, 1_000, heads, width), sizes(tokens, rows, heads, width)
    for a, b in zip(few, many):
        assert 0 < b - a <= 32 * (rows - 1_000) + 64  # a place is 24 bytes
    # at these sizes a segment is of 2048 tokens, and a state of fp32
    state = 4 * heads * width * width
    assert many[0] <= (tokens // 2048) * (state + 32) + 32 * rows + 64
    assert many[1] <= (tokens // 2048) * (2 * state + 32) + 32 * rows + 64


def test_no_segments_no_states():
    assert sizes(100, 60, 8, 64) == (0, 0)
    assert sizes(100, 100, 8, 64)[0] <= 32 * 100 + 64

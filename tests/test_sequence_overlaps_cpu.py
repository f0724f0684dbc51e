"""States and weights' gradients that lie on other tensors of the call are refused. Pointers are made up and
never followed."""
import pytest

from paper_1108_2580_amd import lib
from paper_1108_2580_amd.sequence import _Attention, _Heads, _Rotation

INVALID = 1
TOKENS, HEADS, WIDTH, ROWS = 100, 4, 64, 3
STATES = 4 * ROWS * HEADS * WIDTH * WIDTH      # bytes of all states
TENSOR = 4 * TOKENS * HEADS * WIDTH            # bytes of q, k, v, out or a gradient
at = lambda i: 0x10000000 * (i + 1)  # noqa: E731  (buffers 256 MiB apart)
SHAPE = _Attention(TOKENS, ROWS, at(0), at(0), HEADS, HEADS, WIDTH, WIDTH, 1.0)


def heads(p):
    return _Heads(p, HEADS * WIDTH, WIDTH)


def refused(status, word):
    msg = lib.als_last_error(None).decode()
    assert status == INVALID and word in msg, (status, msg)


def forward(q=at(1), k=at(2), v=at(3), first=at(4), out=at(5), last=at(6)):
    return lib.als_decay_attention(SHAPE, 0, heads(q), heads(k), heads(v), first, out, last, at(15), -1, None)


def backward(do=at(1), q=at(2), k=at(3), v=at(4), first=at(5), dlast=at(6), dq=at(7), dk=at(8), dv=at(9), dfirst=at(10)):
    return lib.als_decay_attention_backward(SHAPE, 0, heads(do), heads(q), heads(k), heads(v), first, dlast, dq, dk, dv,
                                            dfirst, at(15), -1, None)


def test_calls_without_overlaps_pass_these_checks():
    refused(forward(), "workspace")   # of -1 bytes: refused after all other checks
    refused(backward(), "workspace")


@pytest.mark.parametrize("name,place", [("q", at(1)), ("k", at(2)), ("v", at(3)), ("out", at(5)), ("first", at(4))])
@pytest.mark.parametrize("shift", [0, 256, -256])
def test_final_state(name, place, shift):
    size = STATES if name == "first" else TENSOR
    refused(forward(last=place + (shift if shift >= 0 else size + shift)), "overlaps")
    refused(forward(**{name: at(6) + (shift if shift >= 0 else STATES + shift)}), "overlaps")


@pytest.mark.parametrize("shift", [0, STATES - 4, 4 - TENSOR])
def test_out_on_the_initial_state(shift):
    refused(forward(out=at(4) + shift), "overlaps")


@pytest.mark.parametrize("name", ["do", "q", "k", "v", "first", "dlast", "dq", "dk", "dv"])
@pytest.mark.parametrize("shift", [0, 256])
def test_initial_states_gradient(name, shift):
    refused(backward(**{name: at(10) + shift}), "overlaps")


@pytest.mark.parametrize("name", ["dq", "dk", "dv"])
@pytest.mark.parametrize("state", [at(5), at(6)])
def test_gradients_on_states(name, state):
    refused(backward(**{name: state + STATES - 4}), "overlaps")


@pytest.mark.parametrize("i", [0, 1, 2])
def test_a_steps_state_on_an_input(i):
    x = [at(1), at(2), at(3)]
    x[i] = at(6) + 64
    shape = _Attention(0, ROWS, None, at(0), HEADS, HEADS, WIDTH, WIDTH, 1.0)
    refused(lib.als_decay_attention_step(shape, 0, *map(heads, x), at(4), ROWS, None, at(6), at(5), None), "overlaps")


@pytest.mark.parametrize("dqw,dkw", [(at(6), at(6) + 4), (at(7), at(4) + 64), (at(5) + TENSOR - 4, at(8))])
def test_weights_gradients(dqw, dkw):
    s = _Rotation(TOKENS, 5, HEADS, HEADS, WIDTH, WIDTH, 0, 1e-6, at(0), at(0), at(0))
    refused(lib.als_norm_rotate_backward(s, 0, heads(at(0)), heads(at(1)), heads(at(2)), heads(at(3)), at(9), at(9),
                                         heads(at(4)), heads(at(5)), dqw, dkw, at(15), -1, None), "overlap")


def test_tensors_without_tokens_overlap_nothing():
    shape = _Attention(0, ROWS, at(0), at(0), HEADS, HEADS, WIDTH, WIDTH, 1.0)
    inside = at(6) + 64
    refused(lib.als_decay_attention(shape, 0, heads(inside), heads(inside), heads(inside), at(4), inside, at(6), at(15),
                                    -1, None), "workspace")

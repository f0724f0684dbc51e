"""What attention's products keep of their operands. An operand that is not held in its inputs' bf16 goes
into a product in parts of 8 bits each: the weights and the state that bf16 queries read in two, what a
token adds to a state, and every fp32 operand, in three.

Bounds, with the sizes and the fp32 terms of test_gpu_sequence. Of two parts the first cuts the lower bits
off (less than 2^-7 of the value are left) and the second is rounded to nearest, which leaves at most 2^-7 *
2^-9 = 2^-16 of the value."""
import pytest

from .test_gpu_sequence import E, U, attention_inputs, attention_reference, log, within

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def sizes(q, k, v, a, lens, scale, S0, d_out, dS):
    mag = lambda t: None if t is None else t.abs()  # noqa: E731
    return attention_reference(mag(q), mag(k), mag(v), a, lens, scale, mag(S0), mag(d_out), mag(dS))


@pytest.mark.parametrize("lens,H,Hk,K,V", [
    ([64, 3, 0, 130], 4, 2, 64, 64), ([200, 65], 2, 1, 128, 128), ([150], 4, 4, 33, 50), ([70] * 3, 2, 2, 128, 40),
    ([90, 1], 2, 1, 20, 100), ([700, 300], 2, 2, 64, 32)])
def test_bf16_outputs_are_rounded_once(lens, H, Hk, K, V):
    import paper_1108_2580_amd as p

    q, k, v, a, ptr, d_out, S0, dS = attention_inputs(lens, H, Hk, K, V, "bf16", 77 + K)
    want = attention_reference(q, k, v, a, lens, 0.37, S0, d_out, dS)
    size = sizes(q, k, v, a, lens, 0.37, S0, d_out, dS)
    terms = max(lens) + K + V + 48
    log(f"lengths {lens}, {H}/{Hk} heads, {K} x {V}")
    o = p.decay_attention(q, k, v, a, ptr, 0.37, S0)
    grads = p.decay_attention_backward(d_out, q, k, v, a, ptr, 0.37, S0, dS)
    for got, i, name in ((o, 0, "out"), (grads[0], 2, "dq"), (grads[1], 3, "dk"), (grads[2], 4, "dv")):
        # a weight (or the state) is off by 2^-16 of itself, the output by its rounding
        bound = U * want[i].abs() + (2.0 ** -16 + terms * E) * 1.01 * size[i] + 1e-30
        within(got, want[i], bound, name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,K,V", [([200, 7], 64, 64), ([3000], 64, 64), ([150], 128, 128)])
def test_outputs_do_not_depend_on_the_states_asked_for(lens, K, V, dtype):
    import paper_1108_2580_amd as p

    q, k, v, a, ptr, d_out, S0, dS = attention_inputs(lens, 4, 2, K, V, dtype, 5)
    args = (q, k, v, a, ptr, 0.5, S0)
    assert torch.equal(p.decay_attention(*args), p.decay_attention(*args, return_state=True)[0])
    less = p.decay_attention_backward(d_out, *args, dS, d_initial=False)
    more = p.decay_attention_backward(d_out, *args, dS, d_initial=True)
    for x, y in zip(less[:3], more[:3]):
        assert torch.equal(x, y)

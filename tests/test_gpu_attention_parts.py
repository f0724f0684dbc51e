"""What attention's products keep of their operands. An operand that is not held in its inputs' bf16 goes
into a product in parts of 8 bits each: the weights and the state that bf16 queries read in two, what a
token adds to a state, and every fp32 operand, in three.

Bounds, with the sizes and the fp32 terms of test_gpu_sequence. The first part cuts the lower bits off (less
than 2^-7 of the value are left); the second is rounded to nearest, which leaves 2^-7 * 2^-9 = 2^-16 of it: so
much may two parts be off. Of a product of three parts each, those that are left out are at most 2^-7 *
2^-16, twice, and their signs are as random as the second part's rounding."""
import math

import pytest

from .test_gpu_sequence import E, U, attention_inputs, attention_reference, dev, log, within

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


def mantissas(n, seed):
    """fp32 values of any 24 bits, from 1 to 2, with a sign."""
    g = torch.Generator().manual_seed(seed)
    bits = torch.randint(0, 1 << 23, (n,), generator=g, dtype=torch.int32) | 0x3f800000
    sign = torch.randint(0, 2, (n,), generator=g).float() * 2 - 1
    return bits.view(torch.float32) * sign


def test_fp32_products_lean_to_neither_side():
    """Rows of one token with heads one wide: out = q k v, two products of parts. Each is off by its
    rounding, at most 2^-23 of it, and by what is left out, at most 2 * 2^-23; neither has a preferred sign, so
    that the mean of n errors of at most s = 3 * 2^-22 is within 6 s / sqrt(n) of zero."""
    import paper_1108_2580_amd as p

    n = 1 << 16
    q, k, v = (mantissas(n, i).view(n, 1, 1) for i in (1, 2, 3))
    want = (q.double() * k.double() * v.double()).flatten()
    a = torch.zeros(1, device="cuda:0")
    ptr = torch.arange(n + 1, device="cuda:0")
    o, S = p.decay_attention(dev(q), dev(k), dev(v), a, ptr, 1.0, return_state=True)
    off = (o.flatten().double().cpu() - want) / want
    log(f"  out: largest {float(off.abs().max()) / E:.2f} e, mean {float(off.mean()) / E:.4f} e")
    assert float(off.abs().max()) <= 3 * 2.0 ** -22
    assert abs(float(off.mean())) <= 6 * 3 * 2.0 ** -22 / math.sqrt(n)


def test_fp32_lowest_values_stay_finite():
    """The type's lowest value, as a mask leaves it: its parts' sum is the value itself."""
    import paper_1108_2580_amd as p

    low = torch.finfo(torch.float32).min
    one = torch.ones(3, 1, 8, device="cuda:0")
    v = torch.full((3, 1, 8), low, device="cuda:0")
    q = torch.zeros_like(one)
    q[..., 0] = 1.0
    a = torch.full((1,), -math.inf, device="cuda:0")
    ptr = torch.tensor([0, 3], device="cuda:0")
    o, S = p.decay_attention(q, one, v, a, ptr, 1.0, return_state=True)
    assert (o == low).all() and (S == low).all()

"""What attention's products keep of their operands. What a token adds to a state goes into its product in
three bf16 parts, whatever is asked for."""
import pytest

from .test_gpu_sequence import attention_inputs

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


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

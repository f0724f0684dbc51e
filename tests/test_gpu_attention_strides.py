"""Attention on views with strides far above their widths."""
import pytest

from .test_gpu_sequence import attention_inputs

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("stride", [1 << 22, 1 << 27, 1 << 40])
def test_one_token_of_any_stride(stride, dtype):
    """A slice of one token keeps the stride of the tensor that it was cut from, which no pass may use."""
    import paper_1108_2580_amd as p

    q, k, v, a, ptr, d_out, S0, dS = attention_inputs([1], 4, 2, 64, 48, dtype, 30)
    far = lambda t: t.as_strided(t.shape, (stride, *t.stride()[1:]))  # noqa: E731
    want = [*p.decay_attention(q, k, v, a, ptr, None, S0, return_state=True),
            *p.decay_attention_backward(d_out, q, k, v, a, ptr, None, S0, dS)]
    got = [*p.decay_attention(far(q), far(k), far(v), a, ptr, None, S0, return_state=True),
           *p.decay_attention_backward(far(d_out), far(q), far(k), far(v), a, ptr, None, S0, dS)]
    for x, y in zip(got, want):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_steps_of_rows_far_apart(dtype):
    """Rows more than 2^22 values apart, as one token of each history in a padded batch."""
    import paper_1108_2580_amd as p

    q, k, v, a, _, _, S0, _ = attention_inputs([1, 1, 1], 4, 2, 64, 48, dtype, 31)
    apart = (1 << 22) + 8

    def far(t):
        n = t[0].numel()
        x = torch.empty(2 * apart + n, dtype=t.dtype, device=t.device).as_strided((3, n), (apart, 1))
        return x.copy_(t.flatten(1)).unflatten(1, t.shape[1:])

    want = p.decay_attention_step(q, k, v, a, S0.clone())
    got = p.decay_attention_step(far(q), far(k), far(v), a, S0.clone())
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_gradient_of_tokens_far_apart():
    """The output's gradient has the strides that a graph gives it, whatever those of the call were."""
    import paper_1108_2580_amd as p

    q, k, v, a, ptr, d_out, *_ = attention_inputs([2, 1], 2, 2, 16, 16, "f32", 32)
    q = q.clone().requires_grad_()
    o = p.decay_attention(q, k, v, a, ptr)
    apart = (1 << 22) + 8
    far = torch.empty(2 * apart + 32, device="cuda:0").as_strided((3, 2, 16), (apart, 16, 1)).copy_(d_out)
    want, = torch.autograd.grad(o, q, d_out, retain_graph=True)
    got, = torch.autograd.grad(o, q, far)
    assert torch.equal(got, want)

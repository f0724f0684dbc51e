"""What the operators write in place is seen by autograd, and gradients that they do not give are refused
rather than dropped."""
import pytest

from .test_gpu_sequence import attention_inputs

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def step_inputs(n, g):
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda:0")  # noqa: E731
    return rnd(n, 4, 8), rnd(n, 2, 8), rnd(n, 2, 12), torch.full((4,), -0.1, device="cuda:0")


@pytest.mark.parametrize("how", ["in place", "state_out", "reorder"])
def test_a_saved_state_that_is_written_raises(how):
    import paper_1108_2580_amd as p

    q, k, v, a, ptr, d_out, S0, _ = attention_inputs([9, 20], 4, 2, 8, 12, "f32", 4)
    o = p.decay_attention(q.clone().requires_grad_(), k, v, a, ptr, initial_state=S0)
    before = S0._version
    step = step_inputs(2, torch.Generator(device="cuda:0").manual_seed(1))
    if how == "in place":
        p.decay_attention_step(*step, S0)
    elif how == "state_out":
        p.decay_attention_step(*step, S0.clone(), state_out=S0)
    else:
        parents = torch.zeros(1, 2, dtype=torch.int32, device="cuda:0")
        p.reorder_states(S0[None].clone(), parents, out=S0[None])
    assert S0._version > before
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        (o * d_out).sum().backward()


def test_states_that_are_only_read_may_be_saved():
    import paper_1108_2580_amd as p

    q, k, v, a, ptr, d_out, S0, _ = attention_inputs([9, 20], 4, 2, 8, 12, "f32", 4)
    x = q.clone().requires_grad_()
    o = p.decay_attention(x, k, v, a, ptr, initial_state=S0)
    step = step_inputs(2, torch.Generator(device="cuda:0").manual_seed(1))
    source = torch.tensor([1, 0], dtype=torch.int32, device="cuda:0")
    p.decay_attention_step(*step, S0, source=source)
    p.reorder_states(S0[None], source[None])
    (o * d_out).sum().backward()
    assert torch.isfinite(x.grad).all()


def test_a_state_that_requires_a_gradient_is_not_written():
    import paper_1108_2580_amd as p

    step = step_inputs(2, torch.Generator(device="cuda:0").manual_seed(1))
    state = torch.zeros(2, 4, 8, 12, device="cuda:0", requires_grad=True)
    other = torch.zeros(2, 4, 8, 12, device="cuda:0")
    parents = torch.zeros(1, 2, dtype=torch.int32, device="cuda:0")
    for call in (lambda: p.decay_attention_step(*step, state),
                 lambda: p.decay_attention_step(*step, other, state_out=state),
                 lambda: p.reorder_states(other[None], parents, out=state[None])):
        held = state.detach().clone()
        with pytest.raises(ValueError, match="gradient"):
            call()
        assert torch.equal(state, held)
        with torch.no_grad():
            call()
    with torch.inference_mode():  # tensors without a version
        held = torch.zeros(2, 4, 8, 12, device="cuda:0")
        p.decay_attention_step(*step, held)
        p.reorder_states(held[None], parents, out=held[None])


def test_tables_take_no_gradient():
    import paper_1108_2580_amd as p

    x = torch.randn(4, 2, 16, device="cuda:0")
    w = torch.ones(16, device="cuda:0")
    pos = torch.zeros(4, dtype=torch.int32, device="cuda:0")
    for i in range(2):
        tables = list(p.rotary_tables(10, 16))
        tables[i].requires_grad_()
        for q in (x, x.clone().requires_grad_()):
            with pytest.raises(ValueError, match="gradient"):
                p.norm_rotate(q, x, w, w, *tables, pos)
        with torch.no_grad():
            p.norm_rotate(x, x, w, w, *tables, pos)

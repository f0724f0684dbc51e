"""Attention over more rows than are searched for a block's place: tables of places and entries, with rows
of none, one and several segments; joins over entries (where those are fewer than rows) and over rows.
Values and gradients with test_gpu_sequence's bounds."""
import pytest

from .test_gpu_sequence import attention_inputs, test_attention_and_gradients as check

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

ROWS = [  # lengths; segments are of 128 (f32) or 256 (bf16) tokens
    [0, 5, 700, 1, 300, 0, 64, 130] * 9,     # 72 rows; 84 entries in f32, 42 in bf16
    [300, 0, 520, 257] * 17,                 # 68 rows; 143 and 71 entries
    [5, 0, 300, 129, 60] * 26]               # 130 rows; 100 and 50 entries


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,H,Hk,K,V", [(ROWS[0], 2, 1, 24, 16), (ROWS[1], 2, 2, 16, 33), (ROWS[2], 4, 2, 16, 16)])
def test_many_rows_of_several_segments(lens, H, Hk, K, V, dtype):
    check(lens, H, Hk, K, V, True, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_do_not_depend_on_the_rows_beside_them(dtype):
    """A long row alone and among others, cut into the same segments: bitwise the same."""
    import paper_1108_2580_amd as p

    lens = [0, 3, 1500] + [2] * 80 + [1024, 0, 900]
    q, k, v, a, ptr, d_out, S0, dS = attention_inputs(lens, 4, 2, 64, 48, dtype, 21)
    o, S = p.decay_attention(q, k, v, a, ptr, None, S0, return_state=True)
    grads = p.decay_attention_backward(d_out, q, k, v, a, ptr, None, S0, dS)
    at = ptr.tolist()
    for b in (2, 83, 85):
        cut = slice(at[b], at[b + 1])
        one = (q[cut], k[cut], v[cut], a, ptr.new_tensor([0, lens[b]]), None, S0[b:b + 1])
        o1, S1 = p.decay_attention(*one, return_state=True)
        assert torch.equal(o1, o[cut]) and torch.equal(S1[0], S[b])
        for x, y, part in zip(p.decay_attention_backward(d_out[cut], *one, dS[b:b + 1]), grads,
                              (cut, cut, cut, slice(b, b + 1))):
            assert torch.equal(x, y[part])

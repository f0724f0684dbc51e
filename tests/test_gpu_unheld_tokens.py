"""Tokens that no row holds (padding before the first row and behind the last) count as nothing where autograd
records the attentions: their outputs and gradients are zero, whatever the new tensors held before, so that what
sums over all tokens is what the rows alone give."""
import math

import pytest

from .test_gpu_sequence import DTYPES, E, dev, log

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

# tokens before the rows, the rows, tokens behind them
BATCHES = [(0, [30, 41], 70), (3, [30, 0, 41], 0), (130, [64], 1), (5, [2] * 80, 9), (7, [0], 20), (0, [200], 0)]


@pytest.fixture
def poisoned(monkeypatch):
    """New tensors hold NaN."""
    empty = torch.Tensor.new_empty
    monkeypatch.setattr(torch.Tensor, "new_empty", lambda *a, **kw: empty(*a, **kw).fill_(math.nan))


def batch(before, lens, after, W, seed):
    g = torch.Generator().manual_seed(seed)
    N = before + sum(lens) + after
    ptr = torch.tensor([0] + lens).cumsum(0) + before
    held = torch.zeros(N, dtype=torch.bool)
    held[before:before + sum(lens)] = True
    x = dev(torch.randn(N, W, generator=g))
    return g, N, dev(ptr), dev(held), x


def same_sum(got, x, of_tokens, held):
    """got: the gradient of a weight whose products with x have the gradients of_tokens."""
    a, b = x[held].double().T, of_tokens[held].double().flatten(1)
    size = a.abs() @ b.abs()
    off = (got.double().view_as(size) - a @ b).abs()
    # a sum over the tokens in fp32
    assert (off <= (held.numel() + 2) * E * size + 1e-30).all(), float((off / (size + 1e-30)).max())


def parts(y, q, k, D):
    y = y.unflatten(1, (-1, D))
    return y[:, :q], y[:, q:q + k], y[:, q + k:]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("before,lens,after", BATCHES)
def test_projections_around_gap_attention(before, lens, after, dtype, poisoned):
    import paper_1108_2580_amd as p

    H, Hk, D, W = 4, 2, 24, 16
    log(f"{before} tokens, rows {lens[:4]}, {after} tokens, {dtype}")
    g, N, ptr, held, x = batch(before, lens, after, W, 1)
    weight = dev(torch.randn(W, (H + 2 * Hk) * D, generator=g)).requires_grad_()
    back = dev(torch.randn(H * D, W, generator=g)).requires_grad_()
    bias = dev(torch.randn(H, 5, generator=g)).requires_grad_()
    bounds = torch.tensor([1, 4, 20, 100], dtype=torch.int32)
    pos = dev(torch.randint(0, 300, (N,), generator=g).int())
    qkv = parts((x @ weight).to(DTYPES[dtype]), H, Hk, D)
    out = p.gap_attention(*qkv, bias, bounds, pos, ptr, 0.2)
    assert not out[~held].any()
    y = out.float().flatten(1) @ back
    d_y = dev(torch.randn(N, W, generator=g)) * held[:, None]
    grads = torch.autograd.grad(y, (weight, back, bias), d_y)
    assert all(torch.isfinite(t).all() for t in grads)

    args = (*(t.detach() for t in qkv), bias.detach(), bounds, pos, ptr, 0.2)
    plain, saved = p.gap_attention(*args, return_saved=True)
    assert torch.equal(plain[held], out.detach()[held])
    d_out = (d_y @ back.detach().T).unflatten(1, (H, D)).to(DTYPES[dtype])
    dq, dk, dv, dbias = p.gap_attention_backward(d_out, plain, saved, *args)
    assert torch.equal(grads[2], dbias)
    same_sum(grads[0], x, torch.cat([dq, dk, dv], 1), held)
    same_sum(grads[1], plain.float().flatten(1), d_y, held)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("before,lens,after", BATCHES)
def test_projections_around_decay_attention(before, lens, after, dtype, poisoned):
    import paper_1108_2580_amd as p

    H, Hk, D, W = 4, 2, 24, 16
    log(f"{before} tokens, rows {lens[:4]}, {after} tokens, {dtype}")
    g, N, ptr, held, x = batch(before, lens, after, W, 2)
    weight = dev(torch.randn(W, (H + 2 * Hk) * D, generator=g)).requires_grad_()
    back = dev(torch.randn(H * D, W, generator=g)).requires_grad_()
    decay = dev(-torch.rand(H, generator=g))
    qkv = parts((x @ weight).to(DTYPES[dtype]), H, Hk, D)
    out = p.decay_attention(*qkv, decay, ptr, 0.2)
    assert not out[~held].any()
    d_y = dev(torch.randn(N, W, generator=g)) * held[:, None]
    grads = torch.autograd.grad(out.float().flatten(1) @ back, (weight, back), d_y)
    assert all(torch.isfinite(t).all() for t in grads)

    args = (*(t.detach() for t in qkv), decay, ptr, 0.2)
    plain = p.decay_attention(*args)
    assert torch.equal(plain[held], out.detach()[held])
    d_out = (d_y @ back.detach().T).unflatten(1, (H, D)).to(DTYPES[dtype])
    dq, dk, dv, _ = p.decay_attention_backward(d_out, *args)
    same_sum(grads[0], x, torch.cat([dq, dk, dv], 1), held)
    same_sum(grads[1], plain.float().flatten(1), d_y, held)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K,V,offset", [(1, 1, 0), (5, 3, 1), (24, 50, 3), (64, 128, 0)])
@pytest.mark.parametrize("rows", ["few", "many"])
def test_decay_attention_clears_its_places_and_no_others(rows, K, V, offset, dtype):
    """At any alignment of the type; row pointers out of range touch nothing outside. Without clear_unheld all such
    places stay as they are."""
    from paper_1108_2580_amd import lib, sequence as s

    N, H, size = 300, 2, 4 if dtype == "f32" else 2
    q = dev(torch.ones(N, H, K, dtype=DTYPES[dtype]))
    v, decay = dev(torch.ones(N, H, V, dtype=DTYPES[dtype])), dev(-torch.ones(H))
    between = [] if rows == "few" else [40 + i // 2 for i in range(90)]
    for a, b in ((0, 300), (30, 290), (39, 131), (-4, 1 << 40), (400, 400), (7, 7)):
        ptr = [a] + (between if a < 40 and b > 85 else []) + [b]
        t = dev(torch.tensor(ptr))
        first, end = min(max(a, 0), N), min(max(b, 0), N)
        for clear in (0, 1):
            dev_, code, shape, hq, hk, hv = s._attention(q, q, v, decay, t, 1.0)
            shape.clear_unheld = clear
            need = lib.als_decay_attention_workspace(shape)
            work = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda:0")
            whole = torch.full((512 + size * (offset + N * H * V),), 0xA5, dtype=torch.uint8, device="cuda:0")
            at = 256 + size * offset
            s._check(lib.als_decay_attention(shape, code, hq, hk, hv, None, whole.data_ptr() + at, None, work.data_ptr(),
                                             need, s._stream(dev_)))
            out = whole[at:at + N * H * V * size].view(N, -1)
            empty = 0 if clear else 0xA5
            assert (out[:first] == empty).all() and (out[end:] == empty).all(), (ptr, clear)
            assert (whole[:at] == 0xA5).all() and (whole[at + N * H * V * size:] == 0xA5).all()
            if 0 <= a < b <= N:
                assert (out[first:end].contiguous().view(DTYPES[dtype]) > 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hk,D", [(2, 2, 7), (4, 1, 50), (2, 1, 128)])
@pytest.mark.parametrize("before,lens,after", [(3, [30, 0, 41], 200), (130, [64], 1), (5, [2] * 80, 9), (70, [0], 3)])
def test_gap_attention_gives_zeros(before, lens, after, H, Hk, D, dtype, poisoned):
    """Also where nothing is recorded; padding of NaN reaches nothing."""
    import paper_1108_2580_amd as p

    log(f"{before} tokens, rows {lens[:4]}, {after} tokens, {H}/{Hk} heads, width {D}, {dtype}")
    g, N, ptr, held, _ = batch(before, lens, after, 1, 3)
    q, do = (dev(torch.randn(N, H, D, generator=g).to(DTYPES[dtype])) for _ in range(2))
    k, v = (dev(torch.randn(N, Hk, D, generator=g).to(DTYPES[dtype])) for _ in range(2))
    for t in (q, k, v, do):
        t[~held] = math.nan
    bias, bounds = dev(torch.randn(H, 3, generator=g)), torch.tensor([1, 50], dtype=torch.int32)
    pos = dev(torch.randint(0, 300, (N,), generator=g).int())
    args = (q, k, v, bias, bounds, pos, ptr, 0.3)
    out, saved = p.gap_attention(*args, return_saved=True)
    grads = p.gap_attention_backward(do, out, saved, *args)
    for t in (out, *grads[:3]):
        assert not t[~held].any() and torch.isfinite(t).all()
    assert torch.isfinite(grads[3]).all()
    if sum(lens):
        assert out[held].any() and all(t[held].any() for t in grads[:3])

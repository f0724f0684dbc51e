"""Tokens that no row holds (padding before the first row and behind the last) count as nothing where autograd
records the attentions: their outputs and gradients are zero, whatever the new tensors held before, so that what
sums over all tokens is what the rows alone give."""
import ctypes
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


@pytest.mark.parametrize("width,offset", [(1, 0), (2, 3), (13, 1), (48, 0), (100, 7), (4096, 5)])
def test_places_are_cleared_and_no_others(width, offset):
    """At any alignment and number of bytes a token; row pointers out of range touch nothing outside."""
    from paper_1108_2580_amd import lib, sequence as s

    N = 300
    for ptr, first, end in (([0, 300], 0, 300), ([3, 290], 3, 290), ([0, 0], 0, 0), ([17], 17, 17), ([300, 300], 300, 300),
                            ([-4, 5, 1 << 40], 0, 300), ([7, 2], 7, 7), ([400, 400], 300, 300)):
        t = dev(torch.tensor(ptr))
        whole = [torch.full((offset + N * w + 64,), 7, dtype=torch.uint8, device="cuda:0") for w in (width, 2 * width)]
        at = (ctypes.c_void_p * 2)(*(x.data_ptr() + offset for x in whole))
        s._check(lib.als_clear_unheld(N, len(ptr) - 1, t.data_ptr(), 2, at, (ctypes.c_int64 * 2)(width, 2 * width),
                                      s._stream(0)))
        for x, w in zip(whole, (width, 2 * width)):
            want = torch.full_like(x, 7)
            want[offset:offset + N * w].view(N, w)[:first] = 0
            want[offset:offset + N * w].view(N, w)[end:] = 0
            assert torch.equal(x, want), (ptr, w)

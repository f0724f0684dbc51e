"""The sequence operators against their definitions in 64 bits: values, gradients (the formulas' and
differences), rows of length zero and one, odd widths, strides, shared heads, masks that leave
nothing, infinities and NaN in masked places, indexes out of range, streams and graphs.

Bounds. u = 2^-8 is bf16's unit roundoff (8 bits), e = 2^-24 fp32's. A sum of n terms in fp32 is off by at most
about n e times the sum of the terms' sizes, which the reference computes beside each value (`size`,
the same formula over absolute values). bf16 outputs are rounded once (u times the value) and their
terms once (u times the size). What takes an exponential of x = log_decay * tokens is off by another
(2 + |x|) e, and |x| e^-|x| < 1, so each factor adds at most 4 e; a state meets one per chunk.
"""
import math
import sys

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U, E = 2.0 ** -8, 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def log(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def dev(t):
    return None if t is None else t.to("cuda:0")


def within(got, want, bound, what):
    """Elementwise |got - want| <= bound; the same infinities and NaN."""
    got = got.double().cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    plain = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), plain), f"{what}: other places are finite"
    off = (got - want).abs()[plain]
    ratio = float((off / bound.expand_as(want)[plain].clamp(min=1e-300)).max()) if off.numel() else 0.0
    log(f"  {what}: {ratio:.3f} of the bound")
    assert ratio <= 1.0, what


def out_bound(dtype, value, size, terms):
    rounding = U * (value.abs() + 1.01 * size) if dtype == torch.bfloat16 else E * value.abs()
    return rounding + terms * E * size + 1e-30


# ---- norm and rotation ---------------------------------------------------------------------------

def rotate_reference(x, w, cos, sin, pos, eps, neighbours, dy=None):
    """y, or (dx, dweight) given dy, with the sizes of their sums, in fp64 on the CPU."""
    x, w, cos, sin = (t.double().cpu() for t in (x, w, cos, sin))
    R = 2 * cos.shape[1]
    pair = torch.arange(R).view(2, -1) if not neighbours else torch.arange(R).view(-1, 2).t()
    ok = (pos.cpu() >= 0) & (pos.cpu() < cos.shape[0])
    at = torch.where(ok, pos.cpu(), 0).long()
    z = torch.complex(cos[at], sin[at])[:, None]

    def turn(y, z):
        y = y.clone()
        p = torch.complex(y[..., pair[0]], y[..., pair[1]]) * z
        y[..., pair[0]], y[..., pair[1]] = p.real, p.imag
        return y

    r = 1.0 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    nan = torch.where(ok, 1.0, math.nan)[:, None, None].double()
    if dy is None:
        y = x * r * w
        size = y.abs().clone()
        a, b, c, s = y[..., pair[0]].abs(), y[..., pair[1]].abs(), z.real.abs(), z.imag.abs()
        size[..., pair[0]], size[..., pair[1]] = a * c + b * s, b * c + a * s
        return turn(y, z) * nan, size
    g = turn(dy.double().cpu(), z.conj())
    gs = dy.double().cpu().abs().amax(-1, keepdim=True) * 2.0
    n = x * r
    dx = r * (g * w - n * (g * w * n).mean(-1, keepdim=True))
    size = r * gs * w.abs().amax() * (1.0 + n.abs() * n.abs().mean(-1, keepdim=True))
    return dx * nan, size, (g * n * nan).sum((0, 1)), (gs * n.abs()).sum((0, 1))


ROTATE = [  # tokens, heads, key heads, width, rotated, neighbours
    (1, 1, 1, 1, 0, False), (1, 2, 1, 2, 2, True), (3, 4, 2, 64, 64, False), (5, 8, 8, 64, 32, True),
    (130, 3, 1, 100, 100, False), (67, 5, 5, 33, 30, False), (67, 2, 1, 33, 32, True),
    (1000, 4, 4, 128, 128, False), (33, 2, 2, 256, 250, False), (20, 2, 2, 255, 254, True),
    (4099, 2, 1, 20, 8, False), (9, 1, 1, 20, 0, False),
    (40, 3, 2, 100, 60, True), (70, 2, 1, 42, 38, True), (90, 2, 2, 77, 40, False), (33, 1, 1, 12, 0, False),
    (50, 2, 2, 90, 90, True), (21, 4, 1, 9, 8, True)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,H,Hk,D,R,nb", ROTATE)
def test_norm_rotate_and_gradients(N, H, Hk, D, R, nb, dtype):
    import paper_1108_2580_amd as p

    dt = DTYPES[dtype]
    g = torch.Generator().manual_seed(N + D)
    both = torch.randn(N, H + Hk, D + 8, generator=g).to(dt)
    both[0, 0] = 0  # a row of zeros
    q, k = dev(both)[:, :H, :D], dev(both)[:, H:, :D]  # strided views
    wq, wk = (dev(1 + 0.2 * torch.randn(D, generator=g)) for _ in range(2))
    P = 50
    cos, sin = p.rotary_tables(P, R)
    pos = dev(torch.randint(0, P, (N,), generator=g, dtype=torch.int32))
    log(f"{N} tokens, {H}/{Hk} heads, width {D}, {R} rotated, neighbours {nb}, {dtype}")
    outs = p.norm_rotate(q, k, wq, wk, cos, sin, pos, 1e-5, nb)
    for x, w, y, name in ((q, wq, outs[0], "q"), (k, wk, outs[1], "k")):
        want, size = rotate_reference(x, w, cos, sin, pos, 1e-5, nb)
        # the norm sums width squares; then three products and one sum
        within(y, want, (U if dt == torch.bfloat16 else E) * want.abs() + (D + 12) * E * size + 1e-30, name)
    dq, dk = (dev(torch.randn(t.shape, generator=g).to(dt)) for t in (q, k))
    grads = p.norm_rotate_backward(dq, dk, q, k, wq, wk, cos, sin, pos, 1e-5, nb)
    for x, w, dy, dx, dw, name in ((q, wq, dq, grads[0], grads[2], "dq"), (k, wk, dk, grads[1], grads[3], "dk")):
        want, size, want_w, size_w = rotate_reference(x, w, cos, sin, pos, 1e-5, nb, dy)
        within(dx, want, (U if dt == torch.bfloat16 else E) * want.abs() + (2 * D + 24) * E * size + 1e-30, name)
        # a lane, a block and the blocks' sum: no chain is longer than the rows; 12 products before it
        within(dw, want_w, (N + D + 24) * E * size_w + 1e-30, name + " weight")


@pytest.mark.parametrize("nb", [False, True])
def test_norm_rotate_gradient_by_differences(nb):
    import paper_1108_2580_amd as p

    g = torch.Generator().manual_seed(5)
    q, k = torch.randn(7, 3, 24, generator=g), torch.randn(7, 2, 24, generator=g)
    wq, wk = (1 + 0.2 * torch.randn(24, generator=g) for _ in range(2))
    cos, sin = p.rotary_tables(11, 20)
    pos = torch.randint(0, 11, (7,), generator=g, dtype=torch.int32)
    dq, dk = torch.randn(q.shape, generator=g), torch.randn(k.shape, generator=g)
    args = [dev(t).requires_grad_() for t in (q, k, wq, wk)]
    a, b = p.norm_rotate(*args, cos, sin, dev(pos), 1e-6, nb)
    grads = torch.autograd.grad([a, b], args, [dev(dq), dev(dk)])

    def loss(q, k, wq, wk):
        y, _ = rotate_reference(q, wq, cos, sin, pos, 1e-6, nb)
        z, _ = rotate_reference(k, wk, cos, sin, pos, 1e-6, nb)
        return float((y * dq).sum() + (z * dk).sum())

    at = [t.double() for t in (q, k, wq, wk)]
    for i, grad in enumerate(grads):
        d = torch.randn(at[i].shape, generator=g).double()
        move = lambda h: [t + h * d if j == i else t for j, t in enumerate(at)]  # noqa: E731
        h = 1e-5
        want = (loss(*move(h)) - loss(*move(-h))) / (2 * h)
        got = float((grad.double().cpu() * d).sum())
        # fp32 gradients of about 500 values of size 1 to 3; the difference itself is good to h^2
        assert abs(got - want) <= 1e-5 * float((grad.double().cpu().abs() * d.abs()).sum()), (i, got, want)


def test_norm_rotate_position_outside_the_tables_is_nan():
    import paper_1108_2580_amd as p

    q = torch.randn(4, 2, 16, device="cuda:0")
    w = torch.ones(16, device="cuda:0")
    cos, sin = p.rotary_tables(10, 16)
    pos = torch.tensor([3, -1, 10, 9], dtype=torch.int32, device="cuda:0")
    y, z = p.norm_rotate(q, q.clone(), w, w, cos, sin, pos)
    for t in (y, z):
        assert torch.isnan(t[1:3]).all() and torch.isfinite(t[[0, 3]]).all()


def test_norm_rotate_without_tokens():
    import paper_1108_2580_amd as p

    q = torch.empty(0, 2, 16, device="cuda:0")
    w = torch.ones(16, device="cuda:0")
    cos, sin = p.rotary_tables(10, 16)
    pos = torch.empty(0, dtype=torch.int32, device="cuda:0")
    y, _ = p.norm_rotate(q, q, w, w, cos, sin, pos)
    assert y.shape == q.shape
    *_, dw, dv = p.norm_rotate_backward(q, q, q, q, w, w, cos, sin, pos)
    assert (dw == 0).all() and (dv == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nb,D,R", [(False, 37, 30), (True, 37, 30), (False, 44, 22), (True, 44, 26)])
def test_norm_rotate_in_place(nb, D, R, dtype):
    """Through the C entries, outputs that are the inputs themselves (views of one projection)."""
    import ctypes

    import paper_1108_2580_amd as p
    from paper_1108_2580_amd import sequence as s

    N, H, Hk = 50, 3, 2
    both = torch.randn(N, H + Hk, D, device="cuda:0").to(DTYPES[dtype])
    w = torch.rand(D, device="cuda:0") + 0.5
    cos, sin = p.rotary_tables(9, R)
    pos = torch.arange(N, dtype=torch.int32, device="cuda:0") % 9
    args = (w, w, cos, sin, pos, 1e-6, nb)
    want = p.norm_rotate(both[:, :H], both[:, H:], *args)
    dy = torch.randn_like(both)
    grads = p.norm_rotate_backward(dy[:, :H], dy[:, H:], both[:, :H], both[:, H:], *args)
    shape = s._Rotation(N, 9, H, Hk, D, R, int(nb), 1e-6, pos.data_ptr(), cos.data_ptr(), sin.data_ptr())
    heads = lambda t, h: s._Heads(t.data_ptr() + h * D * t.element_size(), (H + Hk) * D, D)  # noqa: E731
    x, code = both.clone(), s._DTYPES[both.dtype]
    assert p.lib.als_norm_rotate(shape, code, heads(x, 0), heads(x, H), w.data_ptr(), w.data_ptr(), heads(x, 0),
                                 heads(x, H), s._stream(0)) == 0
    assert torch.equal(x[:, :H], want[0]) and torch.equal(x[:, H:], want[1])
    dw = torch.empty(2, D, device="cuda:0")
    size = p.lib.als_norm_rotate_workspace(shape)
    work = torch.empty(size, dtype=torch.uint8, device="cuda:0")
    for into in (dy.clone(), both.clone()):  # over the outputs' gradients, and over the inputs
        a, b = (into, both) if torch.equal(into, dy) else (dy, into)
        assert p.lib.als_norm_rotate_backward(
            shape, code, heads(a, 0), heads(a, H), heads(b, 0), heads(b, H), w.data_ptr(), w.data_ptr(),
            heads(into, 0), heads(into, H), dw[0].data_ptr(), dw[1].data_ptr(), work.data_ptr(), size,
            ctypes.c_void_p(s._stream(0))) == 0
        assert torch.equal(into[:, :H], grads[0]) and torch.equal(into[:, H:], grads[1])
        assert torch.equal(dw[0], grads[2]) and torch.equal(dw[1], grads[3])


# ---- attention -----------------------------------------------------------------------------------

def attention_reference(q, k, v, a, lens, scale, S0=None, d_out=None, dS=None):
    """Token by token in fp64 on the CPU: o and the last states; with d_out also dq, dk, dv, dS0."""
    q, k, v = (t.double().cpu() for t in (q, k, v))
    H, group = q.shape[1], q.shape[1] // k.shape[1]
    K, V = q.shape[2], v.shape[2]
    k, v = (t.repeat_interleave(group, 1) for t in (k, v))
    decay = torch.exp(a.double().cpu())[:, None, None]
    o = torch.zeros(q.shape[0], H, V, dtype=torch.float64)
    last = torch.zeros(len(lens), H, K, V, dtype=torch.float64)
    if d_out is not None:
        d_out = d_out.double().cpu()
        dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
        dfirst = torch.zeros_like(last)
    t0 = 0
    for b, n in enumerate(lens):
        S = torch.zeros(H, K, V, dtype=torch.float64) if S0 is None else S0[b].double().cpu()
        for t in range(t0, t0 + n):
            S = decay * S + k[t][:, :, None] * v[t][:, None]
            o[t] = scale * (q[t][:, :, None] * S).sum(1)
            if d_out is not None:
                dq[t] = scale * (S * d_out[t][:, None]).sum(2)
        last[b] = S
        if d_out is not None:
            X = torch.zeros(H, K, V, dtype=torch.float64) if dS is None else dS[b].double().cpu()
            for t in range(t0 + n - 1, t0 - 1, -1):
                X = X + scale * q[t][:, :, None] * d_out[t][:, None]
                dk[t], dv[t] = (X * v[t][:, None]).sum(2), (X * k[t][:, :, None]).sum(1)
                X = decay * X
            dfirst[b] = X
        t0 += n
    if d_out is None:
        return o, last
    shared = lambda x: x.unflatten(1, (-1, group)).sum(2)  # noqa: E731
    return o, last, dq, shared(dk), shared(dv), dfirst


def attention_inputs(lens, H, Hk, K, V, dtype, seed, strided=True):
    g = torch.Generator().manual_seed(seed)
    N, pad = sum(lens), 8 if strided else 0
    dt = DTYPES[dtype]
    # one projection's rows [q heads | k heads | v heads], with a tail that is not used
    row = torch.randn(N, H * K + Hk * (K + V) + pad, generator=g).to(dt)
    q = dev(row)[:, :H * K].unflatten(1, (H, K))
    k = dev(row)[:, H * K:(H + Hk) * K].unflatten(1, (Hk, K))
    v = dev(row)[:, (H + Hk) * K:(H + Hk) * K + Hk * V].unflatten(1, (Hk, V))
    # windows from one token to none forgotten
    a = torch.tensor([-math.inf, -0.7, -0.02, 0.0, -0.1, -3.0, -0.005, -0.3])[torch.arange(H) % 8]
    if H == 1:
        a = torch.tensor([-0.05])
    ptr = torch.tensor([0] + lens).cumsum(0)
    d_out = dev(torch.randn(N, H, V, generator=g).to(dt))
    S0, dS = (dev(torch.randn(len(lens), H, K, V, generator=g)) for _ in range(2))
    return q, k, v, dev(a), dev(ptr), d_out, S0, dS


ATTENTION = [  # lengths, heads, key heads, key width, value width
    ([1], 1, 1, 1, 1), ([0], 2, 2, 4, 4), ([0, 1, 0, 2, 0], 2, 1, 8, 16), ([63, 64, 65], 4, 4, 64, 64),
    ([31, 32, 33, 1, 128], 4, 2, 32, 32), ([200, 0, 7], 3, 3, 33, 50), ([129], 8, 2, 100, 128),
    ([300], 8, 8, 16, 65), ([96, 97], 6, 1, 128, 20), ([5] * 70, 2, 2, 24, 24)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("resumed", [False, True])
@pytest.mark.parametrize("lens,H,Hk,K,V", ATTENTION)
def test_attention_and_gradients(lens, H, Hk, K, V, resumed, dtype):
    import paper_1108_2580_amd as p

    q, k, v, a, ptr, d_out, S0, dS = attention_inputs(lens, H, Hk, K, V, dtype, len(lens) + K)
    if not resumed:
        S0 = dS = None
    scale = 0.37
    log(f"lengths {lens[:6]}, {H}/{Hk} heads, {K} x {V}, resumed {resumed}, {dtype}")
    want = attention_reference(q, k, v, a, lens, scale, S0, d_out, dS)
    mag = lambda t: None if t is None else t.abs()  # noqa: E731
    size = attention_reference(mag(q), mag(k), mag(v), a, lens, scale, mag(S0), mag(d_out), mag(dS))
    terms = (max(lens) if lens else 0) + K + V + 40
    o, S = p.decay_attention(q, k, v, a, ptr, scale, S0, return_state=True)
    dt = DTYPES[dtype]
    within(o, want[0], out_bound(dt, want[0], size[0], terms), "out")
    within(S, want[1], terms * E * size[1] + 1e-30, "state")
    dq, dk, dv, d0 = p.decay_attention_backward(d_out, q, k, v, a, ptr, scale, S0, dS, d_initial=True)
    within(dq, want[2], out_bound(dt, want[2], size[2], terms), "dq")
    within(dk, want[3], out_bound(dt, want[3], size[3], terms + 8), "dk")
    within(dv, want[4], out_bound(dt, want[4], size[4], terms + 8), "dv")
    within(d0, want[5], terms * E * size[5] + 1e-30, "initial state's gradient")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,H,Hk,K,V", [([5000], 1, 1, 16, 16), ([513, 2, 0, 1700, 512], 2, 1, 33, 40)])
def test_attention_cut_into_segments(lens, H, Hk, K, V, dtype):
    """Rows longer than a segment."""
    test_attention_and_gradients(lens, H, Hk, K, V, True, dtype)


def test_attention_reproducible_and_on_any_stream():
    import paper_1108_2580_amd as p

    q, k, v, a, ptr, d_out, S0, dS = attention_inputs([700, 0, 3000], 4, 2, 64, 64, "bf16", 3)
    args = (q, k, v, a, ptr, None, S0)
    first = [*p.decay_attention(*args, return_state=True),
             *p.decay_attention_backward(d_out, *args, dS)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = [*p.decay_attention(*args, return_state=True),
                 *p.decay_attention_backward(d_out, *args, dS)]
    torch.cuda.current_stream().wait_stream(side)
    for x, y in zip(first, again):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_token_takes_nothing_from_later_ones(dtype):
    """Infinities and NaN in a token reach the tokens after it in its row, and no other."""
    import paper_1108_2580_amd as p

    lens = [40, 90, 30]
    q, k, v, a, ptr, *_ = attention_inputs(lens, 4, 4, 32, 48, dtype, 9)
    a = torch.full_like(a, -0.1)
    clean = p.decay_attention(q, k, v, a, ptr)
    for bad in (math.nan, math.inf):
        for at, which in ((50, v), (70, k)):
            q2, k2, v2 = q.clone(), k.clone(), v.clone()
            (v2 if which is v else k2)[at] = bad
            o = p.decay_attention(q2, k2, v2, a, ptr)
            assert torch.equal(o[:at], clean[:at]), (bad, at)
            assert torch.equal(o[130:], clean[130:]), (bad, at)
            assert not torch.isfinite(o[at]).any()
    q2 = q.clone()
    q2[60] = math.nan  # a query reaches its own token alone
    o = p.decay_attention(q2, k, v, a, ptr)
    rest = torch.arange(160, device=o.device) != 60
    assert torch.equal(o[rest], clean[rest]) and torch.isnan(o[60]).all()


def test_attention_decay_above_one_is_nan():
    import paper_1108_2580_amd as p

    q, k, v, a, ptr, *_ = attention_inputs([20], 2, 2, 16, 16, "f32", 1)
    a = torch.tensor([0.1, -0.1], device="cuda:0")
    o = p.decay_attention(q, k, v, a, ptr)
    assert torch.isnan(o[:, 0]).all() and torch.isfinite(o[:, 1]).all()


def test_attention_row_ptr_out_of_range_stays_inside():
    """Values outside [0, tokens] are taken as the nearest bound: the rows that remain are right."""
    import paper_1108_2580_amd as p

    q, k, v, a, ptr, *_ = attention_inputs([30, 40], 2, 2, 16, 16, "f32", 2)
    want = p.decay_attention(q, k, v, a, ptr)
    wild = torch.tensor([-5, 30, 1 << 40], device="cuda:0")
    assert torch.equal(p.decay_attention(q, k, v, a, wild), want)


def test_attention_gradient_by_differences():
    import paper_1108_2580_amd as p

    lens = [9, 0, 40]
    q, k, v, a, ptr, d_out, S0, dS = attention_inputs(lens, 4, 2, 8, 12, "f32", 4)
    args = [t.clone().requires_grad_() for t in (q, k, v, S0)]
    o, S = p.decay_attention(*args[:3], a, ptr, 0.5, args[3], return_state=True)
    grads = torch.autograd.grad([o, S], args, [d_out, dS])

    def loss(q, k, v, S0):
        o, S = attention_reference(q, k, v, a, lens, 0.5, S0)
        return float((o * d_out.double().cpu()).sum() + (S * dS.double().cpu()).sum())

    g = torch.Generator().manual_seed(8)
    at = [t.double().cpu() for t in (q, k, v, S0)]
    for i, grad in enumerate(grads):
        d = torch.randn(at[i].shape, generator=g).double()
        move = lambda h: [t + h * d if j == i else t for j, t in enumerate(at)]  # noqa: E731
        h = 1e-4
        want = (loss(*move(h)) - loss(*move(-h))) / (2 * h)
        got = float((grad.double().cpu() * d).sum())
        assert abs(got - want) <= 1e-5 * float((grad.double().cpu().abs() * d.abs()).sum()), (i, got, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,H,Hk,K,V", [(1, 1, 1, 1, 1), (3, 2, 1, 64, 64), (5, 4, 4, 33, 50),
                                        (2, 8, 2, 128, 128), (70, 3, 3, 7, 125), (9, 2, 2, 100, 4)])
def test_step_continues_a_history(N, H, Hk, K, V, dtype):
    """A step's output and state; with source, states of other rows; in place."""
    import paper_1108_2580_amd as p

    q, k, v, a, ptr, _, S0, _ = attention_inputs([1] * N, H, Hk, K, V, dtype, N + V)
    want, last = attention_reference(q, k, v, a, [1] * N, 0.5, S0)
    size, size_s = attention_reference(q.abs(), k.abs(), v.abs(), a, [1] * N, 0.5, S0.abs())
    dt = DTYPES[dtype]
    held = S0.clone()
    o, S = p.decay_attention_step(q, k, v, a, held, 0.5)
    assert S is held
    within(o, want, (U if dt == torch.bfloat16 else E) * want.abs() + (K + 12) * E * size + 1e-30, "out")
    within(S, last, 12 * E * size_s + 1e-30, "state")
    # states by source: rows 0, 0, 1, ... of a larger table, and one that does not exist
    table = torch.randn(N + 2, H, K, V, device="cuda:0")
    source = torch.tensor([(3 * i) % (N + 2) for i in range(N)], dtype=torch.int32, device="cuda:0")
    o1, S1 = p.decay_attention_step(q, k, v, a, table, 0.5, source)
    o2, S2 = p.decay_attention_step(q, k, v, a, table[source.long()].contiguous(), 0.5)
    assert torch.equal(o1, o2) and torch.equal(S1, S2)
    for bad in (-1, N + 2):
        source[0] = bad
        o3, S3 = p.decay_attention_step(q, k, v, a, table, 0.5, source)
        assert torch.isnan(o3[0]).all() and torch.isnan(S3[0]).all()
        assert torch.equal(o3[1:], o1[1:]) and torch.equal(S3[1:], S1[1:])


def test_step_and_history_agree():
    """Single tokens one after the other give the states and outputs of the whole history."""
    import paper_1108_2580_amd as p

    q, k, v, a, ptr, *_ = attention_inputs([70], 4, 2, 32, 32, "f32", 6)
    o, S = p.decay_attention(q, k, v, a, ptr, return_state=True)
    state = torch.zeros_like(S)
    steps = [p.decay_attention_step(q[t:t + 1], k[t:t + 1], v[t:t + 1], a, state)[0] for t in range(70)]
    size, size_s = attention_reference(q.abs(), k.abs(), v.abs(), a, [70], 32 ** -0.5)
    within(torch.cat(steps), o.double().cpu(), 2 * (70 + 32 + 40) * E * size + 1e-30, "outputs")
    within(state, S.double().cpu(), 2 * 110 * E * size_s + 1e-30, "state")


# ---- beams ---------------------------------------------------------------------------------------

def beam_reference(logits, scores, finished, end, width):
    """Candidates in Python's order: descending score, then the lowest beam and item."""
    B, W, V = logits.shape
    x = torch.nan_to_num(logits.double().cpu(), nan=-math.inf, posinf=torch.finfo(torch.float32).max,
                         neginf=-math.inf)
    out = []
    for b in range(B):
        cand = []
        for w in range(W):
            c = float(scores[b, w])
            if not c > -math.inf:
                continue
            if finished is not None and bool(finished[b, w]):
                cand.append((-c, w, end))
                continue
            row = x[b, w]
            m = float(row.max())
            if m == -math.inf:
                continue
            s = (row - m) + (c - math.log(float(torch.exp(row - m).sum())))
            for t in torch.sort(s, descending=True, stable=True).indices[:width].tolist():
                if row[t] > -math.inf:
                    cand.append((-float(s[t]), w, t))
        cand = sorted(cand)[:width]
        fill = [(math.inf, 0, -1)] * (width - len(cand))
        out.append(cand + fill)
    tab = torch.tensor([[(-s, w, t) for s, w, t in row] for row in out], dtype=torch.float64)
    parents, tokens = tab[..., 1].int(), tab[..., 2].int()
    done = tokens == end if end >= 0 else torch.zeros_like(tokens, dtype=torch.bool)
    if finished is not None:
        done = done | (finished.cpu().bool().gather(1, parents.long()) & (tokens >= 0))
    return parents, tokens, tab[..., 0], done


BEAMS = [  # lists, beams, width, items
    (1, 1, 1, 1), (1, 1, 4, 3), (2, 3, 3, 2), (1, 4, 4, 1000), (3, 5, 5, 8192), (2, 8, 8, 8193),
    (2, 1, 32, 20001), (1, 32, 32, 9001), (2, 4, 7, 16391), (1, 2, 3, 100003)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,W,width,V", BEAMS)
def test_beam_select(B, W, width, V, dtype):
    import paper_1108_2580_amd as p

    g = torch.Generator().manual_seed(V + W)
    logits = (torch.randn(B, W, V, generator=g) * 3).to(DTYPES[dtype])
    scores = -torch.rand(B, W, generator=g) * 3
    finished = torch.rand(B, W, generator=g) < 0.3
    for done, end in ((None, -1), (None, V // 2), (finished, V - 1)):
        want = beam_reference(logits, scores, done, end, width)
        got = p.beam_select(dev(logits), dev(scores), dev(done), end, width)
        log(f"{B} lists, {W} -> {width} beams, {V} items, {dtype}, end {end}")
        for i in (0, 1, 3):
            assert torch.equal(got[i].cpu(), want[i]), i
        # rounded once from fp64; the sum of exponentials is fp32 in slices: 8192 terms of 2 ulp each
        # whose errors enter as a share of the sum, hence 40 e at the most for the sum's 32-term chains
        within(got[2], want[2], 2 * E * want[2].abs() + 100 * E, "scores")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_beam_select_equal_scores_go_by_place(dtype):
    """All items equal; equal beams; few levels."""
    import paper_1108_2580_amd as p

    for V in (5, 700, 20000):
        flat = torch.zeros(1, 4, V, dtype=DTYPES[dtype], device="cuda:0")
        par, tok, s, _ = p.beam_select(flat, torch.zeros(1, 4, device="cuda:0"), width=7)
        want = [divmod(i, V) for i in range(7)]
        assert list(zip(par[0].tolist(), tok[0].tolist())) == want
        g = torch.Generator().manual_seed(V)
        levels = torch.randint(-2, 3, (2, 3, V), generator=g).to(DTYPES[dtype])
        levels[:, 1] = levels[:, 0]
        scores = torch.tensor([[-1.0, -1.0, -2.0]] * 2)
        want = beam_reference(levels, scores, None, -1, 9)
        got = p.beam_select(dev(levels), dev(scores), width=9)
        assert torch.equal(got[0].cpu(), want[0]) and torch.equal(got[1].cpu(), want[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_beam_select_masks(dtype):
    """Rows that a mask leaves empty or nearly so, the type's lowest value as a mask, NaN, +inf, dead
    beams."""
    import paper_1108_2580_amd as p

    dt, V = DTYPES[dtype], 3000
    low = torch.finfo(dt).min
    g = torch.Generator().manual_seed(1)
    logits = torch.randn(6, 3, V, generator=g).to(dt)
    logits[0] = -math.inf                      # nothing left
    logits[1] = -math.inf
    logits[1, 2, 17] = 0.5                     # one item
    logits[2] = low                            # the lowest value is a value: all equal
    logits[3, :, 100:] = math.nan              # NaN masks
    logits[4, 1, 7] = math.inf                 # counts as the largest
    scores = -torch.rand(6, 3, generator=g)
    scores[5, 0], scores[5, 1] = -math.inf, math.nan
    want = beam_reference(logits, scores, None, -1, 4)
    got = p.beam_select(dev(logits), dev(scores), width=4)
    assert torch.equal(got[0].cpu(), want[0]) and torch.equal(got[1].cpu(), want[1])
    none = got[1].cpu() < 0
    assert none.sum() == 4 + 3 and (got[2].cpu()[none] == -math.inf).all()
    both = ~none & (want[2] > -1e30)
    assert ((got[2].double().cpu() - want[2]).abs()[both] <= 1e-5).all()


def test_beam_select_strided_rows_and_first_step():
    import paper_1108_2580_amd as p

    g = torch.Generator().manual_seed(2)
    wide = torch.randn(6, 1011, generator=g)
    logits = dev(wide)[:, 3:1000].unflatten(0, (2, 3))  # rows 1011 apart, not 16-byte aligned
    scores = -torch.rand(2, 3, generator=g)
    want = beam_reference(wide[:, 3:1000].unflatten(0, (2, 3)), scores, None, -1, 3)
    got = p.beam_select(logits, dev(scores))
    assert torch.equal(got[0].cpu(), want[0]) and torch.equal(got[1].cpu(), want[1])


@pytest.mark.parametrize("shape,dt", [((2, 3, 64), torch.float32), ((3, 8, 5, 7), torch.bfloat16),
                                      ((1, 1, 1), torch.uint8), ((2, 32, 1030), torch.float32),
                                      ((2, 5, 3, 2), torch.int64), ((4, 16, 33), torch.bfloat16)])
def test_reorder_states(shape, dt):
    import paper_1108_2580_amd as p

    g = torch.Generator().manual_seed(sum(shape))
    x = torch.randint(0, 100, shape, generator=g).to(dt)
    B, W = shape[:2]
    for width in (W, max(1, W // 2), min(32, W + 3)):
        parents = torch.randint(0, W, (B, width), generator=g, dtype=torch.int32)
        want = torch.stack([x[b][parents[b].long()] for b in range(B)])
        got = p.reorder_states(dev(x), dev(parents))
        assert torch.equal(got.cpu(), want)
        if width == W:
            held = dev(x).clone()
            assert p.reorder_states(held, dev(parents), out=held) is held
            assert torch.equal(held.cpu(), want)
            parents[0, 0] = -1  # leaves its row
            want[0, 0] = x[0, 0]
            held = dev(x).clone()
            p.reorder_states(held, dev(parents), out=held)
            assert torch.equal(held.cpu(), want)


def test_no_lists_no_rows():
    import paper_1108_2580_amd as p

    z = lambda *s, dtype=torch.float32: torch.empty(s, dtype=dtype, device="cuda:0")  # noqa: E731
    got = p.beam_select(z(0, 2, 10), z(0, 2))
    assert all(t.shape == (0, 2) for t in got)
    assert p.reorder_states(z(0, 2, 4), z(0, 2, dtype=torch.int32)).shape == (0, 2, 4)
    o, S = p.decay_attention(z(0, 2, 8), z(0, 2, 8), z(0, 2, 8), z(2), z(1, dtype=torch.int64).zero_(),
                             return_state=True)
    assert o.shape == (0, 2, 8) and S.shape == (0, 2, 8, 8)
    o, S = p.decay_attention_step(z(0, 2, 8), z(0, 2, 8), z(0, 2, 8), z(2), z(0, 2, 8, 8))
    assert o.shape == (0, 2, 8)


def test_calls_replay_in_a_graph():
    """A serving step captured once: every replay on new inputs equals the eager calls."""
    import paper_1108_2580_amd as p

    B, W, H, D, V = 2, 4, 2, 32, 5000
    g = torch.Generator(device="cuda:0").manual_seed(3)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda:0")  # noqa: E731
    q, k, v, logits = rnd(B * W, H, D), rnd(B * W, H, D), rnd(B * W, H, D), rnd(B, W, V)
    state, scores = rnd(B * W, H, D, D), -rnd(B, W).abs()
    a = torch.tensor([-0.1, -0.01], device="cuda:0")
    w = torch.ones(D, device="cuda:0")
    cos, sin = p.rotary_tables(20, D)
    pos = torch.arange(B * W, dtype=torch.int32, device="cuda:0")
    rows = torch.arange(B, dtype=torch.int32, device="cuda:0")[:, None] * W

    def token():
        q1, k1 = p.norm_rotate(q, k, w, w, cos, sin, pos)
        parents, tokens, new, done = p.beam_select(logits, scores)
        o, S = p.decay_attention_step(q1, k1, v, a, state, source=(parents + rows).flatten())
        return parents, tokens, new, o, S, p.reorder_states(state.view(B, W, -1), parents)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        token()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = token()
    for _ in range(4):
        for t in (q, k, v, logits, state):
            t.copy_(rnd(*t.shape))
        want = [t.clone() for t in token()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(held, want):
            assert torch.equal(x, y)


@pytest.mark.parametrize("wanted", ["out", "state", "both"])
def test_autograd_of_a_training_step(wanted):
    """norm_rotate and decay_attention in a graph of torch's, from keys that all rows share, with the
    loss on the outputs, the states, or both: what the operators' own backward calls give."""
    import paper_1108_2580_amd as p

    lens, H, Hk, K, V = [40, 0, 71], 4, 2, 32, 24
    q, k, v, a, ptr, d_out, S0, dS = attention_inputs(lens, H, Hk, K, V, "f32", 11)
    N = sum(lens)
    w = torch.ones(K, device="cuda:0")
    cos, sin = p.rotary_tables(N, K)
    pos = torch.arange(N, dtype=torch.int32, device="cuda:0")
    one = k[:1].clone().requires_grad_()  # broadcast over the tokens
    q, v = q.clone().requires_grad_(), v.clone().requires_grad_()
    keys = one.expand(N, Hk, K)
    q1, k1 = p.norm_rotate(q, keys, w, w, cos, sin, pos)
    got = p.decay_attention(q1, k1, v, a, ptr, return_state=wanted != "out")
    out, state = got if wanted != "out" else (got, None)
    loss = 0.0
    if wanted != "state":
        loss = loss + (out * d_out).sum()
    if wanted != "out":
        loss = loss + (state * dS).sum()
    grads = torch.autograd.grad(loss, (q, one, v))
    with torch.no_grad():
        dq1, dk1, dv, _ = p.decay_attention_backward(
            d_out if wanted != "state" else torch.zeros_like(d_out), q1, k1, v, a, ptr,
            dstate=dS if wanted != "out" else None)
        dq, dk, _, _ = p.norm_rotate_backward(dq1, dk1, q, keys, w, w, cos, sin, pos)
    assert torch.equal(grads[0], dq) and torch.equal(grads[2], dv)
    # a sum over the tokens in some other order
    bound = N * 2.0 ** -24 * dk.abs().sum(0, keepdim=True) + 1e-30
    assert ((grads[1] - dk.sum(0, keepdim=True)).abs() <= 2 * bound).all()

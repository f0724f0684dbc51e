"""Attention over gaps of time against its definition in 64 bits: values, gradients (the formulas' and
differences), single tokens of beams; rows of length zero and one, odd widths and strides, shared heads,
biases that mask rows or take the type's lowest value, infinities and NaN in masked places, indexes out of
range, long gaps, streams and graphs.

Bounds. U = 2^-8 is bf16's unit roundoff, E = 2^-24 fp32's. With S the largest size of a score (the sum of its
products' sizes and its bias), D the width and n the longest row:
- a score is off by (D + 16) E S (its sum of products of at most D terms, 2^-22 of fp32 products that parts
  leave out, which is 4 E S, the scale, the bias and their factors log2 e), so that a weight before its sum is
  off by that and 4 E (the exponential and the difference), and the weight by twice that and n E of itself;
- an output is off by the weights' error and n E (its sum) times the sum of its terms' sizes (`size`, the
  formula over absolute values), two bf16 parts of a weight by 2^-16 of it, and its own rounding;
- ds = p (do . v - do . o): with A = p (sum |do| |v| + sum |do| |o's size|), it is off by A times the weight's
  error, (D + 8) E for each product, the outputs' error (n E and twice the scores') and, in bf16, what rest
  leaves of them (2^-24);
- a gradient by that and n E (its sum) of the sum of its terms' sizes, 2^-16 for two parts, and its rounding.
"""
import math
import sys

import pytest

from .test_gpu_sequence import DTYPES, E, U, dev, log, within

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
LOWEST = torch.finfo(torch.float32).min


def inputs(lens, H, Hk, D, buckets, dtype, seed, last=2000, positions="ascending"):
    """q, k and v are views of one projection; positions ascend within rows over about 3 last bounds."""
    g = torch.Generator().manual_seed(seed)
    N = sum(lens)
    both = torch.randn(N, H + 2 * Hk, D, generator=g).to(DTYPES[dtype])
    both = dev(both)
    q, k, v = both[:, :H], both[:, H:H + Hk], both[:, H + Hk:]
    d_out = dev(torch.randn(N, H, D, generator=g).to(DTYPES[dtype]))
    bounds = torch.unique(torch.tensor([max(1, round(last ** (b / buckets))) for b in range(1, buckets)]
                                       + list(range(1, buckets)))).int()
    bounds = bounds[torch.linspace(0, bounds.numel() - 1, buckets - 1).long()] if buckets > 1 else \
        torch.zeros(0, dtype=torch.int32)
    bias = dev(0.7 * torch.randn(H, buckets, generator=g))
    rows = [torch.randint(0, 3 * last, (n,), generator=g) for n in lens]
    if positions == "ascending":
        rows = [r.sort().values for r in rows]
    pos = torch.cat(rows).int() if N else torch.zeros(0, dtype=torch.int32)
    ptr = torch.tensor([0] + lens).cumsum(0)
    return q, k, v, bias, bounds, dev(pos), dev(ptr), d_out


def kinds(bounds, at, of):
    gap = at.long()[:, None] - of.long()[None, :]
    return (gap[..., None] >= bounds.long()).sum(-1)


def softmax(x):
    """Over the last axis; zero where nothing is left, in the order of fp32's lowest value."""
    top = x.amax(-1, keepdim=True)
    w = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = w.sum(-1, keepdim=True)
    return torch.where(total == 0.0, 0.0, w / total)


def reference(q, k, v, bias, bounds, pos, ptr, scale, d_out=None):
    """dict of values and of the sizes of their sums (with "of_"), S and n, in fp64 on the CPU. Places that a
    mask leaves out are not looked at."""
    q, k, v, bias = (t.detach().double().cpu() for t in (q, k, v, bias))
    d_out = None if d_out is None else d_out.double().cpu()
    pos, ptr = pos.cpu(), ptr.cpu().tolist()
    N, H, D = q.shape
    group = H // k.shape[1]
    z = torch.zeros_like
    r = {"out": z(q), "of_out": z(q), "dq": z(q), "of_dq": z(q), "dk": z(k), "of_dk": z(k), "dv": z(v),
         "of_dv": z(v), "dbias": z(bias), "of_dbias": z(bias)}
    S, longest = 0.0, 0
    for a, b in zip(ptr, ptr[1:]):
        n = b - a
        longest = max(longest, n)
        if n == 0:
            continue
        kind = kinds(bounds, pos[a:b], pos[a:b])
        keep = torch.ones(n, n, dtype=torch.bool).tril()
        for h in range(H):
            Q, K, V = q[a:b, h], k[a:b, h // group], v[a:b, h // group]
            x = scale * (Q @ K.T) + bias[h][kind]
            x = torch.where(keep, x, -math.inf)
            live = keep & torch.isfinite(x)
            s = abs(scale) * (Q.abs() @ K.abs().T) + torch.nan_to_num(bias[h].abs(), nan=0.0, posinf=0.0)[kind]
            S = max(S, float(torch.where(live, s, 0.0).nan_to_num(0.0, 0.0, 0.0).amax()))
            w = softmax(x)
            mul = lambda p, y: torch.stack([p[i, :i + 1] @ y[:i + 1] for i in range(n)])  # noqa: E731
            o, so = mul(w, V), mul(w, V.abs())
            r["out"][a:b, h], r["of_out"][a:b, h] = o, so
            if d_out is None:
                continue
            G = d_out[a:b, h]
            ds = torch.where(keep, w * (G @ V.T - (G * o).sum(-1, keepdim=True)), 0.0)
            A = w * (G.abs() @ V.abs().T + (G.abs() * so).sum(-1, keepdim=True))
            r["dq"][a:b, h], r["of_dq"][a:b, h] = scale * ds @ K, abs(scale) * A @ K.abs()
            r["dk"][a:b, h // group] += scale * ds.T @ Q
            r["of_dk"][a:b, h // group] += abs(scale) * A.T @ Q.abs()
            r["dv"][a:b, h // group] += w.T @ G
            r["of_dv"][a:b, h // group] += w.T @ G.abs()
            r["dbias"][h].index_add_(0, kind.flatten(), ds.flatten())
            r["of_dbias"][h].index_add_(0, kind.flatten(), torch.where(keep, A, 0.0).flatten())
    r["S"], r["n"] = S, longest
    return r


def bounds_of(r, name, D, dtype, group=1):
    n, S, bf16 = r["n"], r["S"], dtype == "bf16"
    weight = 2 * ((D + 16) * S + 4) * E + n * E
    if name == "out":
        rel = weight + n * E + bf16 * 2.0 ** -16
    elif name == "dv":
        rel = weight + group * n * E + bf16 * 2.0 ** -16
    else:
        rel = 2 * weight + 2 * (D + 8) * E + (group + 1) * n * E + 64 * E + bf16 * 2.0 ** -15
    own = E if name == "dbias" or not bf16 else U
    return own * r[name].abs() + 1.05 * rel * r["of_" + name] + 1e-30


def check(r, got, D, dtype, group=1):
    for name, x in got.items():
        within(x, r[name], bounds_of(r, name, D, dtype, group), name)


def run(p, q, k, v, bias, bounds, pos, ptr, d_out, scale):
    args = (q, k, v, bias, bounds, pos, ptr, scale)
    out, saved = p.gap_attention(*args, return_saved=True)
    dq, dk, dv, dbias = p.gap_attention_backward(d_out, out, saved, *args)
    return {"out": out, "dq": dq, "dk": dk, "dv": dv, "dbias": dbias}


SHAPES = [  # lengths, heads, key heads, width, buckets, last bound
    ([1], 1, 1, 1, 1, 10), ([25], 4, 4, 32, 16, 2000), ([64], 1, 1, 64, 8, 50), ([65, 0, 1, 127], 2, 1, 64, 32, 2000),
    ([128, 129], 4, 2, 128, 64, 5000), ([3, 0, 0, 40, 1, 1, 90], 4, 2, 50, 7, 300), ([300], 2, 2, 33, 2, 100),
    ([2] * 80, 2, 1, 20, 16, 500), ([500, 17], 8, 2, 64, 32, 3000), ([200, 31, 32, 33], 3, 3, 100, 40, 900),
    ([10, 260], 1, 1, 7, 3, 40), ([700], 2, 1, 64, 32, 6000), ([5] * 70 + [150], 2, 2, 8, 5, 1000),
    ([400], 4, 1, 128, 16, 2000),
    # as many blocks as share columns of dbias's sums and go through a key head's query heads in turn
    ([300] * 30, 8, 8, 64, 32, 3000), ([100] * 170, 16, 8, 8, 4, 200), ([90] * 190, 16, 8, 64, 64, 4000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,H,Hk,D,buckets,last", SHAPES)
def test_values_and_gradients(lens, H, Hk, D, buckets, last, dtype):
    import paper_1108_2580_amd as p

    log(f"lengths {lens[:6]}, {H}/{Hk} heads, width {D}, {buckets} buckets to {last}, {dtype}")
    args = inputs(lens, H, Hk, D, buckets, dtype, sum(lens) + D, last)
    scale = D ** -0.5
    r = reference(*args[:7], scale, args[7])
    got = run(p, *args, scale)
    check(r, got, D, dtype, H // Hk)
    again = run(p, *args, scale)
    assert all(torch.equal(got[x], again[x]) for x in got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("last,positions", [(100_000, "ascending"), (2 ** 29, "ascending"), (3000, "any"),
                                            (100_000, "any")])
def test_long_gaps_and_positions_of_any_order(last, positions, dtype):
    """Bounds past the table of buckets; gaps below zero."""
    import paper_1108_2580_amd as p

    log(f"last bound {last}, positions {positions}, {dtype}")
    args = inputs([150, 80], 4, 2, 40, 24, dtype, 3, last, positions)
    check(reference(*args[:7], 0.2, args[7]), run(p, *args, 0.2), 40, dtype, 2)


def test_gaps_that_do_not_fit_32_bits():
    import paper_1108_2580_amd as p

    q, k, v, bias, _, pos, ptr, do = inputs([6], 1, 1, 16, 4, "f32", 4)
    bounds = torch.tensor([1, 5, 2 ** 31 - 1], dtype=torch.int32)
    pos = dev(torch.tensor([-2 ** 31, -2 ** 31, 2 ** 31 - 1, 2 ** 31 - 1, -2 ** 31, 0], dtype=torch.int32))
    check(reference(q, k, v, bias, bounds, pos, ptr, 0.3, do), run(p, q, k, v, bias, bounds, pos, ptr, do, 0.3),
          16, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [-0.2, 0.0, 3.0])
def test_scales(scale, dtype):
    import paper_1108_2580_amd as p

    args = inputs([200, 30], 2, 1, 48, 16, dtype, 9)
    log(f"scale {scale}, {dtype}")
    check(reference(*args[:7], scale, args[7]), run(p, *args, scale), 48, dtype, 2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,pad,start", [(64, 3, 0), (64, 8, 1), (50, 1, 1), (7, 2, 3), (128, 0, 0)])
def test_strides(D, pad, start, dtype):
    """Rows at any alignment of the type; heads apart from tokens."""
    import paper_1108_2580_amd as p

    q, k, v, bias, bounds, pos, ptr, do = inputs([130, 9], 4, 2, D, 12, dtype, 11)
    log(f"width {D}, padding {pad} from {start}, {dtype}")

    def moved(t, by_head):
        N, H, _ = t.shape
        flat = torch.full((N * H * (D + pad) + start,), math.nan, dtype=t.dtype, device=t.device)
        shape = (H, N) if by_head else (N, H)
        x = flat[start:].view(*shape, D + pad)[..., :D]
        x = x.transpose(0, 1) if by_head else x
        x.copy_(t)
        return x

    want = run(p, q, k, v, bias, bounds, pos, ptr, do, 0.2)
    for by_head in (False, True):
        got = run(p, *(moved(t, by_head) for t in (q, k, v)), bias, bounds, pos, ptr, moved(do, by_head), 0.2)
        assert all(torch.equal(got[x], want[x]) for x in got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masked_buckets(dtype):
    """Biases of -inf: buckets that are not read, and tokens left without a key."""
    import paper_1108_2580_amd as p

    q, k, v, bias, bounds, pos, ptr, do = inputs([140, 20], 4, 4, 64, 8, dtype, 21)
    bias[0, :] = -math.inf
    bias[1, 0] = -math.inf  # a token's own gap: the first has no key
    bias[2, 3:] = -math.inf
    r = reference(q, k, v, bias, bounds, pos, ptr, 0.2, do)
    got = run(p, q, k, v, bias, bounds, pos, ptr, do, 0.2)
    assert not got["out"][:, 0].any() and not got["dbias"][0].any()
    check(r, got, 64, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_lowest_biases(dtype):
    """The lowest value as a mask: it takes any score in, so that rows that have nothing else weigh all keys
    alike, and rows that have something else give such places nothing."""
    import paper_1108_2580_amd as p

    q, k, v, bias, bounds, pos, ptr, do = inputs([140, 20], 2, 2, 64, 8, dtype, 22)
    q[3] *= 40.0  # scores of some hundreds
    bias[0, :] = LOWEST
    bias[1, 2:] = LOWEST
    got = run(p, q, k, v, bias, bounds, pos, ptr, do, 1.0)
    even = torch.zeros_like(bias)
    zero = q.clone()
    zero[:, 0] = 0  # all scores alike
    masked = bias.clone()
    masked[1, 2:] = -math.inf
    masked[0, :] = 0
    r = reference(zero, k, v, masked, bounds, pos, ptr, 1.0, do)
    real = reference(q, k, v, torch.where(bias == LOWEST, even, bias), bounds, pos, ptr, 1.0, do)
    r["S"] = real["S"]
    check(r, {x: got[x] for x in ("out", "dv")}, 64, dtype)
    for x in ("dq", "dk"):
        bound = bounds_of(r, x, 64, dtype)
        within(got[x][:, 1], r[x][:, 1], bound[:, 1], x)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [3, 24, 50, 64, 128])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_masked_places_reach_nothing(bad, D, dtype):
    """Infinities and NaN in a token's q, k, v and d_out: rows before it and other rows stay as they are."""
    import paper_1108_2580_amd as p

    lens = [40, 90, 61]
    q, k, v, bias, bounds, pos, ptr, do = inputs(lens, 2, 1, D, 8, dtype, 23)
    r = reference(q, k, v, bias, bounds, pos, ptr, 0.2, do)
    limit = {x: bounds_of(r, x, D, dtype, 2) for x in ("out", "dq", "dk", "dv")}
    log(f"{bad} at width {D}, {dtype}")

    def same(name, rows):
        off = (got[name].double().cpu() - r[name])[rows].abs()
        assert (off <= limit[name][rows]).all(), (t, "qkvg"[which], name)

    for t in (0, 41, 100, 129, 190):
        row = 0 if t < 40 else 1 if t < 130 else 2
        first, end = sum(lens[:row]), sum(lens[:row + 1])
        others = [i for i in range(sum(lens)) if i < first or i >= end]
        for which in range(4):
            x = [y.clone() for y in (q, k, v, do)]
            x[which][t, :, D // 2] = bad
            got = run(p, *x[:3], bias, bounds, pos, ptr, x[3], 0.2)
            for name in ("out", "dq", "dk", "dv"):
                same(name, others)
            for name in ("out", "dq"):  # queries before the token do not read it
                same(name, slice(first, t))
            if which in (0, 3):  # what a query holds reaches no other query, and no key behind it
                for name in ("out", "dq"):
                    same(name, slice(t + 1, end))
                for name in ("dk", "dv"):
                    same(name, slice(t + 1, end))
            if which == 2:
                assert not torch.isfinite(got["out"][t:end, :, D // 2]).any()


def test_a_bucket_of_nan_reaches_its_tokens_alone():
    import paper_1108_2580_amd as p

    q, k, v, bias, bounds, pos, ptr, do = inputs([60, 50], 2, 2, 32, 4, "f32", 24)
    bias[1, 3] = math.nan
    got = run(p, q, k, v, bias, bounds, pos, ptr, do, 0.2)
    far = torch.zeros(110, dtype=torch.bool)
    for a, e in ((0, 60), (60, 110)):
        far[a:e] = (torch.tril((kinds(bounds, pos[a:e].cpu(), pos[a:e].cpu()) == 3).long()).sum(1) > 0)
    assert far.any() and not far.all()
    for name in ("out", "dq"):
        nan = torch.isnan(got[name].cpu()).all(-1)
        assert torch.equal(nan[:, 1], far) and not nan[:, 0].any(), name
    assert torch.isnan(got["dbias"][1]).any() and torch.isfinite(got["dbias"][0]).all()


def test_gradients_by_differences():
    import paper_1108_2580_amd as p

    q, k, v, bias, bounds, pos, ptr, do = inputs([9, 30, 1], 4, 2, 24, 6, "f32", 31)
    leaves = [t.detach().clone().requires_grad_() for t in (q, k, v, bias)]
    out = p.gap_attention(*leaves, bounds, pos, ptr, 0.4)
    grads = torch.autograd.grad(out, leaves, do)
    at = [t.detach().double().cpu() for t in leaves]
    G = do.double().cpu()
    loss = lambda x: float((reference(*x, bounds, pos, ptr, 0.4)["out"] * G).sum())  # noqa: E731
    g = torch.Generator().manual_seed(8)
    for i, grad in enumerate(grads):
        d = torch.randn(at[i].shape, generator=g).double()
        move = lambda h: [t + h * d if j == i else t for j, t in enumerate(at)]  # noqa: E731
        h = 1e-4
        want = (loss(move(h)) - loss(move(-h))) / (2 * h)
        got = float((grad.double().cpu() * d).sum())
        assert abs(got - want) <= 1e-5 * float((grad.double().cpu().abs() * d.abs()).sum()), (i, got, want)


def test_autograd_of_parts():
    """Only some inputs need gradients; the output's gradient has strides of its own; nothing is saved where
    none does."""
    import paper_1108_2580_amd as p

    q, k, v, bias, bounds, pos, ptr, do = inputs([50], 2, 2, 16, 6, "bf16", 32)
    args = (q, k, v, bias, bounds, pos, ptr)
    want = run(p, *args, do, 0.25)
    held = bias.clone().requires_grad_()
    out = p.gap_attention(q, k, v, held, bounds, pos, ptr, 0.25)
    assert torch.equal(out, want["out"])
    out.backward(do.transpose(0, 1).contiguous().transpose(0, 1))
    assert torch.equal(held.grad, want["dbias"])
    held.grad = None
    out, saved = p.gap_attention(q, k, v, held, bounds, pos, ptr, 0.25, return_saved=True)
    assert out.requires_grad and not any(t.requires_grad for t in saved)
    # the bounds of the forward pass count, whatever becomes of their tensor
    moved = bounds.clone()
    out = p.gap_attention(q, k, v, held, moved, pos, ptr, 0.25)
    moved.fill_(7)
    out.backward(do)
    assert torch.equal(held.grad, want["dbias"])


def test_tokens_of_no_row_stay_as_they_are():
    """Through the library's own entries, whose outputs are the caller's."""
    import paper_1108_2580_amd as p
    from paper_1108_2580_amd import lib, sequence as s

    for n_rows in (2, 90):
        lens = [30, 41] + [1] * (n_rows - 2)
        used = sum(lens)
        q, k, v, bias, bounds, pos, ptr, do = inputs([used + 70], 2, 1, 32, 6, "f32", 33)
        ptr = dev(torch.tensor([0] + lens).cumsum(0))
        want = run(p, *(t[:used] for t in (q, k, v)), bias, bounds, pos[:used], ptr, do[:used], 0.2)
        q[used:], k[used:], v[used:], do[used:] = (math.nan,) * 4
        dev_, code, shape, hq, hk, hv = s._gaps(q, k, v, bias, bounds, pos, ptr, 0.2)
        out, dq = torch.full_like(q.contiguous(), 5.0), torch.full_like(q.contiguous(), 6.0)
        dk, dv = torch.full_like(k.contiguous(), 7.0), torch.full_like(v.contiguous(), 8.0)
        stats, dbias = torch.full((2, 2, used + 70), math.nan, device="cuda:0"), torch.empty_like(bias)
        size = lib.als_gap_attention_backward_workspace(shape)
        work = torch.empty(size, dtype=torch.uint8, device="cuda:0")
        hdo = s._heads(do, "d_out", do.dtype, dev_)
        st = s._stream(dev_)
        s._check(lib.als_gap_attention(shape, code, hq, hk, hv, out.data_ptr(), stats.data_ptr(), None,
                                       work.data_ptr(), size, st))
        s._check(lib.als_gap_attention_backward(shape, code, hdo, hq, hk, hv, out.data_ptr(), stats.data_ptr(),
                                                None, dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                                                dbias.data_ptr(), work.data_ptr(), size, st))
        for x, name, fill in ((out, "out", 5.0), (dq, "dq", 6.0), (dk, "dk", 7.0), (dv, "dv", 8.0)):
            assert torch.equal(x[:used], want[name]), name
            assert (x[used:] == fill).all(), name
        assert torch.equal(dbias, want["dbias"])


def test_no_tokens():
    import paper_1108_2580_amd as p

    args = inputs([0, 0], 2, 1, 16, 4, "f32", 34)
    got = run(p, *args, 0.2)
    assert got["out"].shape == (0, 2, 16) and got["dbias"].shape == (2, 4) and not got["dbias"].any()


def test_row_pointers_out_of_range_touch_nothing():
    """Decreasing and too large values: results of such rows mean nothing, other memory stays as it is."""
    import paper_1108_2580_amd as p

    for extra in (0, 100):
        q, k, v, bias, bounds, pos, _, do = inputs([200], 2, 1, 32, 8, "bf16", 35)
        ptr = dev(torch.tensor([0, 150, 20, -5, 1 << 40, 70] + [200] * extra + [1 << 50]))
        run(p, q, k, v, bias, bounds, pos, ptr, do, 0.2)
        torch.cuda.synchronize()


# ---- steps -----------------------------------------------------------------------------------------

def step_inputs(lens, beams, steps, H, Hk, D, buckets, dtype, seed, last=2000, alike=True):
    q, k, v, bias, bounds, pos, ptr, _ = inputs(lens, H, Hk, D, buckets, dtype, seed, last)
    g = torch.Generator().manual_seed(seed + 1)
    rows = len(lens) * beams
    rand = lambda *shape: dev(torch.randn(shape, generator=g).to(DTYPES[dtype]))  # noqa: E731
    q1, kp, vp = rand(rows, H, D), rand(steps, rows, Hk, D), rand(steps, rows, Hk, D)
    path = dev(torch.randint(0, beams, (len(lens), beams, steps), generator=g, dtype=torch.int32))
    at = torch.randint(2 * last, 4 * last, (len(lens), 1 if alike else beams), generator=g).expand(-1, beams)
    q_pos = dev(at.reshape(-1).int())
    p_pos = dev((at.reshape(1, -1) - torch.randint(0, 30, (steps, rows), generator=g)).int())
    return q1, k, v, bias, bounds, q_pos, pos, ptr, kp, vp, p_pos, path


def step_reference(q, k, v, bias, bounds, q_pos, pos, ptr, kp, vp, p_pos, path, scale):
    """(out, sizes, S, terms) in fp64 on the CPU."""
    q, k, v, bias, kp, vp = (t.double().cpu() for t in (q, k, v, bias, kp, vp))
    q_pos, pos, p_pos, path, ptr = (t.cpu() for t in (q_pos, pos, p_pos, path, ptr))
    B, W, T = path.shape
    H, group = q.shape[1], q.shape[1] // k.shape[1]
    out, size, S, terms = torch.zeros_like(q), torch.zeros_like(q), 0.0, 0
    for row in range(B * W):
        b, w = divmod(row, W)
        a, e = int(ptr[b]), int(ptr[b + 1])
        held = [b * W + int(x) for x in path[b, w]]
        keys = torch.cat([k[a:e], torch.stack([kp[t, r] for t, r in enumerate(held)])]) if T else k[a:e]
        values = torch.cat([v[a:e], torch.stack([vp[t, r] for t, r in enumerate(held)])]) if T else v[a:e]
        of = torch.cat([pos[a:e]] + [p_pos[t, r:r + 1] for t, r in enumerate(held)])
        if keys.shape[0] == 0:
            continue
        terms = max(terms, keys.shape[0])
        kind = kinds(bounds, q_pos[row:row + 1], of)[0]
        K, V = keys.repeat_interleave(group, 1), values.repeat_interleave(group, 1)
        x = scale * (q[row][None] * K).sum(-1) + bias[:, kind].T
        s = abs(scale) * (q[row].abs()[None] * K.abs()).sum(-1) + bias[:, kind].T.abs().nan_to_num(0.0, 0.0, 0.0)
        S = max(S, float(s.amax()))
        wt = softmax(x.T)
        out[row] = torch.einsum("hn,nhd->hd", wt, V)
        size[row] = torch.einsum("hn,nhd->hd", wt, V.abs())
    return out, size, S, terms


def check_step(got, want, D, dtype):
    out, size, S, n = want
    # as forward; parts of rows are joined (3 roundings each, at most one part for each 32 tokens)
    rel = 2 * ((D + 16) * S + 4) * E + 2 * n * E + 64 * E + (dtype == "bf16") * 2.0 ** -16
    within(got, out, (U if dtype == "bf16" else E) * out.abs() + 1.05 * rel * size + 1e-30, "out")


STEPS = [  # lengths, beams, steps, heads, key heads, width, buckets
    ([1], 1, 1, 1, 1, 1, 1), ([262], 8, 5, 8, 8, 64, 32), ([0, 40, 0], 5, 3, 4, 2, 50, 16), ([33, 128, 129, 1], 4, 1, 4, 1, 128, 64),
    ([700, 20], 16, 9, 8, 2, 64, 32), ([300], 32, 20, 4, 4, 32, 9), ([90] * 70, 2, 2, 2, 1, 20, 5),
    ([150], 16, 2, 8, 1, 64, 8), ([200, 5], 16, 4, 16, 2, 100, 16), ([2000], 3, 7, 2, 2, 7, 40), ([64, 31], 7, 0, 2, 2, 64, 8),
    # as many beams and heads as take a wave each, or a part of one; segments of 256 tokens
    ([20] * 40, 16, 3, 4, 2, 50, 16), ([12, 0, 30] * 50, 16, 6, 8, 4, 40, 8), ([40] * 70, 16, 9, 16, 4, 128, 8),
    ([70_000], 2, 1, 4, 4, 16, 8)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,beams,steps,H,Hk,D,buckets", STEPS)
def test_step(lens, beams, steps, H, Hk, D, buckets, dtype):
    import paper_1108_2580_amd as p

    for alike, last in ((True, 2000), (False, 50_000)):
        log(f"lengths {lens[:4]}, {beams} beams, {steps} steps, {H}/{Hk} heads, width {D}, {dtype}, {alike}")
        args = step_inputs(lens, beams, steps, H, Hk, D, buckets, dtype, sum(lens) + D, last, alike)
        scale = -0.2 if alike else D ** -0.5
        got = p.gap_attention_step(*args, scale=scale)
        check_step(got, step_reference(*args, scale), D, dtype)
        assert torch.equal(got, p.gap_attention_step(*args, scale=scale))
        if steps == 0:
            assert torch.equal(got, p.gap_attention_step(*args[:8], scale=scale))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_step_strides_and_parts_of_longer_tensors(dtype):
    import paper_1108_2580_amd as p

    q, k, v, bias, bounds, q_pos, pos, ptr, kp, vp, p_pos, path = step_inputs(
        [70, 30], 4, 3, 4, 2, 40, 8, dtype, 41)
    want = p.gap_attention_step(q, k, v, bias, bounds, q_pos, pos, ptr, kp, vp, p_pos, path)
    long = torch.full((9, 8, 2, 2, 43), math.nan, dtype=q.dtype, device="cuda:0")
    long[:3, :, :, 0, 1:41], long[:3, :, :, 1, 1:41] = kp, vp
    table = torch.full((2, 4, 9), -1, dtype=torch.int32, device="cuda:0")
    table[..., :3] = path
    wide = torch.full((8, 4, 51), math.nan, dtype=q.dtype, device="cuda:0")
    wide[..., 5:45] = q
    got = p.gap_attention_step(wide[..., 5:45], k, v, bias, bounds, q_pos, pos, ptr, long[:3, :, :, 0, 1:41],
                               long[:3, :, :, 1, 1:41], torch.cat([p_pos] * 2)[:3], table[..., :3])
    assert torch.equal(got, want)


def test_step_masks_and_holders_out_of_range():
    import paper_1108_2580_amd as p

    q, k, v, bias, bounds, q_pos, pos, ptr, kp, vp, p_pos, path = step_inputs([70, 0], 2, 3, 2, 2, 32, 8, "f32", 42)
    bias[0, :] = -math.inf
    bias[1, 3:] = -math.inf
    args = (q, k, v, bias, bounds, q_pos, pos, ptr, kp, vp, p_pos)
    got = p.gap_attention_step(*args, path)
    assert not got[:, 0].any()
    check_step(got, step_reference(*args, path, 32 ** -0.5), 32, "f32")
    for bad in (-1, 2, 1 << 30):
        other = path.clone()
        other[0, 1, 2] = bad
        out = p.gap_attention_step(*args, other)
        assert torch.isnan(out[1]).all()
        keep = [0, 2, 3]
        assert torch.equal(out[keep], got[keep])


def test_step_infinities_reach_no_other_list_or_beam():
    import paper_1108_2580_amd as p

    for dtype in ("f32", "bf16"):
        q, k, v, bias, bounds, q_pos, pos, ptr, kp, vp, p_pos, path = step_inputs(
            [70, 35], 3, 2, 2, 2, 32, 8, dtype, 43)
        path[:] = torch.arange(3, device="cuda:0")[:, None]
        rest = (bias, bounds, q_pos, pos, ptr)
        want = p.gap_attention_step(q, k, v, *rest, kp, vp, p_pos, path)
        x = [t.clone() for t in (q, k, v, kp, vp)]
        x[0][4] = math.nan
        x[3][1, 5] = math.nan
        x[4][0, 3] = math.inf
        out = p.gap_attention_step(*x[:3], *rest, *x[3:], p_pos, path)
        assert torch.equal(out[:3], want[:3])
        assert torch.isnan(out[4:]).all() and not torch.isfinite(out[3]).any()
        x = [t.clone() for t in (k, v)]
        x[0][70], x[1][80] = math.nan, math.nan
        out = p.gap_attention_step(q, *x, *rest, kp, vp, p_pos, path)
        assert torch.equal(out[:3], want[:3]) and torch.isnan(out[3:]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_model_reads_learns_and_answers(dtype):
    """The operators as they run together: gradients over histories, then lists by beam search whose every
    step is what the whole sequence (history and the beam's path) gives at its last token."""
    import paper_1108_2580_amd as p

    dt, D, H, Hk, items, W, steps = DTYPES[dtype], 32, 4, 2, 300, 4, 4
    g = torch.Generator().manual_seed(5)
    rand = lambda *s: dev(torch.randn(s, generator=g))  # noqa: E731
    table = rand(items, D).to(dt)
    proj = (rand(D, (H + 2 * Hk) * D) / D ** 0.5).to(dt)
    back = (rand(H * D, D) / (H * D) ** 0.5).to(dt)
    bounds = torch.tensor([1, 4, 20, 100, 700], dtype=torch.int32)
    bias = (0.3 * rand(H, 6)).requires_grad_()
    lens = [40, 3, 0, 75]
    ptr = dev(torch.tensor([0] + lens).cumsum(0))
    ids = dev(torch.randint(0, items, (sum(lens),), generator=g))
    pos = dev(torch.cat([torch.randint(0, 900, (n,), generator=g).sort().values for n in lens]).int())

    def split(x):
        y = (x @ proj).view(-1, H + 2 * Hk, D)
        return y[:, :H], y[:, H:H + Hk], y[:, H + Hk:]

    proj.requires_grad_()
    out = p.gap_attention(*split(table[ids]), bias, bounds, pos, ptr)
    (out.flatten(1) @ back).float().square().mean().backward()
    assert torch.isfinite(bias.grad).all() and bias.grad.abs().sum() > 0 and proj.grad.abs().sum() > 0

    with torch.no_grad():
        B = len(lens)
        _, k, v = split(table[ids])
        scores = torch.full((B, W), -math.inf, device="cuda:0")
        scores[:, 0] = 0
        chosen = torch.zeros(B, W, steps, dtype=torch.int32, device="cuda:0")
        path = torch.zeros(B, W, steps, dtype=torch.int32, device="cuda:0")
        kp, vp = (torch.zeros(steps, B * W, Hk, D, dtype=dt, device="cuda:0") for _ in range(2))
        pp = torch.zeros(steps, B * W, dtype=torch.int32, device="cuda:0")
        token = dev(torch.randint(0, items, (B, W), generator=g).int())
        for t in range(steps):
            x = table[token.flatten().long()]
            q, kp[t], vp[t] = split(x)
            pp[t] = 900 + t
            chosen[..., t], path[..., t] = token, torch.arange(W, device="cuda:0", dtype=torch.int32)
            out = p.gap_attention_step(q, k, v, bias, bounds, pp[t], pos, ptr, kp[:t + 1], vp[:t + 1],
                                       pp[:t + 1], path[..., :t + 1])
            # the same by whole sequences
            for b in range(B):
                for w in range(W):
                    a, e = int(ptr[b]), int(ptr[b + 1])
                    seq = torch.cat([ids[a:e], chosen[b, w, :t + 1].long()])
                    at = torch.cat([pos[a:e], 900 + torch.arange(t + 1, device="cuda:0", dtype=torch.int32)])
                    whole = p.gap_attention(*split(table[seq]), bias, bounds, at,
                                            dev(torch.tensor([0, seq.numel()])))
                    off = (whole[-1].double() - out[b * W + w].double()).abs().max()
                    # matrix products of other shapes may round q, k and v to the neighbouring value
                    assert off <= (0.06 if dtype == "bf16" else 2e-5), (t, b, w, float(off))
            logits = ((out.flatten(1) @ back).float() @ table.float().T).view(B, W, items)
            parents, token, scores, _ = p.beam_select(logits, scores)
            p.reorder_states(chosen, parents, chosen)
            p.reorder_states(path, parents, path)


# ---- streams and graphs ------------------------------------------------------------------------------

def test_on_another_stream():
    import paper_1108_2580_amd as p

    args = inputs([300, 20], 2, 1, 64, 16, "bf16", 51)
    want = run(p, *args, 0.2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run(p, *args, 0.2)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(got[x], want[x]) for x in got)


@pytest.mark.parametrize("rows", [2, 100])
def test_captured(rows):
    """A training pass and a step in graphs of their own, replayed several times with eager work between."""
    import paper_1108_2580_amd as p

    lens = [150, 60] + [2] * (rows - 2)
    args = inputs(lens, 4, 2, 64, 16, "bf16", 52)
    other = inputs(lens, 4, 2, 64, 16, "bf16", 53)
    step = step_inputs(lens, 3, 2, 4, 2, 64, 16, "bf16", 54)
    run(p, *args, 0.2), p.gap_attention_step(*step)
    torch.cuda.synchronize()
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1):
        got = run(p, *args, 0.2)
    with torch.cuda.graph(g2):
        out = p.gap_attention_step(*step)
    for i in range(4):
        source = other if i % 2 else inputs(lens, 4, 2, 64, 16, "bf16", 52)
        for a, b in zip(args, source):
            if a.is_cuda:
                a.copy_(b)
        step[0].mul_(-1.0)
        g1.replay()
        g2.replay()
        want = run(p, *args, 0.2)
        torch.cuda.synchronize()
        assert all(torch.equal(got[x], want[x]) for x in got), i
        assert torch.equal(out, p.gap_attention_step(*step)), i


def test_captured_autograd():
    """A backward pass through the graph of autograd, captured with the leaves' gradients as outputs."""
    import paper_1108_2580_amd as p

    q, k, v, bias, bounds, pos, ptr, do = inputs([150, 60], 2, 2, 32, 8, "f32", 55)
    leaves = [t.detach().clone().requires_grad_() for t in (q, k, v, bias)]
    step = lambda: torch.autograd.grad(p.gap_attention(*leaves, bounds, pos, ptr), leaves, do)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))

"""Timed cases of the attention over gaps of time: softmax attention over packed histories with a
learned bias for each bucket of the gap between two ratings, its gradients, and its step for the
beams of a list, which share the user's history.

A next-item model reads a user's ratings in the order of time: a token is a rated item, its
position is its time bin, and the users' histories are packed one after the other like the rows of
the rating matrix (``row_ptr``). A rating attends to the ratings of its user up to itself; how long
ago those were enters the scores as a bias that each head learns for each bucket of the gap. The
model answers with lists of items by beam search: the beams of a list read the one history of their
user, and each the few items that it has chosen itself. Sizes are those of the library's matrices:
histories with a mean of 25 (the small set) and 262 ratings and of up to a tenth of the catalogue
(62 496), 6649 time bins, widths up to 128.

Where ``own`` is false, ``run`` computes the operators in their plain form: elementary torch
operations in 32 bits over padded batches of histories, rounded once at the end. Where it is true,
it calls the library's operators. ``exact`` repeats a pass in 64 bits, history by history.
"""
from __future__ import annotations

import functools
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TIME_BINS = 6_649
SCORES = 1 << 27  # scores that the plain form holds at a time
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one user of the small set; latency
        dict(name="read_one_user_f32", task="read", train=False, users=1, tokens=25, law="even",
             q_heads=4, k_heads=4, width=32, buckets=16, dtype="f32"),
        # the small set's histories at an odd width, shared key heads
        dict(name="read_odd_f32", task="read", train=False, users=2_000, tokens=50_000,
             law="lognormal", q_heads=4, k_heads=2, width=50, buckets=16, dtype="f32"),
        # reading in the histories of 512 users of the full-size set, before their lists are made
        dict(name="read_ragged_bf16", task="read", train=False, users=512, tokens=134_219,
             law="lognormal", q_heads=8, k_heads=8, width=64, buckets=32, dtype="bf16"),
        # reading in the longest history (a user who rated a tenth of the catalogue)
        dict(name="read_long_bf16", task="read", train=False, users=1, tokens=62_496, law="even",
             q_heads=8, k_heads=2, width=64, buckets=32, dtype="bf16"),
        # a small training batch; latency
        dict(name="train_small_bf16", task="read", train=True, users=8, tokens=2_001,
             law="lognormal", q_heads=8, k_heads=8, width=64, buckets=32, dtype="bf16"),
        # a training batch of 4096 users with histories of the full-size set's lengths
        dict(name="train_ragged_bf16", task="read", train=True, users=4_096, tokens=1_075_431,
             law="lognormal", q_heads=8, k_heads=8, width=64, buckets=32, dtype="bf16"),
        # training on long histories at the widest heads, with the most buckets
        dict(name="train_long_bf16_w128", task="read", train=True, users=4, tokens=32_003,
             law="even", q_heads=8, k_heads=8, width=128, buckets=64, dtype="bf16"),
        # training in 32 bits at the widest heads, four query heads to a key head
        dict(name="train_shared_f32_w128", task="read", train=True, users=100, tokens=25_003,
             law="lognormal", q_heads=8, k_heads=2, width=128, buckets=32, dtype="f32"),
        # serving one user: the fifth item of each of 8 beams; latency
        dict(name="step_one_user_bf16", task="step", lists=1, tokens=262, law="even", beams=8,
             steps=5, q_heads=8, k_heads=8, width=64, buckets=32, dtype="bf16"),
        # serving the user with the longest history
        dict(name="step_long_bf16", task="step", lists=1, tokens=62_496, law="even", beams=8,
             steps=5, q_heads=8, k_heads=8, width=64, buckets=32, dtype="bf16"),
        # serving many users, an odd width, five beams, shared key heads
        dict(name="step_odd_f32", task="step", lists=200, tokens=52_400, law="lognormal", beams=5,
             steps=3, q_heads=4, k_heads=2, width=50, buckets=16, dtype="f32"),
        # serving many users with wide beams
        dict(name="step_many_bf16", task="step", lists=1_024, tokens=268_859, law="lognormal",
             beams=16, steps=9, q_heads=8, k_heads=8, width=64, buckets=32, dtype="bf16"),
    ]


def draw(rng):
    def log_int(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))

    task = rng.choice(["read", "read", "step"])
    dtype = rng.choice(["f32", "bf16"])
    k = rng.choice([1, 2, 4, 8])
    q = k * rng.choice([1, 1, 2, 4])
    width = rng.choice([64, 128, rng.randint(8, 128), 8 * rng.randint(2, 16)])
    case = dict(task=task, law=rng.choice(["even", "lognormal", "lognormal"]), q_heads=q, k_heads=k,
                width=width, buckets=rng.choice([1, 8, 16, 32, 64, rng.randint(2, 64)]), dtype=dtype)
    if task == "step":
        beams = rng.choice([1, 4, 5, 8, 16])
        steps = rng.randint(1, 20)
        tokens = log_int(100, min(260_000, int(2.5e10 / (q * width * beams))))
        lists = log_int(1, max(1, min(1_024, tokens // 4)))
        return dict(case, lists=lists, tokens=tokens, beams=beams, steps=steps)
    train = rng.random() < 0.5
    # pairs of a query and a key that all heads' products may have, and values of the inputs
    pairs = (2e8 if train else 6e8) * (8 * 64) / (q * width) * (1.0 if dtype == "bf16" else 0.25)
    mean = log_int(16, int(min(40_000, 0.4 * pairs ** 0.5)))
    users = log_int(1, int(min(4_096, max(1.0, pairs / (2.0 * mean * mean)), max(1.0, 5e8 / (q * width * mean)))))
    return dict(case, train=train, users=users, tokens=max(1, users * mean + rng.randint(-7, 7)))


# ---- inputs --------------------------------------------------------------------------------

def _lengths(case):
    """Tokens of each user: about even, or lognormal around half the mean with some users without
    a rating, as in the library's full-size sets. The same for every seed, in another order."""
    B, N = case["users"] if case["task"] == "read" else case["lists"], case["tokens"]
    rng = np.random.default_rng(1_000_003 * B + N)
    if case["law"] == "even":
        share = np.full(B, 1.0 / B)
    else:
        share = np.exp(math.sqrt(2.0 * math.log(2.0)) * rng.standard_normal(B))
        share[rng.random(B) < 0.02] = 0.0
        share = share / share.sum() if share.sum() > 0 else np.full(B, 1.0 / B)
    ends = np.floor(np.cumsum(share) * N + 0.5).astype(np.int64)
    ends[-1] = N
    return np.diff(np.concatenate([[0], np.minimum(ends, N)]))


def _bounds(buckets):
    """First gap of each bucket but the first, on the host: one by one, then by equal factors."""
    out = []
    for b in range(1, buckets):
        at = round(TIME_BINS ** (b / buckets))
        out.append(max(at, out[-1] + 1 if out else 1))
    return torch.tensor(out, dtype=torch.int32)


def _batches(lens, heads):
    """Rows of about one length, whose padded scores are held at a time: (rows, longest)."""
    order = np.argsort(-lens, kind="stable")
    order = order[lens[order] > 0]
    out, i = [], 0
    while i < order.size:
        most = int(lens[order[i]])
        n = int(min(max(1, SCORES // (heads * most * most)), order.size - i))
        # rows much shorter than the longest go with others
        n = max(1, int(np.searchsorted(-lens[order[i:i + n]], -0.6 * most, side="right")))
        out.append((torch.from_numpy(order[i:i + n]).to(DEV), most))
        i += n
    return out


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    rng = np.random.default_rng(seed)
    dtype = DTYPES[case["dtype"]]

    def normal(*shape, dtype=dtype):
        return torch.randn(shape, generator=gen, device=DEV).to(dtype)

    q, k, D = case["q_heads"], case["k_heads"], case["width"]
    N = case["tokens"]
    lens = rng.permutation(_lengths(case))
    s = dict(case=case, task=case["task"], lens=lens, scale=D ** -0.5, bounds=_bounds(case["buckets"]),
             bias=0.5 * normal(q, case["buckets"], dtype=torch.float32))
    s["row_ptr"] = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)])).to(DEV)
    # time bins, ascending within each user's history
    user = torch.repeat_interleave(torch.arange(lens.size, device=DEV), torch.from_numpy(lens).to(DEV),
                                   output_size=N)
    bins = torch.randint(0, TIME_BINS, (N,), generator=gen, device=DEV)
    s["positions"] = ((user * TIME_BINS + bins).sort().values - user * TIME_BINS).int()
    # queries, keys and values are views of one projection's rows, as a model has them
    if s["task"] == "read":
        both = normal(N, q + 2 * k, D)
        s.update(q=both[:, :q], k=both[:, q:q + k], v=both[:, q + k:])
        if case["train"]:
            s["do"] = normal(N, q, D)
    else:
        B, W, T = case["lists"], case["beams"], case["steps"]
        both = normal(N, 2 * k, D)
        s.update(k=both[:, :k], v=both[:, k:], q=normal(B * W, q, D))
        s.update(k_path=normal(T, B * W, k, D), v_path=normal(T, B * W, k, D))
        # the beam that holds each step of a beam's path; its own at the last
        path = torch.randint(0, W, (B, W, T), generator=gen, device=DEV, dtype=torch.int32)
        path[:, :, -1] = torch.arange(W, device=DEV, dtype=torch.int32)
        # lists go on at the bin of their user's last rating
        last = torch.where(torch.from_numpy(lens > 0).to(DEV),
                           s["positions"][(s["row_ptr"][1:] - 1).clamp(min=0)], 0).int()
        at = last.repeat_interleave(W)
        s.update(path=path, q_positions=at, path_positions=at.expand(T, -1).contiguous())
    s["batches"] = _batches(lens, q)
    return s


# ---- the plain forms -------------------------------------------------------------------------

def _table(s):
    """The bucket of each gap up to the last bound."""
    last = int(s["bounds"][-1]) if s["bounds"].numel() else 0
    gaps = torch.arange(last + 1)
    return (gaps[:, None] >= s["bounds"][None, :]).sum(1).to(DEV)


def _buckets(table, gap):
    return table[gap.clamp(0, table.numel() - 1).long()]


def _padded(s, rows, most):
    """Tokens [rows, most] of a batch, and which of them there are."""
    first = s["row_ptr"][rows]
    at = torch.arange(most, device=DEV)
    live = at < (s["row_ptr"][rows + 1] - first)[:, None]
    return torch.where(live, first[:, None] + at, 0), live


def _weights(scores):
    """Softmax over the last axis, zero where it has only masked places; and the scores' sum."""
    top = scores.amax(-1, keepdim=True)
    w = torch.exp(scores - torch.where(torch.isinf(top), 0.0, top))
    return w / w.sum(-1, keepdim=True).clamp(min=1e-37)


def _plain_read(s):
    case, dtype = s["case"], DTYPES[s["case"]["dtype"]]
    H, group = case["q_heads"], case["q_heads"] // case["k_heads"]
    N, D = case["tokens"], case["width"]
    table = _table(s)
    kinds = torch.arange(case["buckets"], device=DEV)
    # a row behind the last takes what lies past a history's end
    new = lambda heads: torch.zeros((N + 1, heads, D), device=DEV)  # noqa: E731
    out = new(H)
    if case["train"]:
        dq, dk, dv = new(H), new(case["k_heads"]), new(case["k_heads"])
        dbias = torch.zeros_like(s["bias"])
    for rows, most in s["batches"]:
        token, live = _padded(s, rows, most)
        to = torch.where(live, token, N)
        cut = lambda x: (x[token].float() * live[..., None, None]).transpose(1, 2)  # noqa: E731
        q = cut(s["q"]) * s["scale"]
        k, v = (cut(s[x]).repeat_interleave(group, 1) for x in "kv")
        at = s["positions"][token]
        if case["train"]:
            do = cut(s["do"])
            gk, gv = torch.zeros_like(k), torch.zeros_like(v)
        step = max(1, min(most, SCORES // (rows.numel() * H * most)))
        for i in range(0, most, step):  # queries i .. e - 1 and the keys up to them
            e = min(most, i + step)
            bucket = _buckets(table, at[:, i:e, None] - at[:, None, :e])
            later = torch.arange(i, e, device=DEV)[:, None] < torch.arange(e, device=DEV)
            masked = (later | ~live[:, None, :e])[:, None]
            scores = torch.matmul(q[:, :, i:e], k[:, :, :e].transpose(2, 3))
            scores = scores + s["bias"][:, bucket].transpose(0, 1)
            w = _weights(scores.masked_fill(masked, -math.inf))
            o = torch.matmul(w, v[:, :, :e])
            out[to[:, i:e]] = o.transpose(1, 2)
            if case["train"]:
                g = do[:, :, i:e]
                ds = torch.matmul(g, v[:, :, :e].transpose(2, 3))
                ds = w * (ds - (g * o).sum(-1, keepdim=True))
                gv[:, :, :e] += torch.matmul(w.transpose(2, 3), g)
                gk[:, :, :e] += torch.matmul(ds.transpose(2, 3), q[:, :, i:e])
                dq[to[:, i:e]] = (torch.matmul(ds, k[:, :, :e]) * s["scale"]).transpose(1, 2)
                kind = (bucket[..., None] == kinds).float()
                dbias += torch.matmul(ds.transpose(0, 1).reshape(H, -1), kind.view(-1, kinds.numel()))
        if case["train"]:
            shared = lambda x: x.unflatten(1, (-1, group)).sum(2).transpose(1, 2)  # noqa: E731
            dk[to], dv[to] = shared(gk), shared(gv)
    if not case["train"]:
        return [out[:N].to(dtype)]
    return [x[:N].to(dtype) for x in (out, dq, dk, dv)] + [dbias]


def _plain_step(s):
    case, dtype = s["case"], DTYPES[s["case"]["dtype"]]
    H, group = case["q_heads"], case["q_heads"] // case["k_heads"]
    B, W, T = case["lists"], case["beams"], case["steps"]
    table = _table(s)
    wide = lambda x, dim: x.float().repeat_interleave(group, dim)  # noqa: E731
    q = s["q"].view(B, W, H, -1).transpose(1, 2).float() * s["scale"]
    at = s["q_positions"].view(B, W)
    # each beam's own path: [lists, heads, beams, steps, ...]
    beam = torch.arange(B, device=DEV)[:, None, None] * W + s["path"]
    nth = torch.arange(T, device=DEV)
    kp, vp = (wide(s[x][nth, beam], 3).permute(0, 3, 1, 2, 4) for x in ("k_path", "v_path"))
    bucket = _buckets(table, at[..., None] - s["path_positions"][nth, beam])
    own = (q[:, :, :, None] * kp).sum(-1) + s["bias"][:, bucket].transpose(0, 1)
    out = torch.empty_like(q)
    some = torch.zeros(B, dtype=torch.bool, device=DEV)
    for rows, most in s["batches"]:
        token, live = _padded(s, rows, most)
        some[rows] = True
        k, v = (wide(s[x][token] * live[..., None, None], 2).transpose(1, 2) for x in "kv")
        bucket = _buckets(table, at[rows][..., None] - s["positions"][token][:, None])
        scores = torch.matmul(q[rows], k.transpose(2, 3)) + s["bias"][:, bucket].transpose(0, 1)
        scores = scores.masked_fill(~live[:, None, None], -math.inf)
        w = _weights(torch.cat([scores, own[rows]], -1))
        out[rows] = torch.matmul(w[..., :most], v) + (w[..., most:, None] * vp[rows]).sum(3)
    alone = (_weights(own)[..., None] * vp).sum(3)  # users without a history
    out = torch.where(some[:, None, None, None], out, alone)
    return [out.transpose(1, 2).reshape(B * W, H, -1).to(dtype)]


# ---- the library's operators -------------------------------------------------------------------

@functools.cache
def _library():
    from paper_1108_2580_amd import sequence

    return sequence


def _own(s):
    lib = _library()
    if s["task"] == "step":
        return [lib.gap_attention_step(s["q"], s["k"], s["v"], s["bias"], s["bounds"], s["q_positions"],
                                       s["positions"], s["row_ptr"], s["k_path"], s["v_path"],
                                       s["path_positions"], s["path"], scale=s["scale"])]
    args = (s["q"], s["k"], s["v"], s["bias"], s["bounds"], s["positions"], s["row_ptr"])
    if not s["case"]["train"]:
        return [lib.gap_attention(*args, scale=s["scale"])]
    out, saved = lib.gap_attention(*args, scale=s["scale"], return_saved=True)
    return [out, *lib.gap_attention_backward(s["do"], out, saved, *args, scale=s["scale"])]


def run(state):
    if own:
        return _own(state)
    return _plain_step(state) if state["task"] == "step" else _plain_read(state)


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    q, k, D, N = case["q_heads"], case["k_heads"], case["width"], case["tokens"]
    bias = 4 * q * case["buckets"]
    lens = _lengths(case).astype(float)
    if case["task"] == "step":
        rows, T = case["lists"] * case["beams"], case["steps"]
        pairs = case["beams"] * N + rows * T
        return {"bytes": (2 * (N + rows * T) * k + 2 * rows * q) * D * size + 4 * (N + rows * (2 * T + 1)) + bias,
                "flops": 4 * pairs * q * D}
    pairs = float((lens * (lens + 1.0)).sum()) / 2.0
    once = (2 * q + 2 * k) * D * size * N + 4 * N + bias  # q, k, v, out
    if not case["train"]:
        return {"bytes": once, "flops": 4 * pairs * q * D}
    # backward: q, k, v, out and its gradient again, three gradients; five products of the pairs
    return {"bytes": 2 * once + (2 * q + 2 * k) * D * size * N + bias, "flops": 14 * pairs * q * D}


# ---- the definitions in 64 bits ------------------------------------------------------------------

def _kinds(bounds, gap):
    """The number of bounds that a gap reaches."""
    return torch.searchsorted(bounds.to(DEV).long(), gap.long().clamp(min=0), right=True)


def _exact_read(s):
    case = s["case"]
    H, Hk, D, N = case["q_heads"], case["k_heads"], case["width"], case["tokens"]
    group, train = H // Hk, case["train"]
    squares = float((s["lens"].astype(float) ** 2).sum()) / 2.0 * H
    if squares * (8 * D * (3.5 if train else 1.0) / 2e13 + (700 if train else 120) / 2e12) \
            + s["lens"].size * (2e-3 if train else 3e-4) > 15.0:
        return None
    f64 = dict(device=DEV, dtype=torch.float64)
    bias = s["bias"].double()
    out = torch.zeros((N, H, D), **f64)
    if train:
        dq, dk, dv = (torch.zeros((N, h, D), **f64) for h in (H, Hk, Hk))
        dbias = torch.zeros_like(bias)
    ptr = np.concatenate([[0], np.cumsum(s["lens"])])
    for a, b in zip(ptr[:-1], ptr[1:]):
        if a == b:
            continue
        heads = lambda x, n: x[a:b].double().movedim(0, 1).contiguous()[:, None].expand(  # noqa: E731
            -1, n, -1, -1).reshape(H, b - a, D)
        q, k, v = heads(s["q"], 1), heads(s["k"], group), heads(s["v"], group)
        at = s["positions"][a:b].long()
        step = max(1, min(b - a, (1 << 26) // (H * (b - a))))
        for i in range(0, b - a, step):
            e = min(b - a, i + step)
            kind = _kinds(s["bounds"], at[i:e, None] - at[None, :e])
            x = torch.bmm(q[:, i:e], k[:, :e].mT) * s["scale"] + bias[:, kind]
            x = torch.where(torch.ones(e - i, e, dtype=torch.bool, device=DEV).tril(i), x, -math.inf)
            w = torch.softmax(x, -1)
            o = torch.bmm(w, v[:, :e])
            out[a + i:a + e] = o.movedim(0, 1)
            if train:
                g = s["do"][a + i:a + e].double().movedim(0, 1).contiguous()
                dw = torch.bmm(g, v[:, :e].mT)
                dx = w * (dw - (w * dw).sum(-1, keepdim=True))
                dq[a + i:a + e] = torch.bmm(dx, k[:, :e]).movedim(0, 1) * s["scale"]
                dk[a:a + e] += (torch.bmm(dx.mT, q[:, i:e]) * s["scale"]).view(Hk, group, e, D).sum(1).movedim(0, 1)
                dv[a:a + e] += torch.bmm(w.mT, g).view(Hk, group, e, D).sum(1).movedim(0, 1)
                for n in range(case["buckets"]):
                    dbias[:, n] += (dx * (kind == n)).sum((1, 2))
    return [out] + ([dq, dk, dv, dbias] if train else [])


def _exact_step(s):
    case = s["case"]
    H, Hk, W, T = case["q_heads"], case["k_heads"], case["beams"], case["steps"]
    if 8 * W * H * case["tokens"] * case["width"] / 2e12 + case["lists"] * 2e-3 > 15.0:
        return None
    bias, bounds = s["bias"].double(), s["bounds"]
    out = torch.empty(s["q"].shape, device=DEV, dtype=torch.float64)
    ptr = np.concatenate([[0], np.cumsum(s["lens"])])
    nth = torch.arange(T, device=DEV)
    for n in range(case["lists"]):
        a, b = ptr[n], ptr[n + 1]
        mine = slice(n * W, (n + 1) * W)
        q = s["q"][mine].double().unflatten(1, (Hk, -1)) * s["scale"]  # beams, key heads, group, width
        at = s["q_positions"][mine].long()
        rows = n * W + s["path"][n].long()
        kp, vp = (s[x][nth, rows].double() for x in ("k_path", "v_path"))  # beams, steps, key heads, width
        x = torch.einsum("wkgd,nkd->wkgn", q, s["k"][a:b].double())
        x = x + bias.view(Hk, -1, bias.shape[1])[:, :, _kinds(bounds, at[:, None] - s["positions"][a:b])].permute(2, 0, 1, 3)
        y = torch.einsum("wkgd,wtkd->wkgt", q, kp)
        y = y + bias.view(Hk, -1, bias.shape[1])[:, :, _kinds(bounds, at[:, None] - s["path_positions"][nth, rows])].permute(2, 0, 1, 3)
        w = torch.softmax(torch.cat([x, y], -1), -1)
        o = torch.einsum("wkgn,nkd->wkgd", w[..., :b - a], s["v"][a:b].double())
        out[mine] = (o + torch.einsum("wkgt,wtkd->wkgd", w[..., b - a:], vp)).flatten(1, 2)
    return [out]


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_step(s) if s["task"] == "step" else _exact_read(s)

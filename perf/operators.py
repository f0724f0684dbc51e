"""Timed cases of the sequence operators: norm and rotation of queries and keys, linear
attention with a decay for each head, and beam selection with its states.

A next-item model reads a user's ratings in the order of time: a token is a rated item, its
position is its time bin, and the users' histories are packed one after the other like the
rows of the rating matrix (``row_ptr``). The model answers with lists of items from the
whole catalogue, by beam search over the recurrent states. Sizes are those of the library's
matrices: catalogues of 1 000, 50 000 and 624 961 items, histories with a mean of 262
ratings and of up to a tenth of the catalogue, 6649 time bins, widths up to 128.

Where ``own`` is false, ``run`` computes the operators in their plain form: elementary torch
operations in 32 bits, rounded once at the end. Where it is true, it calls the library's
operators. ``exact`` repeats a pass in 64 bits from the definitions, token by token.
"""
from __future__ import annotations

import functools
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
EPS = 1e-6
TIME_BINS = 6_649
CHUNK = 64  # tokens per chunk of the plain attention
END = 0     # the item that ends a list
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # serving: the queries and keys of one token for 8 users x 8 beams; latency
        dict(name="rotate_token_bf16", task="rotate", train=False, tokens=64, q_heads=8, k_heads=8,
             width=64, rotated=64, neighbours=False, dtype="bf16"),
        # training in 32 bits at the library's wide factor width (100), an odd number of tokens
        dict(name="rotate_train_f32_w100", task="rotate", train=True, tokens=200_003, q_heads=4,
             k_heads=4, width=100, rotated=100, neighbours=False, dtype="f32"),
        # a large training batch: a token for every user of the full-size set, shared key heads
        dict(name="rotate_train_bf16_w128", task="rotate", train=True, tokens=1_000_990, q_heads=8,
             k_heads=2, width=128, rotated=128, neighbours=True, dtype="bf16"),
        # serving one user: a token for each of 8 beams, states taken from the beams' parents
        dict(name="step_one_user", task="step", rows=8, beams=8, q_heads=8, k_heads=8, key_width=64,
             value_width=64, dtype="bf16"),
        # serving many users: one new rating each, states of 0.5 GB
        dict(name="step_many_users", task="step", rows=4_096, beams=0, q_heads=8, k_heads=8,
             key_width=64, value_width=64, dtype="bf16"),
        # reading in the longest history (a user who rated a tenth of the catalogue)
        dict(name="prefill_long_bf16", task="attend", train=False, users=1, tokens=62_496,
             law="even", resumed=False, q_heads=8, k_heads=8, key_width=64, value_width=64,
             dtype="bf16"),
        # the small set's histories at odd widths, resumed from stored states, shared key heads
        dict(name="prefill_odd_f32", task="attend", train=False, users=2_000, tokens=50_000,
             law="lognormal", resumed=True, q_heads=4, k_heads=2, key_width=33, value_width=50,
             dtype="f32"),
        # a training batch of 4096 users with histories of the full-size set's lengths
        dict(name="train_ragged_bf16", task="attend", train=True, users=4_096, tokens=1_075_431,
             law="lognormal", resumed=False, q_heads=8, k_heads=8, key_width=64, value_width=64,
             dtype="bf16"),
        # training in 32 bits at the widest heads, four query heads to a key head
        dict(name="train_shared_f32_w128", task="attend", train=True, users=100, tokens=100_003,
             law="lognormal", resumed=False, q_heads=8, k_heads=2, key_width=128, value_width=128,
             dtype="f32"),
        # one list from the small catalogue; latency
        dict(name="beam_small_f32", task="beam", lists=1, beams=4, items=1_000, finished=0.0,
             state=2 * 32 * 32, dtype="f32"),
        # 32 users' lists from the ordinary catalogue, with their states of 8 heads
        dict(name="beam_mid_bf16", task="beam", lists=32, beams=8, items=50_000, finished=0.1,
             state=8 * 64 * 64, dtype="bf16"),
        # wide beams over the full-size catalogue
        dict(name="beam_full_f32", task="beam", lists=8, beams=16, items=624_961, finished=0.1,
             state=8 * 64 * 64, dtype="f32"),
    ]


def draw(rng):
    def log_int(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))

    def width():
        return rng.choice([64, 128, rng.randint(8, 128), 8 * rng.randint(2, 16)])

    def heads():
        k = rng.choice([1, 2, 4, 8])
        return k * rng.choice([1, 1, 2, 4]), k

    task = rng.choice(["rotate", "attend", "attend", "step", "beam"])
    dtype = rng.choice(["f32", "bf16"])
    size = 4 if dtype == "f32" else 2
    if task == "rotate":
        q, k = heads()
        w = width()
        most = max(100, min(1_000_000, int(2.5e9 / ((q + k) * w * size))))
        return dict(task=task, train=rng.random() < 0.6, tokens=log_int(1, most), q_heads=q,
                    k_heads=k, width=w, rotated=2 * rng.randint(max(1, w // 4), w // 2),
                    neighbours=rng.random() < 0.5, dtype=dtype)
    if task == "step":
        q, k = heads()
        a, b = width(), width()
        beams = rng.choice([0, 0, 4, 8])
        rows = log_int(1, max(16, min(4_096, int(5e8 / (q * a * b * 4)))))
        return dict(task=task, rows=max(1, rows // beams) * beams if beams else rows, beams=beams,
                    q_heads=q, k_heads=k, key_width=a, value_width=b, dtype=dtype)
    if task == "attend":
        q, k = heads()
        a, b = width(), width()
        most = max(2_000, min(1_000_000, int(2.0e9 / (q * (a + b) * size)), int(1.5e10 / (q * a * b))))
        tokens = log_int(1_000, most)
        law = rng.choice(["even", "lognormal", "lognormal"])
        users = log_int(1, max(1, min(4_096, tokens // 8, int(1e9 / (q * a * b * 4)))))
        return dict(task=task, train=rng.random() < 0.5, users=users, tokens=tokens, law=law,
                    resumed=rng.random() < 0.3, q_heads=q, k_heads=k, key_width=a, value_width=b,
                    dtype=dtype)
    beams = rng.choice([1, 2, 4, 5, 8, 16])
    items = log_int(100, 624_961)
    return dict(task=task, lists=log_int(1, max(1, min(64, int(6e7 / (beams * items))))), beams=beams,
                items=items, finished=rng.choice([0.0, 0.2]), state=log_int(256, 8 * 64 * 64),
                dtype=dtype)


# ---- inputs --------------------------------------------------------------------------------

def _lengths(case, rng):
    """Tokens of each user (host): about even, or lognormal around half the mean with some users
    without a rating, as in the library's full-size sets."""
    B, N = case["users"], case["tokens"]
    if case["law"] == "even":
        share = np.full(B, 1.0 / B)
    else:
        share = np.exp(math.sqrt(2.0 * math.log(2.0)) * rng.standard_normal(B))
        share[rng.random(B) < 0.02] = 0.0
        share = share / share.sum() if share.sum() > 0 else np.full(B, 1.0 / B)
    ends = np.floor(np.cumsum(share) * N + 0.5).astype(np.int64)
    ends[-1] = N
    return np.diff(np.concatenate([[0], np.minimum(ends, N)]))


def _log_decay(heads, rng):
    """One decay for each head, windows from about 2 to 1000 tokens."""
    half = 1.0 + 9.0 * (np.arange(heads) + rng.random(heads)) / heads
    return torch.from_numpy(np.log1p(-np.exp2(-half)).astype(np.float32)).to(DEV)


def _tables(rotated):
    """Cosines and sines [TIME_BINS, rotated / 2] of the time bins."""
    step = 10_000.0 ** (-np.arange(rotated // 2) * 2.0 / rotated)
    angle = np.arange(TIME_BINS)[:, None] * step
    return [torch.from_numpy(f(angle).astype(np.float32)).to(DEV) for f in (np.cos, np.sin)]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    rng = np.random.default_rng(seed)
    dtype = DTYPES[case["dtype"]]

    def normal(*shape, dtype=dtype):
        return torch.randn(shape, generator=gen, device=DEV).to(dtype)

    s = dict(case=case, task=case["task"])
    if s["task"] == "rotate":
        N, q, k, D = case["tokens"], case["q_heads"], case["k_heads"], case["width"]
        # queries and keys are views of one projection's rows, as a model has them
        both = normal(N, q + k, D)
        s.update(q=both[:, :q], k=both[:, q:], q_weight=1.0 + 0.1 * normal(D, dtype=torch.float32),
                 k_weight=1.0 + 0.1 * normal(D, dtype=torch.float32),
                 positions=torch.randint(0, TIME_BINS, (N,), generator=gen, device=DEV,
                                         dtype=torch.int32).sort().values)
        s["cos"], s["sin"] = _tables(case["rotated"])
        if case["train"]:
            s.update(dq=normal(N, q, D), dk=normal(N, k, D))
        return s
    if s["task"] == "beam":
        B, W, V = case["lists"], case["beams"], case["items"]
        logits = torch.randn((B, W, V), generator=gen, device=DEV) * 4.0
        # items that the user has already rated are masked
        logits.masked_fill_(torch.rand((B, 1, V), generator=gen, device=DEV) < 0.002, -math.inf)
        s.update(logits=logits.to(dtype),
                 scores=-10.0 - 4.0 * torch.rand((B, W), generator=gen, device=DEV),
                 finished=torch.rand((B, W), generator=gen, device=DEV) < case["finished"],
                 states=normal(B, W, case["state"], dtype=torch.float32),
                 states_out=torch.empty((B, W, case["state"]), device=DEV))
        return s
    q, k, a, b = case["q_heads"], case["k_heads"], case["key_width"], case["value_width"]
    N = case["rows"] if s["task"] == "step" else case["tokens"]
    s.update(q=normal(N, q, a), k=normal(N, k, a), v=normal(N, k, b), scale=a ** -0.5,
             log_decay=_log_decay(q, rng))
    if s["task"] == "step":
        s["state"] = normal(N, q, a, b, dtype=torch.float32)
        s["state_out"] = torch.empty_like(s["state"])
        s["source"] = None
        if case["beams"]:  # the row that each row's state comes from: a beam of the same user
            W = case["beams"]
            parent = torch.randint(0, W, (N,), generator=gen, device=DEV, dtype=torch.int32)
            s["source"] = torch.arange(N, device=DEV, dtype=torch.int32) // W * W + parent
        return s
    lens = _lengths(case, rng)
    s["lens"] = lens
    s["row_ptr"] = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)])).to(DEV)
    s["initial"] = normal(case["users"], q, a, b, dtype=torch.float32) if case["resumed"] else None
    if case["train"]:
        s["do"] = normal(N, q, b)
        s["dstate"] = normal(case["users"], q, a, b, dtype=torch.float32) if case["resumed"] else None
    return s


# ---- the plain forms -------------------------------------------------------------------------

def _pairs(x, half, neighbours):
    return (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if neighbours \
        else (x[..., :half], x[..., half:2 * half])


def _joined(a, b, rest, neighbours):
    both = torch.stack([a, b], -1).flatten(-2) if neighbours else torch.cat([a, b], -1)
    return torch.cat([both, rest], -1)


def _plain_rotate(x, weight, cos, sin, neighbours):
    half = cos.shape[-1]
    x = x.float()
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight
    a, b = _pairs(y, half, neighbours)
    return _joined(a * cos - b * sin, b * cos + a * sin, y[..., 2 * half:], neighbours)


def _plain_rotate_backward(dy, x, weight, cos, sin, neighbours):
    half = cos.shape[-1]
    x, dy = x.float(), dy.float()
    a, b = _pairs(dy, half, neighbours)
    g = _joined(a * cos + b * sin, b * cos - a * sin, dy[..., 2 * half:], neighbours)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = x * r
    dweight = (g * n).sum((0, 1))
    g = g * weight
    return r * (g - n * (g * n).mean(-1, keepdim=True)), dweight


def _plain_attend(q, k, v, log_decay, row_ptr, chunks, most, initial, out_off=1, end_off=0):
    """o_t = sum over s <= t of e^(a (t - s)) (q_t . k_s) v_s, plus e^(a (t + out_off)) q_t S_0, in
    chunks; and the state after each user's last token, sum of e^(a (L - 1 - s + end_off)) k_s v_s^T
    plus e^(a L) S_0. ``chunks``: their number, ``most``: of one user at most."""
    token_count, heads = q.shape[:2]
    C = CHUNK
    lens = row_ptr[1:] - row_ptr[:-1]
    per = (lens + C - 1) // C
    ends = torch.cumsum(per, 0)
    user = torch.repeat_interleave(torch.arange(lens.numel(), device=DEV), per, output_size=chunks)
    nth = torch.arange(chunks, device=DEV) - (ends - per)[user]
    size = (lens[user] - nth * C).clamp_(max=C)
    at = torch.arange(C, device=DEV)
    live = at < size[:, None]
    token = (row_ptr[user] + nth * C)[:, None] + at * live
    def cut(x):  # [chunks, heads, C, width], nothing past a user's end
        x = (x.float()[token] * live[:, :, None, None]).transpose(1, 2)
        return x.repeat_interleave(heads // x.shape[1], 1) if x.shape[1] < heads else x

    q, k, v = cut(q), cut(k), cut(v)
    a = log_decay[:, None, None]
    gap = (at[:, None] - at[None, :]).float()
    weight = torch.where(gap >= 0, torch.exp(a * gap.clamp(min=0)), 0.0)
    o = torch.matmul(torch.matmul(q, k.transpose(2, 3)) * weight, v)
    left = (size[:, None] - 1 - at).clamp(min=0).float()  # tokens after each in its chunk
    k = k * torch.exp(log_decay[:, None] * (left + end_off)[:, None, :])[..., None]
    state = torch.matmul(k.transpose(2, 3), v)  # of the chunk alone
    whole = torch.exp(log_decay * size[:, None].float())[..., None, None]
    first = nth == 0
    if initial is not None:
        state = state + torch.where(first[:, None, None, None], whole * initial[user], 0.0)
    step = 1
    while step < most:  # doubling: each chunk adds the one `step` before it, with its decay
        joins = (nth >= step)[step:, None, None, None]
        decay = whole[step:] * torch.exp(log_decay * float(C * (step - 1)))[:, None, None]
        state = torch.cat([state[:step], state[step:] + torch.where(joins, decay * state[:-step], 0.0)])
        step *= 2
    before = torch.cat([torch.zeros_like(state[:1]), state[:-1]])
    at_first = torch.zeros((), device=DEV) if initial is None else initial[user]
    before = torch.where(first[:, None, None, None], at_first, before)
    o = o + torch.exp(log_decay[:, None] * (at + out_off).float())[..., None] * torch.matmul(q, before)
    target = torch.where(live, token, token_count).flatten()  # what lies past a user's end goes to a row of its own
    out = torch.empty((token_count + 1, heads, v.shape[-1]), device=DEV)
    out[target] = o.transpose(1, 2).flatten(0, 1)
    last = torch.where((lens > 0)[:, None, None, None], state[(ends - 1).clamp(min=0)],
                       0.0 if initial is None else initial)
    return out[:token_count], last


def _plain_attend_backward(do, q, k, v, log_decay, row_ptr, chunks, most, initial, dstate, scale):
    """Each gradient is a pass of the same form: dq runs on do, v, k, and dv and dk run from the
    last token to the first on k, q, do and v, do, q."""
    group = q.shape[1] // k.shape[1]
    wide = lambda x: x.float().repeat_interleave(group, 1)  # noqa: E731
    turned = lambda x: x.flip(0)  # noqa: E731
    plan = (log_decay, row_ptr, chunks, most)
    back = (log_decay, turned(row_ptr[-1] - row_ptr), chunks, most)
    do, k, v = do.float() * scale, wide(k), wide(v)
    dq, _ = _plain_attend(do, v, k, *plan, None if initial is None else initial.transpose(2, 3))
    end = None if dstate is None else turned(dstate)
    dv, dinitial = _plain_attend(turned(k), turned(q), turned(do), *back, end, 0, 1)
    dk, _ = _plain_attend(turned(v), turned(do), turned(q), *back,
                          None if end is None else end.transpose(2, 3), 0, 1)
    shared = lambda x: turned(x).unflatten(1, (-1, group)).sum(2)  # noqa: E731
    return dq, shared(dk), shared(dv), None if initial is None else turned(dinitial)


def _plain(s):
    case, dtype = s["case"], DTYPES[s["case"]["dtype"]]
    if s["task"] == "rotate":
        cos, sin = (t[s["positions"].long()][:, None] for t in (s["cos"], s["sin"]))
        rest = (cos, sin, case["neighbours"])
        out = [_plain_rotate(s[x], s[x + "_weight"], *rest).to(dtype) for x in "qk"]
        if case["train"]:
            for x in "qk":
                dx, dw = _plain_rotate_backward(s["d" + x], s[x], s[x + "_weight"], *rest)
                out += [dx.to(dtype), dw]
        return out
    if s["task"] == "step":
        group = case["q_heads"] // case["k_heads"]
        k, v = (s[x].float().repeat_interleave(group, 1) for x in "kv")
        state = s["state"] if s["source"] is None else s["state"][s["source"].long()]
        state = torch.exp(s["log_decay"])[:, None, None] * state + k[..., None] * v[:, :, None]
        o = torch.matmul(s["q"].float()[:, :, None], state)[:, :, 0] * s["scale"]
        return [o.to(dtype), state]
    if s["task"] == "attend":
        chunks, most = int((-(-s["lens"] // CHUNK)).sum()), int(-(-s["lens"].max() // CHUNK))
        plan = (s["log_decay"], s["row_ptr"], chunks, most)
        o, state = _plain_attend(s["q"].float() * s["scale"], s["k"], s["v"], *plan, s["initial"])
        out = [o.to(dtype), state]
        if case["train"]:
            grads = _plain_attend_backward(s["do"], s["q"], s["k"], s["v"], *plan, s["initial"],
                                           s["dstate"], s["scale"])
            out += [g.to(dtype) for g in grads[:3]] + ([] if grads[3] is None else [grads[3]])
        return out
    # beam: a beam that is finished goes on with the end item alone, at its own score
    x = s["logits"].float()
    x = torch.where(torch.isnan(x), -math.inf, x)
    B, W, V = x.shape
    top = x.amax(-1, keepdim=True)
    x = x - torch.where(torch.isinf(top), 0.0, top)
    x = x - torch.log(torch.exp(x).sum(-1, keepdim=True))
    is_end = (torch.arange(V, device=DEV) == END).expand(B, W, V)
    x = torch.where(s["finished"][..., None], torch.where(is_end, 0.0, -math.inf), x)
    x = (x + s["scores"][..., None] + 0.0).view(B, W * V)
    # one whole number orders score first, then the lowest place among equal scores
    bits = x.view(torch.int32)
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * 2 ** 32
    key = key + (2 ** 32 - 1 - torch.arange(W * V, device=DEV))
    place = 2 ** 32 - 1 - (key.topk(W, -1).values & (2 ** 32 - 1))
    scores = x.gather(1, place)
    none = scores == -math.inf
    parents = torch.where(none, 0, torch.div(place, V, rounding_mode="floor"))
    tokens = torch.where(none, -1, place % V)
    finished = s["finished"].gather(1, parents) | (tokens == END)
    states = s["states"].gather(1, parents[..., None].expand(-1, -1, s["states"].shape[-1]))
    return [parents.int(), tokens.int(), scores, finished & ~none, states]


# ---- the library's operators -------------------------------------------------------------------

@functools.cache
def _library():
    from paper_1108_2580_amd import sequence

    return sequence


def _own(s):
    lib, case = _library(), s["case"]
    if s["task"] == "rotate":
        args = (s["q"], s["k"], s["q_weight"], s["k_weight"], s["cos"], s["sin"], s["positions"])
        more = dict(eps=EPS, neighbours=case["neighbours"])
        out = list(lib.norm_rotate(*args, **more))
        if case["train"]:
            dq, dk, dqw, dkw = lib.norm_rotate_backward(s["dq"], s["dk"], *args, **more)
            out += [dq, dqw, dk, dkw]
        return out
    if s["task"] == "step":
        return list(lib.decay_attention_step(s["q"], s["k"], s["v"], s["log_decay"], s["state"],
                                             scale=s["scale"], source=s["source"],
                                             state_out=s["state_out"]))
    if s["task"] == "attend":
        args = (s["q"], s["k"], s["v"], s["log_decay"], s["row_ptr"])
        more = dict(scale=s["scale"], initial_state=s["initial"])
        out = list(lib.decay_attention(*args, return_state=True, **more))
        if case["train"]:
            grads = lib.decay_attention_backward(s["do"], *args, dstate=s["dstate"], **more)
            out += [g for g in grads if g is not None]
        return out
    parents, tokens, scores, finished = lib.beam_select(s["logits"], s["scores"], s["finished"], END)
    states = lib.reorder_states(s["states"], parents, out=s["states_out"])
    return [parents, tokens, scores, finished, states]


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["task"] == "rotate":
        heads, N, D = case["q_heads"] + case["k_heads"], case["tokens"], case["width"]
        table = 4 * min(N, TIME_BINS) * case["rotated"]
        units = 5 if case["train"] else 2  # x, y; dy, x, dx
        flops = (20 if case["train"] else 6) * N * heads * D
        return {"bytes": units * N * heads * D * size + 4 * N + table, "flops": flops}
    if case["task"] == "beam":
        rows = case["lists"] * case["beams"]
        read = rows * (1.0 - case["finished"])
        return {"bytes": read * case["items"] * size + 8 * rows * case["state"] + 20 * rows,
                "flops": 4 * read * case["items"]}
    q, k, a, b = case["q_heads"], case["k_heads"], case["key_width"], case["value_width"]
    N = case["rows"] if case["task"] == "step" else case["tokens"]
    qkv, o = (q * a + k * (a + b)) * size, q * b * size
    if case["task"] == "step":
        return {"bytes": N * (qkv + o) + 8 * N * q * a * b, "flops": 5 * N * q * a * b}
    states = (2 if case["resumed"] else 1) * 4 * case["users"] * q * a * b
    if case["train"]:  # forward; then q, k, v, do again and three gradients
        states += (3 if case["resumed"] else 0) * 4 * case["users"] * q * a * b
        return {"bytes": N * (3 * qkv + 2 * o) + states, "flops": 4 * 4 * N * q * a * b}
    return {"bytes": N * (qkv + o) + states, "flops": 4 * N * q * a * b}


# ---- the definitions in 64 bits ------------------------------------------------------------------

def _exact_rotate(s, x, dy):
    half, case = s["cos"].shape[1], s["case"]
    places = torch.arange(2 * half, device=DEV)
    one, two = (places[0::2], places[1::2]) if case["neighbours"] else (places[:half], places[half:])
    at = s["positions"].long()
    turn = torch.complex(s["cos"][at].double(), s["sin"][at].double())[:, None]

    def turned(y, by):
        z = torch.complex(y[..., one], y[..., two]) * by
        y = y.clone()
        y[..., one], y[..., two] = z.real, z.imag
        return y

    x, w = s[x].double(), s[x + "_weight"].double()
    size = torch.sqrt(x.square().mean(-1, keepdim=True) + EPS)
    y = turned(x / size * w, turn)
    if dy is None:
        return y, None, None
    g = turned(dy.double(), turn.conj())
    along = (g * w * x).mean(-1, keepdim=True)
    return y, g * w / size - x * along / size ** 3, torch.einsum("nhd,nhd->d", g, x / size)


def _exact_attend(s):
    """Token by token: the users go by descending length, so that those with a t-th token are the
    first ones."""
    case, lens = s["case"], s["lens"]
    H, group = case["q_heads"], case["q_heads"] // case["k_heads"]
    a, b = case["key_width"], case["value_width"]
    order = np.argsort(-lens, kind="stable")
    length = lens[order]
    most = int(length[0])
    passes = 2 if case["train"] else 1
    if passes * (most * 1e-4 + 6 * 8 * case["tokens"] * H * a * b / 3e12) > 15.0:
        return None
    active = np.searchsorted(-length, -np.arange(most), side="left")  # users longer than t
    first = s["row_ptr"][:-1][torch.from_numpy(order).to(DEV)]
    order = torch.from_numpy(order).to(DEV)
    q = s["q"].double() * s["scale"]
    k, v = (torch.repeat_interleave(s[x].double(), group, 1) for x in "kv")
    decay = torch.exp(s["log_decay"].double())[:, None, None]

    def start(x):
        return torch.zeros((lens.size, H, a, b), device=DEV, dtype=torch.float64) if x is None             else x.double()[order]

    def by_user(x):
        y = torch.empty_like(x)
        y[order] = x
        return y

    do = s["do"].double() * s["scale"] if case["train"] else None
    o, dq = torch.empty((q.shape[0], H, b), device=DEV, dtype=torch.float64), torch.empty_like(q)
    S = start(s["initial"])
    for t in range(most):
        n = int(active[t])
        at = first[:n] + t
        S[:n] = S[:n] * decay + k[at][..., None] * v[at][:, :, None]
        o[at] = torch.matmul(q[at][:, :, None], S[:n])[:, :, 0]
        if do is not None:
            dq[at] = torch.matmul(S[:n], do[at][..., None])[..., 0]
    out = [o, by_user(S)]
    if do is None:
        return out
    dk, dv = torch.empty_like(k), torch.empty_like(v)
    dS = start(s["dstate"])  # of the state after the token at hand
    for t in range(most - 1, -1, -1):
        n = int(active[t])
        at = first[:n] + t
        # q holds the scale here
        dS[:n] += q[at][..., None] * (do[at] / s["scale"])[:, :, None]
        dk[at] = torch.matmul(dS[:n], v[at][..., None])[..., 0]
        dv[at] = torch.matmul(k[at][:, :, None], dS[:n])[:, :, 0]
        dS[:n] *= decay
    shared = lambda x: x.unflatten(1, (-1, group)).sum(2)  # noqa: E731
    return out + [dq, shared(dk), shared(dv)] + ([by_user(dS)] if s["initial"] is not None else [])


def exact(case, seed):
    s = prepare(case, seed)
    if s["task"] == "rotate":
        y, grads = [], []
        for x in "qk":
            out, dx, dw = _exact_rotate(s, x, s.get("d" + x))
            y.append(out)
            grads += [] if dx is None else [dx, dw]
        return y + grads
    if s["task"] == "step":
        group = case["q_heads"] // case["k_heads"]
        state = s["state"].double()
        if s["source"] is not None:
            state = state[s["source"].long()]
        k, v = (torch.repeat_interleave(s[x].double(), group, 1) for x in "kv")
        decay = torch.exp(s["log_decay"].double())
        state = torch.einsum("h,nhab->nhab", decay, state) + torch.einsum("nha,nhb->nhab", k, v)
        return [torch.einsum("nha,nhab->nhb", s["q"].double(), state) * s["scale"], state]
    if s["task"] == "attend":
        return _exact_attend(s)
    scores = []
    for logits, score, finished in zip(s["logits"], s["scores"], s["finished"]):
        p = torch.log_softmax(logits.double(), -1) + score.double()[:, None]
        p[finished] = -math.inf
        p[finished, END] = score.double()[finished]
        scores.append(p.flatten().topk(case["beams"]).values)
    return [None, None, torch.stack(scores), None, None]

"""Sequence operators of libals (include/als.h): the parts of a next-item model.

A next-item model reads a user's ratings in the order of time and answers with lists of items:
``norm_rotate`` prepares queries and keys, ``decay_attention`` runs over the histories
(``decay_attention_step`` over one new rating), ``beam_select`` extends the lists and
``reorder_states`` moves the beams' states along. Histories are packed one after the other, with a
``row_ptr`` like the rating matrix's.

Argument marshalling only: the work runs in the HIP kernels of ``csrc/``. Every call is enqueued on
the current HIP stream of the current device, on which its tensors have to lie, and nothing is
synchronised. Inputs are fp32 or bf16 tensors whose features are contiguous; tokens and heads may
have any strides (tokens of ``decay_attention`` up to 2^22 values). Where an input of ``norm_rotate`` or
``decay_attention`` requires a gradient, the result carries it, or the call raises where there is none
for that input (``cos``, ``sin``, ``log_decay``). The other operators' results carry none. What a call
writes to a caller's tensor counts as an in-place operation.
"""
from __future__ import annotations

import ctypes
import math

import torch

from . import ALS_ERR_INVALID_ARG, ALS_OK, ALSError, lib

ALS_F32, ALS_BF16 = 0, 1
_DTYPES = {torch.float32: ALS_F32, torch.bfloat16: ALS_BF16}
MAX_BEAMS = 32

_P, _i64, _i32, _f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float


class _Heads(ctypes.Structure):
    _fields_ = [("data", _P), ("token_stride", _i64), ("head_stride", _i64)]


class _Rotation(ctypes.Structure):
    _fields_ = [("n_tokens", _i64), ("n_positions", _i64), ("q_heads", _i32), ("k_heads", _i32),
                ("width", _i32), ("rotated", _i32), ("neighbours", _i32), ("eps", _f32),
                ("positions", _P), ("cos_table", _P), ("sin_table", _P)]


class _Attention(ctypes.Structure):
    _fields_ = [("n_tokens", _i64), ("n_rows", _i64), ("row_ptr", _P), ("log_decay", _P),
                ("q_heads", _i32), ("k_heads", _i32), ("k_width", _i32), ("v_width", _i32),
                ("scale", _f32)]


class _Beams(ctypes.Structure):
    _fields_ = [("n_lists", _i64), ("n_items", _i64), ("row_stride", _i64), ("beams", _i32),
                ("width", _i32), ("end_token", _i32)]


def _declare():
    R, A, B = (ctypes.POINTER(t) for t in (_Rotation, _Attention, _Beams))
    H, st = _Heads, ctypes.c_int
    for name, args in (
            ("als_norm_rotate", [R, st, H, H, _P, _P, H, H, _P]),
            ("als_norm_rotate_backward",
             [R, st, H, H, H, H, _P, _P, H, H, _P, _P, _P, _i64, _P]),
            ("als_decay_attention", [A, st, H, H, H, _P, _P, _P, _P, _i64, _P]),
            ("als_decay_attention_backward",
             [A, st, H, H, H, H, _P, _P, _P, _P, _P, _P, _P, _i64, _P]),
            ("als_decay_attention_step", [A, st, H, H, H, _P, _i64, _P, _P, _P, _P]),
            ("als_beam_select", [B, st, _P, _P, _P, _P, _P, _P, _P, _P, _i64, _P]),
            ("als_reorder_states", [_i64, _i32, _i32, _i64, _P, _P, _P, _P])):
        f = getattr(lib, name)
        f.argtypes, f.restype = args, st
    for name, arg in (("als_norm_rotate_workspace", R), ("als_decay_attention_workspace", A),
                      ("als_decay_attention_backward_workspace", A),
                      ("als_beam_select_workspace", B)):
        f = getattr(lib, name)
        f.argtypes, f.restype = [arg], _i64


_declare()


def _check(status):
    if status != ALS_OK:
        raise ALSError(status, lib.als_last_error(None).decode())


# A token's calls are bound by the host: the current device and the current stream's handle by
# themselves take a fifth of the time of what torch.cuda has around them.
_raw_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(device):
    return _raw_stream(device) if _raw_stream else torch.cuda.current_stream(device).cuda_stream


def _device(t, name):
    """The current device's index, on which t has to lie."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    device = _raw_device()
    if t.get_device() != device:
        raise ValueError(f"{name} is on {t.device}, not on the current device")
    return device


def _array(t, name, dtype, shape, device):
    """A contiguous tensor of this type and shape, as a pointer."""
    if not isinstance(t, torch.Tensor) or t.get_device() != device or t.dtype != dtype or \
            not t.is_contiguous() or t.shape != shape:
        _device(t, name)
        if t.dtype != dtype or not t.is_contiguous():
            raise TypeError(f"{name} must be contiguous {dtype}")
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    return t.data_ptr()


def _heads(t, name, dtype, device):
    """A [tokens, heads, width] tensor with contiguous features."""
    if not isinstance(t, torch.Tensor) or t.get_device() != device:
        _device(t, name)
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    stride = t.stride()
    if len(stride) != 3:
        raise ValueError(f"{name} must have the dimensions tokens, heads, width")
    if stride[2] != 1 and t.shape[2] > 1:
        raise TypeError(f"the features of {name} must be contiguous")
    return _Heads(t.data_ptr(), stride[0], stride[1])


def _dtype(t, name):
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32 or bfloat16, not {t.dtype}")
    return code


def _shaped(t, name, shape):
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")


def _workspace(size, device):
    return torch.empty(size, dtype=torch.uint8, device=device) if size > 0 else None


def _ptr(t):
    return None if t is None else t.data_ptr()


def _no_gradient(t, name):
    if isinstance(t, torch.Tensor) and t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} takes no gradient")


def _writable(t, name):
    """Refuses a caller's tensor whose gradient a write by a kernel would lose unseen."""
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient, which writing to it would lose")


def _written(t):
    """As after torch's in-place operations, a graph that has saved the tensor notices."""
    if not t.is_inference():
        torch.autograd.graph.increment_version(t)


# ---- norm and rotation -------------------------------------------------------------------------

def rotary_tables(n_positions, rotated, base=10_000.0, device="cuda"):
    """(cos, sin) fp32 tables [n_positions, rotated / 2] of the angles position * base^(-2 p /
    rotated), formed in fp64."""
    pair = torch.arange(rotated // 2, dtype=torch.float64)
    angle = torch.arange(n_positions, dtype=torch.float64)[:, None] * base ** (-2.0 * pair / max(rotated, 1))
    return angle.cos().float().to(device), angle.sin().float().to(device)


def _rotation(q, k, q_weight, k_weight, cos, sin, positions, eps, neighbours):
    dev = _device(q, "q")
    code = _dtype(q, "q")
    hq, hk = _heads(q, "q", q.dtype, dev), _heads(k, "k", q.dtype, dev)
    N, Hq, D = q.shape
    Hk = k.shape[1]
    _shaped(k, "k", (N, Hk, D))
    if not isinstance(cos, torch.Tensor) or cos.dim() != 2:
        raise ValueError("cos must have the dimensions positions, pairs")
    P, half = cos.shape
    f32 = torch.float32
    shape = _Rotation(N, P, Hq, Hk, D, 2 * half, 1 if neighbours else 0, eps,
                      _array(positions, "positions", torch.int32, (N,), dev),
                      _array(cos, "cos", f32, (P, half), dev), _array(sin, "sin", f32, (P, half), dev))
    return dev, code, shape, hq, hk, _array(q_weight, "q_weight", f32, (D,), dev), \
        _array(k_weight, "k_weight", f32, (D,), dev)


def _packed(t):
    """A new tensor like t, tokens one after the other, and its strides."""
    _, H, D = t.shape
    out = t.new_empty(t.shape)
    return out, _Heads(out.data_ptr(), H * D, D)


def _norm_rotate(q, k, q_weight, k_weight, cos, sin, positions, eps, neighbours):
    dev, code, shape, hq, hk, wq, wk = _rotation(q, k, q_weight, k_weight, cos, sin, positions, eps,
                                                 neighbours)
    q_out, ho = _packed(q)
    k_out, ko = _packed(k)
    _check(lib.als_norm_rotate(shape, code, hq, hk, wq, wk, ho, ko, _stream(dev)))
    return q_out, k_out


def norm_rotate(q, k, q_weight, k_weight, cos, sin, positions, eps=1e-6, neighbours=False):
    """Norm of queries [tokens, heads, width] and keys [tokens, key heads, width] for each head, and
    the rotation by position: y = x / sqrt(mean x^2 + eps) * weight, then the first 2 * cos.shape[1]
    features turned in pairs by the angle of the token's position.

    ``q_weight``, ``k_weight``: fp32 [width]; ``cos``, ``sin``: fp32 [positions, pairs]
    (``rotary_tables``); ``positions``: int32 [tokens], a row of the tables each (one outside them
    makes its token NaN). ``neighbours``: pair p is features 2 p and 2 p + 1 instead of p and
    p + pairs. Returns new (q, k). ``cos`` and ``sin`` take no gradient."""
    _no_gradient(cos, "cos")
    _no_gradient(sin, "sin")
    if torch.is_grad_enabled() and (
            q.requires_grad or k.requires_grad or q_weight.requires_grad or k_weight.requires_grad):
        return _NormRotate.apply(q, k, q_weight, k_weight, cos, sin, positions, eps, neighbours)
    return _norm_rotate(q, k, q_weight, k_weight, cos, sin, positions, eps, neighbours)


def norm_rotate_backward(dq, dk, q, k, q_weight, k_weight, cos, sin, positions, eps=1e-6,
                         neighbours=False):
    """Gradients of ``norm_rotate``'s inputs (dq, dk, dq_weight, dk_weight) from those of its
    outputs."""
    dev, code, shape, hq, hk, wq, wk = _rotation(q, k, q_weight, k_weight, cos, sin, positions, eps,
                                                 neighbours)
    hdq, hdk = _heads(dq, "dq", q.dtype, dev), _heads(dk, "dk", q.dtype, dev)
    _shaped(dq, "dq", q.shape)
    _shaped(dk, "dk", k.shape)
    q_out, ho = _packed(q)
    k_out, ko = _packed(k)
    dwq, dwk = torch.empty_like(q_weight), torch.empty_like(k_weight)
    size = lib.als_norm_rotate_workspace(shape)
    work = _workspace(size, q.device)
    _check(lib.als_norm_rotate_backward(shape, code, hdq, hdk, hq, hk, wq, wk, ho, ko,
                                        dwq.data_ptr(), dwk.data_ptr(), _ptr(work), size,
                                        _stream(dev)))
    return q_out, k_out, dwq, dwk


MAX_TOKEN_STRIDE = 1 << 22  # of decay_attention


def _dense(t):
    """A gradient, which has the strides that its graph gives it, as the operators take it."""
    fits = (t.stride(-1) == 1 or t.shape[-1] == 1) and t.stride(0) <= MAX_TOKEN_STRIDE
    return t if fits else t.contiguous()


class _NormRotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, cos, sin, positions, eps, neighbours):
        ctx.save_for_backward(q, k, q_weight, k_weight, cos, sin, positions)
        ctx.more = (eps, neighbours)
        return _norm_rotate(q, k, q_weight, k_weight, cos, sin, positions, eps, neighbours)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dq, dk):
        return (*norm_rotate_backward(_dense(dq), _dense(dk), *ctx.saved_tensors, *ctx.more),
                None, None, None, None, None)


# ---- attention with a decay for each head --------------------------------------------------------

def _attention(q, k, v, log_decay, row_ptr, scale):
    dev = _device(q, "q")
    code = _dtype(q, "q")
    dtype = q.dtype
    hq, hk, hv = _heads(q, "q", dtype, dev), _heads(k, "k", dtype, dev), _heads(v, "v", dtype, dev)
    N, Hq, K = q.shape
    n, Hk, V = v.shape
    if n != N or k.shape != (N, Hk, K):
        raise ValueError(f"q, k and v have shapes {tuple(q.shape)}, {tuple(k.shape)} and "
                         f"{tuple(v.shape)}")
    rows = N
    if row_ptr is not None:
        if not isinstance(row_ptr, torch.Tensor) or row_ptr.dim() != 1 or row_ptr.numel() < 1:
            raise ValueError("row_ptr must have one more entry than there are rows")
        rows = row_ptr.numel() - 1
        row_ptr = _array(row_ptr, "row_ptr", torch.int64, (rows + 1,), dev)
    shape = _Attention(N, rows, row_ptr, _array(log_decay, "log_decay", torch.float32, (Hq,), dev), Hq,
                       Hk, K, V, K ** -0.5 if scale is None else scale)
    return dev, code, shape, hq, hk, hv


def _state_ptr(t, name, shape, dev):
    return None if t is None else _array(
        t, name, torch.float32, (shape.n_rows, shape.q_heads, shape.k_width, shape.v_width), dev)


def _new_state(shape, device):
    return torch.empty((shape.n_rows, shape.q_heads, shape.k_width, shape.v_width), device=device)


def _decay_attention(q, k, v, log_decay, row_ptr, scale, initial_state, return_state):
    dev, code, shape, hq, hk, hv = _attention(q, k, v, log_decay, row_ptr, scale)
    first = _state_ptr(initial_state, "initial_state", shape, dev)
    out = q.new_empty((q.shape[0], shape.q_heads, shape.v_width))
    state = _new_state(shape, q.device) if return_state else None
    size = lib.als_decay_attention_workspace(shape)
    work = _workspace(size, q.device)
    _check(lib.als_decay_attention(shape, code, hq, hk, hv, first, out.data_ptr(), _ptr(state),
                                   _ptr(work), size, _stream(dev)))
    return out, state


def decay_attention(q, k, v, log_decay, row_ptr, scale=None, initial_state=None,
                    return_state=False):
    """Linear attention with a decay for each head over packed rows of tokens: with
    S_t = exp(log_decay) S_{t-1} + k_t v_t^T, out_t = scale S_t^T q_t.

    ``q``: [tokens, heads, key width]; ``k``, ``v``: [tokens, key heads, width], each key head shared
    by heads / key heads query heads; widths up to 128. ``log_decay``: fp32 [heads], <= 0.
    ``row_ptr``: int64 [rows + 1] on the device, from 0 to the number of tokens, row b holding tokens
    row_ptr[b] .. row_ptr[b + 1] - 1; a token that no row holds (padding behind the last row) is not
    worked on, and its place in the new tensors, outputs and gradients, is left unset.
    ``scale``: 1 / sqrt(key width) if None. ``initial_state``: fp32 [rows, heads, key width, value
    width], zero if None. Returns out [tokens, heads, value width], with ``return_state`` (out, the
    states after the rows' last tokens). ``log_decay`` takes no gradient."""
    _no_gradient(log_decay, "log_decay")
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad
                                       for t in (q, k, v, initial_state)):
        out, state = _DecayAttention.apply(q, k, v, initial_state, log_decay, row_ptr, scale,
                                           return_state)
    else:
        out, state = _decay_attention(q, k, v, log_decay, row_ptr, scale, initial_state, return_state)
    return (out, state) if return_state else out


def decay_attention_backward(d_out, q, k, v, log_decay, row_ptr, scale=None, initial_state=None,
                             dstate=None, d_initial=None):
    """Gradients (dq, dk, dv, d_initial_state) of ``decay_attention`` from that of its output and,
    if given, of its returned state (``dstate``). The last is None unless there is an
    ``initial_state`` or ``d_initial`` is true."""
    dev, code, shape, hq, hk, hv = _attention(q, k, v, log_decay, row_ptr, scale)
    hdo = _heads(d_out, "d_out", q.dtype, dev)
    _shaped(d_out, "d_out", (q.shape[0], shape.q_heads, shape.v_width))
    first = _state_ptr(initial_state, "initial_state", shape, dev)
    last = _state_ptr(dstate, "dstate", shape, dev)
    dq, dk, dv = q.new_empty(q.shape), k.new_empty(k.shape), v.new_empty(v.shape)
    wanted = initial_state is not None if d_initial is None else d_initial
    dfirst = _new_state(shape, q.device) if wanted else None
    size = lib.als_decay_attention_backward_workspace(shape)
    work = _workspace(size, q.device)
    _check(lib.als_decay_attention_backward(shape, code, hdo, hq, hk, hv, first, last, dq.data_ptr(),
                                            dk.data_ptr(), dv.data_ptr(), _ptr(dfirst), _ptr(work),
                                            size, _stream(dev)))
    return dq, dk, dv, dfirst


class _DecayAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, initial_state, log_decay, row_ptr, scale, return_state):
        ctx.save_for_backward(q, k, v, log_decay, row_ptr, initial_state)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        return _decay_attention(q, k, v, log_decay, row_ptr, scale, initial_state, return_state)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_out, dstate):
        q, k, v, log_decay, row_ptr, initial_state = ctx.saved_tensors
        if d_out is None:
            d_out = torch.zeros((q.shape[0], q.shape[1], v.shape[2]), dtype=q.dtype, device=q.device)
        dstate = None if dstate is None else dstate.contiguous()
        grads = decay_attention_backward(_dense(d_out), q, k, v, log_decay, row_ptr, ctx.scale,
                                         initial_state, dstate, d_initial=ctx.needs_input_grad[3])
        return (*grads, None, None, None, None)


def decay_attention_step(q, k, v, log_decay, state, scale=None, source=None, state_out=None):
    """One token of each row: state_out = exp(log_decay) state[source] + k v^T, out = scale
    state_out^T q, for ``q``: [rows, heads, key width] and ``k``, ``v``: [rows, key heads, width].

    ``state``: fp32 [rows, heads, key width, value width], updated in place unless ``state_out`` is
    given. ``source``: int32 [rows], the row of ``state`` that each row goes on from (a beam's
    parent; one outside it gives NaN); ``state`` may then have another number of rows, and
    ``state_out`` (a new tensor if None) must not overlap it. Returns (out, state_out), neither of
    which carries a gradient; a ``state`` or ``state_out`` that requires one is written only under
    ``torch.no_grad()``."""
    dev, code, shape, hq, hk, hv = _attention(q, k, v, log_decay, None, scale)
    N, H, K, V = shape.n_rows, shape.q_heads, shape.k_width, shape.v_width
    sources, src = N, None
    if source is not None:
        _device(state, "state")
        sources = state.shape[0] if state.dim() else 0
        src = _array(source, "source", torch.int32, (N,), dev)
    sp = _array(state, "state", torch.float32, (sources, H, K, V), dev)
    if state_out is None:
        state_out = state if source is None else _new_state(shape, q.device)
    to = sp if state_out is state else _array(state_out, "state_out", torch.float32, (N, H, K, V), dev)
    _writable(state_out, "state" if state_out is state else "state_out")
    out = q.new_empty((N, H, V))
    _check(lib.als_decay_attention_step(shape, code, hq, hk, hv, sp, sources, src, to, out.data_ptr(),
                                        _stream(dev)))
    _written(state_out)
    return out, state_out


# ---- beams ---------------------------------------------------------------------------------------

def beam_select(logits, scores, finished=None, end_token=-1, width=None):
    """The best ``width`` (as many as there are beams if None) extensions of each list's beams.

    ``logits``: fp32 or bf16 [lists, beams, items] (-inf and NaN mask an item); ``scores``: fp32
    [lists, beams], -inf for a beam without candidates; ``finished``: bool or uint8 [lists, beams],
    beams that go on with ``end_token`` alone at their own score. A candidate scores its beam's score
    plus the log-softmax of its item; equal scores (in fp64) go by the lowest beam, then the largest
    logit, then the lowest item.
    Returns (parents int32, tokens int32, scores fp32, finished bool), each [lists, width] by
    descending score; where candidates run out: 0, -1, -inf and False. None carries a gradient."""
    dev = _device(logits, "logits")
    code = _dtype(logits, "logits")
    if logits.dim() != 3:
        raise ValueError("logits must have the dimensions lists, beams, items")
    B, W, V = logits.shape
    apart, stride, unit = logits.stride()
    if W == 1:
        stride = apart if B > 1 else V
    if (V > 1 and unit != 1) or (B > 1 and apart != W * stride):
        raise TypeError("logits must have contiguous items and evenly spaced rows")
    sp = _array(scores, "scores", torch.float32, (B, W), dev)
    fp = None
    if finished is not None:
        if isinstance(finished, torch.Tensor) and finished.dtype == torch.bool:
            fp = _array(finished, "finished", torch.bool, (B, W), dev)
        else:
            fp = _array(finished, "finished", torch.uint8, (B, W), dev)
    width = W if width is None else int(width)
    shape = _Beams(B, V, stride, W, width, end_token)
    size = lib.als_beam_select_workspace(shape)
    if size < 0:
        raise ALSError(ALS_ERR_INVALID_ARG, lib.als_last_error(None).decode())
    device = logits.device
    parents, tokens = torch.empty((2, B, width), dtype=torch.int32, device=device).unbind()
    new = torch.empty((B, width), device=device)
    done = torch.empty((B, width), dtype=torch.bool, device=device)
    work = _workspace(size, device)
    _check(lib.als_beam_select(shape, code, logits.data_ptr(), sp, fp, parents.data_ptr(),
                               tokens.data_ptr(), new.data_ptr(), done.data_ptr(), _ptr(work), size,
                               _stream(dev)))
    return parents, tokens, new, done


def reorder_states(states, parents, out=None):
    """The beams' states in their new order: out[b, w] = states[b, parents[b, w]] for ``states``
    [lists, beams, ...] of any type, contiguous, and ``parents`` int32 [lists, width]. ``out`` (a new
    tensor if None) may be ``states`` itself where width equals beams; one that requires a gradient is
    written only under ``torch.no_grad()``. A parent outside [0, beams) leaves its row of ``out`` as it is.
    The result carries no gradient."""
    dev = _device(states, "states")
    if states.dim() < 2 or not states.is_contiguous():
        raise TypeError("states must be contiguous with the dimensions lists, beams, ...")
    if not isinstance(parents, torch.Tensor) or parents.dim() != 2:
        raise ValueError("parents must have the dimensions lists, width")
    B, W, *rest = states.shape
    width = parents.shape[1]
    pp = _array(parents, "parents", torch.int32, (B, width), dev)
    shape = (B, width, *rest)
    if out is None:
        out = torch.empty(shape, dtype=states.dtype, device=states.device)
    else:
        _array(out, "out", states.dtype, shape, dev)
        _writable(out, "out")
    size = math.prod(rest) * states.element_size()
    _check(lib.als_reorder_states(B, W, width, size, states.data_ptr(), out.data_ptr(), pp,
                                  _stream(dev)))
    _written(out)
    return out

"""The sequence operators' refusals: arguments that the host can check are checked before any device
call, so these run without a GPU. Pointers are made up and never followed."""
import ctypes
import math

import pytest

import paper_1108_2580_amd as p
from paper_1108_2580_amd import lib, sequence
from paper_1108_2580_amd.sequence import _Attention, _Beams, _Heads, _Rotation

torch = pytest.importorskip("torch")

A, B, C, D, W = (0x10000000 * i for i in range(1, 6))  # buffers 256 MiB apart
INVALID = 1


def refused(status, word):
    msg = lib.als_last_error(None).decode()
    assert status == INVALID and word in msg, (status, msg)


def rotation(**kw):
    d = dict(n_tokens=10, n_positions=5, q_heads=4, k_heads=2, width=64, rotated=64, neighbours=0, eps=1e-6,
             positions=A, cos_table=A, sin_table=A)
    d.update(kw)
    return _Rotation(**d)


def norm_rotate(shape, dtype=0, q=None, k=None, wq=A, wk=A, qo=None, ko=None):
    return lib.als_norm_rotate(shape, dtype, q or _Heads(A, 256, 64), k or _Heads(B, 128, 64), wq, wk,
                               qo or _Heads(C, 256, 64), ko or _Heads(D, 128, 64), None)


@pytest.mark.parametrize("change,word", [
    (dict(n_tokens=-1), "n_tokens"), (dict(n_tokens=1 << 31), "n_tokens"), (dict(q_heads=0), "heads"),
    (dict(k_heads=1025), "heads"), (dict(width=0), "width"), (dict(width=257), "width"),
    (dict(rotated=3), "rotated"), (dict(rotated=66), "rotated"), (dict(neighbours=2), "neighbours"),
    (dict(eps=-1.0), "eps"), (dict(eps=math.nan), "eps"), (dict(n_positions=0), "n_positions"),
    (dict(positions=None), "positions"), (dict(sin_table=None), "table")])
def test_norm_rotate_shapes(change, word):
    refused(norm_rotate(rotation(**change)), word)


@pytest.mark.parametrize("change,word", [
    (dict(dtype=2), "dtype"), (dict(wq=None), "weight"), (dict(q=_Heads(None, 256, 64)), "NULL"),
    (dict(k=_Heads(B, -1, 64)), "stride"), (dict(q=_Heads(A + 2, 256, 64)), "aligned"),
    (dict(qo=_Heads(C, 100, 64)), "overlapping rows"), (dict(qo=_Heads(A + 256, 256, 64)), "in part"),
    (dict(ko=_Heads(C, 256, 64)), "the same"), (dict(ko=_Heads(C + 64, 128, 64)), "overlap")])
def test_norm_rotate_tensors(change, word):
    refused(norm_rotate(rotation(), **change), word)


@pytest.mark.parametrize("change", [
    dict(ko=_Heads(A, 128, 64)), dict(qo=_Heads(B, 256, 64)), dict(q=_Heads(A, 256, 64), k=_Heads(A, 128, 64),
                                                                   qo=_Heads(A, 256, 64))])
def test_norm_rotate_output_on_the_other_sides_input(change):
    refused(norm_rotate(rotation(), **change), "overlaps")


def test_norm_rotate_backward_workspace():
    s = rotation()
    need = lib.als_norm_rotate_workspace(s)
    assert need > 0 and lib.als_norm_rotate_workspace(rotation(width=0)) == -1
    q, k, qo, ko = _Heads(A, 256, 64), _Heads(B, 128, 64), _Heads(C, 256, 64), _Heads(D, 128, 64)
    back = lambda work, size, dw=B: lib.als_norm_rotate_backward(  # noqa: E731
        s, 0, q, k, q, k, A, A, qo, ko, dw, A, work, size, None)
    refused(back(W, need - 1), "workspace")
    refused(back(None, need), "workspace")
    refused(back(W + 8, need), "aligned")
    refused(back(W, need, None), "NULL")
    refused(back(W, need, A), "the same")


def attention(**kw):
    d = dict(n_tokens=5000, n_rows=3, row_ptr=A, log_decay=A, q_heads=4, k_heads=2, k_width=64, v_width=32,
             scale=0.125)
    d.update(kw)
    return _Attention(**d)


def forward(shape, dtype=0, q=None, k=None, v=None, first=None, out=C, last=None, work=W, size=1 << 40):
    return lib.als_decay_attention(shape, dtype, q or _Heads(A, 256, 64), k or _Heads(A, 128, 64),
                                   v or _Heads(B, 64, 32), first, out, last, work, size, None)


@pytest.mark.parametrize("change,word", [
    (dict(n_tokens=-1), "n_tokens"), (dict(n_rows=(1 << 30) + 1), "n_rows"), (dict(q_heads=3), "multiple"),
    (dict(k_heads=0), "multiple"), (dict(k_width=129), "k_width"), (dict(v_width=0), "v_width"),
    (dict(scale=math.inf), "scale"), (dict(log_decay=None), "log_decay"), (dict(row_ptr=None), "row_ptr"),
    (dict(n_rows=0), "without rows")])
def test_attention_shapes(change, word):
    refused(forward(attention(**change)), word)


@pytest.mark.parametrize("change,word", [
    (dict(dtype=-1), "dtype"), (dict(v=_Heads(None, 64, 32)), "NULL"), (dict(out=None), "out"),
    (dict(q=_Heads(A, (1 << 22) + 1, 64)), "token_stride"), (dict(k=_Heads(A, 1 << 50, 64)), "stride"),
    (dict(out=C + 1), "aligned"), (dict(out=A + 1024), "overlaps"), (dict(first=D, last=D + 64), "overlaps"),
    (dict(size=16), "workspace"), (dict(work=None), "workspace"), (dict(work=W + 4), "aligned")])
def test_attention_tensors(change, word):
    refused(forward(attention(), **change), word)


def test_attention_backward_and_step():
    s = attention()
    need = lib.als_decay_attention_backward_workspace(s)
    assert need > lib.als_decay_attention_workspace(s) > 0
    assert lib.als_decay_attention_workspace(attention(k_width=0)) == -1
    h = _Heads(A, 256, 64)
    back = lambda dq, dk, dv, size=need: lib.als_decay_attention_backward(  # noqa: E731
        s, 0, h, h, h, h, None, None, dq, dk, dv, None, W, size, None)
    refused(back(B, C, None), "NULL")
    refused(back(B, B + 4, D), "two gradients")
    refused(back(A + 4, C, D), "overlaps an input")
    refused(back(B, C, D, need - 1), "workspace")
    step = lambda state, n, source, to, out=D: lib.als_decay_attention_step(  # noqa: E731
        s, 0, h, h, h, state, n, source, to, out, None)
    refused(step(B, 4, None, C), "without source")
    refused(step(B, 3, A, B), "overlaps")           # with source never in place
    refused(step(B, 3, None, B + 64), "overlaps")
    refused(step(None, 3, None, C), "NULL")
    refused(step(B, 0, A, C), "without a state")
    refused(step(B, 3, None, C, A), "overlaps an input")
    refused(step(B, 3, None, C, B + 16), "overlaps a state")


def beams(**kw):
    d = dict(n_lists=2, n_items=100, row_stride=100, beams=4, width=4, end_token=-1)
    d.update(kw)
    return _Beams(**d)


@pytest.mark.parametrize("change,word", [
    (dict(n_lists=-1), "n_lists"), (dict(beams=33), "beams"), (dict(width=0), "width"),
    (dict(n_items=0), "n_items"), (dict(row_stride=99), "row_stride"), (dict(end_token=100), "end_token"),
    (dict(end_token=-2), "end_token")])
def test_beam_shapes(change, word):
    s = beams(**change)
    assert lib.als_beam_select_workspace(s) == -1
    refused(lib.als_beam_select(s, 0, A, B, None, C, C, C, C, W, 1 << 40, None), word)


def test_beam_tensors():
    need = lib.als_beam_select_workspace(beams())
    call = lambda s=beams(), dtype=0, x=A, done=None, to=C, work=W, size=need: lib.als_beam_select(  # noqa: E731
        s, dtype, x, B, done, C + 4096, C + 8192, to, D, work, size, None)
    refused(call(dtype=7), "dtype")
    refused(call(x=None), "NULL")
    refused(call(x=A + 2), "aligned")
    refused(call(done=A), "end_token")
    refused(call(to=B + 8), "overlaps an input")
    refused(call(to=C + 4096), "two outputs")
    refused(call(to=C + 2), "aligned")
    refused(call(size=need - 1), "workspace")
    refused(lib.als_reorder_states(2, 4, 4, 64, A, A + 64, B, None), "overlaps")
    refused(lib.als_reorder_states(2, 4, 5, 64, A, A, B, None), "overlaps")
    refused(lib.als_reorder_states(2, 40, 4, 64, A, B, C, None), "beams")
    refused(lib.als_reorder_states(2, 4, 4, -1, A, B, C, None), "row_bytes")
    refused(lib.als_reorder_states(2, 4, 4, 64, None, B, C, None), "NULL")


def test_binding_refuses_host_tensors():
    x = torch.zeros(4, 2, 8)
    w = torch.zeros(8)
    for call in (lambda: p.norm_rotate(x, x, w, w, x, x, x), lambda: p.decay_attention(x, x, x, w, w),
                 lambda: p.decay_attention_step(x, x, x, w, x), lambda: p.beam_select(x, w),
                 lambda: p.reorder_states(x, w)):
        with pytest.raises(TypeError, match="CUDA"):
            call()


def test_structures_match_the_header():
    """Sizes and offsets of the binding's structures against the compiler's, from the header."""
    import os
    import subprocess
    import tempfile

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = {"als_heads": _Heads, "als_rotation": _Rotation, "als_attention": _Attention, "als_beams": _Beams}
    lines = []
    for c, t in names.items():
        lines.append(f'printf("{c} %zu\\n", sizeof({c}));')
        lines += [f'printf("{c}.{f} %zu\\n", offsetof({c}, {f}));' for f, _ in t._fields_]
    src = '#include <stddef.h>\n#include <stdio.h>\n#include "als.h"\nint main(void) {' + "\n".join(lines) + "}"
    with tempfile.TemporaryDirectory() as d:
        open(os.path.join(d, "a.c"), "w").write(src)
        subprocess.check_call(["gcc", "-I", os.path.join(root, "include"), os.path.join(d, "a.c"), "-o",
                               os.path.join(d, "a")])
        said = dict(line.split() for line in subprocess.check_output([os.path.join(d, "a")], text=True).splitlines())
    for c, t in names.items():
        assert int(said[c]) == ctypes.sizeof(t)
        for f, _ in t._fields_:
            assert int(said[f"{c}.{f}"]) == getattr(t, f).offset
    assert sequence.MAX_BEAMS == 32


# ---- grids: launches of more threads than one HIP grid holds (2^32 - 1) go in slices ---------------

LAUNCH = """
import ctypes, sys
ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
sys.path.insert(0, sys.argv[2])
lib = ctypes.CDLL(sys.argv[3])
lib.als_last_error.restype = ctypes.c_char_p
class H(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("t", ctypes.c_int64), ("h", ctypes.c_int64)]
class S(ctypes.Structure):
    _fields_ = [("a", ctypes.c_int64), ("b", ctypes.c_int64), ("p", ctypes.c_void_p), ("l", ctypes.c_void_p),
                ("qh", ctypes.c_int32), ("kh", ctypes.c_int32), ("k", ctypes.c_int32), ("v", ctypes.c_int32),
                ("scale", ctypes.c_float)]
class B(ctypes.Structure):
    _fields_ = [("lists", ctypes.c_int64), ("items", ctypes.c_int64), ("stride", ctypes.c_int64),
                ("beams", ctypes.c_int32), ("width", ctypes.c_int32), ("end", ctypes.c_int32)]
P, i64 = ctypes.c_void_p, ctypes.c_int64
at = lambda n: (n + 1) << 50
case, n = sys.argv[4], int(sys.argv[5])
if case == "rows":  # n rows of one token
    s = S(n, n, at(0), at(1), 4, 4, 8, 8, 1.0)
    h = lambda i: H(at(i), 32, 8)
    lib.als_decay_attention.argtypes = [P, ctypes.c_int, H, H, H, P, P, P, P, i64, P]
    st = lib.als_decay_attention(ctypes.byref(s), 0, h(2), h(3), h(4), None, at(5), None, at(6), 1 << 50, None)
elif case == "step":
    s = S(0, n, None, at(1), 4, 4, 8, 8, 1.0)
    h = lambda i: H(at(i), 32, 8)
    lib.als_decay_attention_step.argtypes = [P, ctypes.c_int, H, H, H, P, i64, P, P, P, P]
    st = lib.als_decay_attention_step(ctypes.byref(s), 0, h(2), h(3), h(4), at(5), n, None, at(6), at(7), None)
else:
    s = B(n, 5000, 5000, 2, 2, -1)
    lib.als_beam_select.argtypes = [P, ctypes.c_int] + [P] * 8 + [i64, P]
    st = lib.als_beam_select(ctypes.byref(s), 0, at(0), at(1), None, at(2), at(3), at(4), at(5), at(6), 1 << 50, None)
if st:
    sys.exit(lib.als_last_error(None).decode())
"""


@pytest.mark.parametrize("case,n,totals", [
    # places (4 rows a block), segments' states, their join, outputs: heads * slots
    ("rows", 3_000_000, None), ("rows", 400_000_000, None),
    ("step", 1000, {256: 4000}), ("step", 5_000_000, {256: 20_000_000}),
    ("beam", 1000, {256: 4000, 1024: 1000}), ("beam", 6_000_000, {256: 24_000_000, 1024: 6_000_000})])
def test_grids_hold_their_threads(case, n, totals, tmp_path):
    import os
    import subprocess
    import sys

    here = os.path.dirname(os.path.abspath(__file__))
    so = str(tmp_path / "librecorder.so")
    subprocess.check_call(["gcc", "-O1", "-shared", "-fPIC", "-o", so, os.path.join(here, "launch_recorder.c")])
    r = subprocess.run([sys.executable, "-c", LAUNCH, so, os.path.dirname(here), p.LIB_PATH, case, str(n)],
                       capture_output=True, text=True, env=dict(os.environ, RECORDED_ARGS="0"))
    assert r.returncode == 0, r.stderr
    out = [[int(w) for w in line.split()] for line in r.stdout.splitlines()]
    assert out and all(threads * blocks < 2 ** 32 for threads, blocks in out)
    if totals:
        seen = {}
        for threads, blocks in out:
            seen[threads] = seen.get(threads, 0) + blocks
        assert seen == totals

"""Strides on their way to the attention kernels, seen at the launch (nothing runs): the passes from the
last token to the first address a row from C - 1 rows below it, so that a stride that no token needs must
not reach them."""
import os
import subprocess
import sys

import pytest

import paper_1108_2580_amd as p

CALL = """
import ctypes, sys
ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
lib.als_last_error.restype = ctypes.c_char_p
class H(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("t", ctypes.c_int64), ("h", ctypes.c_int64)]
class S(ctypes.Structure):
    _fields_ = [("a", ctypes.c_int64), ("b", ctypes.c_int64), ("p", ctypes.c_void_p), ("l", ctypes.c_void_p),
                ("qh", ctypes.c_int32), ("kh", ctypes.c_int32), ("k", ctypes.c_int32), ("v", ctypes.c_int32),
                ("scale", ctypes.c_float)]
P, i64 = ctypes.c_void_p, ctypes.c_int64
at = lambda n: (n + 1) << 52
case, dtype, n, stride = sys.argv[3], int(sys.argv[4]), int(sys.argv[5]), int(sys.argv[6])
h = lambda i: H(at(i), stride, 64)
s = S(n, 1 if case != "step" else n, at(0), at(1), 4, 4, 64, 64, 1.0)
if case == "forward":
    lib.als_decay_attention.argtypes = [P, ctypes.c_int, H, H, H, P, P, P, P, i64, P]
    st = lib.als_decay_attention(ctypes.byref(s), dtype, h(2), h(3), h(4), None, at(5), None, at(6), 1 << 50, None)
elif case == "backward":
    lib.als_decay_attention_backward.argtypes = [P, ctypes.c_int, H, H, H, H, P, P, P, P, P, P, P, i64, P]
    st = lib.als_decay_attention_backward(ctypes.byref(s), dtype, h(2), h(3), h(4), h(5), None, None, at(6), at(7),
                                          at(8), None, at(9), 1 << 50, None)
else:
    lib.als_decay_attention_step.argtypes = [P, ctypes.c_int, H, H, H, P, i64, P, P, P, P]
    st = lib.als_decay_attention_step(ctypes.byref(s), dtype, h(2), h(3), h(4), at(5), n, None, at(6), at(7), None)
if st:
    sys.exit(lib.als_last_error(None).decode())
"""


@pytest.fixture(scope="module")
def recorder(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("recorder") / "librecorder.so")
    here = os.path.dirname(os.path.abspath(__file__))
    subprocess.check_call(["gcc", "-O1", "-shared", "-fPIC", "-o", so, os.path.join(here, "args_recorder.c")])
    return so


def launches(recorder, words, *args):
    r = subprocess.run([sys.executable, "-c", CALL, recorder, p.LIB_PATH, *map(str, args)], capture_output=True,
                       text=True, env=dict(os.environ, RECORDED_WORDS=str(words)))
    return r, [[int(w) for w in line.split()] for line in r.stdout.splitlines()]


@pytest.mark.parametrize("case", ["forward", "backward"])
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("stride", [1 << 22, 1 << 26, 1 << 27, 1 << 30, (1 << 50) + 64])
def test_one_tokens_stride_reaches_no_kernel(recorder, case, dtype, stride):
    """The three passes' description is 48 words and more in all."""
    r, out = launches(recorder, 48, case, dtype, 1, stride)
    assert r.returncode == 0, r.stderr
    assert out
    for words in out:
        assert (4 << 52) in words  # the description is there: k's data (v's, in a pass of the gradients)
        assert stride not in words


@pytest.mark.parametrize("case", ["forward", "backward"])
@pytest.mark.parametrize("dtype", [0, 1])
def test_two_tokens_strides_are_bounded(recorder, case, dtype):
    """From 2^22 + 1 values on: refused. Up to there 63 rows' offsets in bytes stay below 2^31."""
    r, out = launches(recorder, 48, case, dtype, 2, (1 << 22) + 1)
    assert r.returncode != 0 and "token_stride" in r.stderr and not out
    assert 63 * (1 << 22) * 4 < 1 << 31
    r, out = launches(recorder, 48, case, dtype, 2, 1 << 22)
    assert r.returncode == 0 and out, r.stderr


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("stride", [(1 << 22) + 64, 1 << 30])
def test_a_steps_rows_may_lie_any_distance_apart(recorder, dtype, stride):
    """As one token of each history in a padded batch does. The step addresses its rows in 64 bits."""
    r, out = launches(recorder, 1, "step", dtype, 3, stride)
    assert r.returncode == 0 and len(out) == 1, r.stderr

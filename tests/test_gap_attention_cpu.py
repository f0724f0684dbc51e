"""Refusals of the attention over gaps of time: arguments that the host can check are checked before any device
call, so these run without a GPU. Pointers are made up and never followed, but for the host's bounds."""
import ctypes
import math

import pytest

from paper_1108_2580_amd import lib, sequence
from paper_1108_2580_amd.sequence import _GapPath, _Gaps, _Heads

torch = pytest.importorskip("torch")

# buffers 256 MiB apart
A, B, C, D, E, F, G, I, J, K, L, M, N, W = (0x10000000 * i for i in range(1, 15))
INVALID = 1
BOUNDS = (ctypes.c_int32 * 63)(*range(1, 64))


def refused(status, word):
    msg = lib.als_last_error(None).decode()
    assert status == INVALID and word in msg, (status, msg)


def bounds(*values):
    return ctypes.cast((ctypes.c_int32 * len(values))(*values), ctypes.c_void_p)


def gaps(**kw):
    d = dict(n_tokens=5000, n_rows=3, row_ptr=A, positions=B, bias=C, bounds=ctypes.cast(BOUNDS, ctypes.c_void_p),
             q_heads=4, k_heads=2, width=64, buckets=16, scale=0.125)
    d.update(kw)
    return _Gaps(**d)


def path(**kw):
    d = dict(beams=4, steps=3, q_positions=I, k=_Heads(J, 128, 64), v=_Heads(K, 128, 64), k_step=12 * 128,
             v_step=12 * 128, positions=L, path=M, path_stride=3)
    d.update(kw)
    return _GapPath(**d)


Q, KH, VH = _Heads(D, 256, 64), _Heads(E, 128, 64), _Heads(F, 128, 64)


def read(shape, dtype=1, q=Q, k=KH, v=VH, out=G, stats=None, rest=None, work=None, size=0):
    return lib.als_gap_attention(shape, dtype, q, k, v, out, stats, rest, work, size, None)


def back(shape, dtype=1, d_out=_Heads(I, 256, 64), q=Q, k=KH, v=VH, out=G, stats=J, rest=None, dq=K, dk=L, dv=M,
         dbias=N, work=W, size=1 << 40):
    return lib.als_gap_attention_backward(shape, dtype, d_out, q, k, v, out, stats, rest, dq, dk, dv, dbias, work,
                                          size, None)


def step(shape, p, dtype=1, q=Q, k=KH, v=VH, out=G, work=W, size=1 << 40):
    return lib.als_gap_attention_step(shape, p, dtype, q, k, v, out, work, size, None)


SHAPES = [
    (dict(n_tokens=-1), "n_tokens"), (dict(n_tokens=(1 << 31) - 255), "n_tokens"), (dict(n_rows=-1), "n_rows"),
    (dict(n_rows=(1 << 30) + 1), "n_rows"), (dict(n_rows=0), "without rows"), (dict(row_ptr=None), "row_ptr"),
    (dict(positions=None), "positions"), (dict(bias=None), "bias"), (dict(bounds=None), "bounds"),
    (dict(q_heads=0), "q_heads"), (dict(q_heads=1025, k_heads=1), "q_heads"), (dict(q_heads=3), "multiple"),
    (dict(k_heads=0), "k_heads"), (dict(width=0), "width"), (dict(width=129), "width"), (dict(buckets=0), "buckets"),
    (dict(buckets=65), "buckets"), (dict(scale=math.nan), "scale"), (dict(scale=math.inf), "scale"),
    (dict(buckets=2, bounds=bounds(0)), "bounds[0]"), (dict(buckets=2, bounds=bounds(-3)), "bounds[0]"),
    (dict(buckets=4, bounds=bounds(1, 5, 5)), "bounds[2]"), (dict(buckets=3, bounds=bounds(7, 6)), "bounds[1]")]


@pytest.mark.parametrize("change,word", SHAPES)
def test_shapes(change, word):
    refused(read(gaps(**change)), word)
    refused(back(gaps(**change)), word)
    refused(step(gaps(**change), path()), word)


def test_no_shape_and_types():
    refused(read(None), "NULL")
    refused(read(gaps(), dtype=2), "dtype")
    refused(step(gaps(), None), "path is NULL")


@pytest.mark.parametrize("change,word", [
    (dict(q=_Heads(None, 256, 64)), "NULL"), (dict(k=_Heads(E, -1, 64)), "stride"),
    (dict(v=_Heads(F + 1, 128, 64)), "aligned"), (dict(q=_Heads(D, (1 << 22) + 1, 64)), "2^22"), (dict(out=None), "out"),
    (dict(out=G + 1), "aligned"), (dict(stats=I + 2), "stats"), (dict(rest=I + 1), "rest"),
    (dict(rest=I, dtype=0), "bf16"), (dict(out=D), "overlaps q"), (dict(out=B), "overlaps"),
    (dict(stats=G), "overlaps out"), (dict(rest=G + 64), "overlaps out"), (dict(stats=A), "overlaps row_ptr")])
def test_reading(change, word):
    refused(read(gaps(), **change), word)


def test_workspaces():
    assert lib.als_gap_attention_workspace(gaps()) == 0  # few rows are counted
    many = gaps(n_rows=100)
    need = lib.als_gap_attention_workspace(many)
    assert need == 8 * 5000
    refused(read(many, work=W, size=need - 1), "workspace")
    refused(read(many, work=None, size=need), "workspace")
    refused(read(many, work=W + 8, size=need), "aligned")
    refused(read(many, work=G, size=need), "overlaps")
    need = lib.als_gap_attention_backward_workspace(gaps())
    # delta, a part of dbias for each 64 tokens, dk and dv of each query head
    assert need == 4 * 5000 * 4 + 4 * 79 * 4 * 16 + 2 * 4 * 5000 * 4 * 64
    refused(back(gaps(), size=need - 1), "workspace")
    assert lib.als_gap_attention_step_workspace(gaps(), path()) > 0
    refused(step(gaps(), path(), size=lib.als_gap_attention_step_workspace(gaps(), path()) - 1), "workspace")
    for bad in (dict(width=0), dict(q_heads=3), dict(buckets=65), dict(n_tokens=-1), dict(k_heads=0)):
        assert lib.als_gap_attention_workspace(gaps(**bad)) == -1
        assert lib.als_gap_attention_backward_workspace(gaps(**bad)) == -1
        assert lib.als_gap_attention_step_workspace(gaps(**bad), path()) == -1
    assert lib.als_gap_attention_step_workspace(gaps(), path(beams=33)) == -1
    assert lib.als_gap_attention_step_workspace(gaps(), None) == -1


@pytest.mark.parametrize("change,word", [
    (dict(d_out=_Heads(None, 256, 64)), "NULL"), (dict(out=None), "out"), (dict(stats=None), "stats"),
    (dict(rest=C, dtype=0), "bf16"), (dict(dq=None), "dq"), (dict(dk=None), "dk"), (dict(dv=None), "dv"),
    (dict(dbias=None), "dbias"), (dict(dbias=N + 2), "dbias"), (dict(dk=K), "overlaps dq"), (dict(dv=L), "overlaps dk"),
    (dict(dq=G), "overlaps out"), (dict(dq=I), "overlaps d_out"), (dict(dv=D), "overlaps q"),
    (dict(dbias=C), "overlaps bias"), (dict(dbias=J), "overlaps stats"), (dict(work=K), "overlaps dq")])
def test_gradients(change, word):
    need = lib.als_gap_attention_backward_workspace(gaps())
    refused(back(gaps(), size=need, **change), word)


@pytest.mark.parametrize("change,word", [
    (dict(beams=0), "beams"), (dict(beams=33), "beams"), (dict(steps=-1), "steps"), (dict(steps=(1 << 20) + 1), "steps"),
    (dict(q_positions=None), "q_positions"), (dict(k=_Heads(None, 128, 64)), "path's k"),
    (dict(v=_Heads(K, -1, 64)), "path's v"), (dict(k_step=-1), "step"), (dict(v_step=1 << 60), "step"),
    (dict(positions=None), "positions"), (dict(path=None), "path"), (dict(path_stride=2), "path_stride"),
    (dict(k=_Heads(G, 128, 64)), "overlaps the path's k"), (dict(path=G), "overlaps path"),
    (dict(positions=W), "overlaps")])
def test_paths(change, word):
    refused(step(gaps(), path(**change), size=lib.als_gap_attention_step_workspace(gaps(), path())), word)


def test_too_many_beams():
    refused(step(gaps(n_rows=1 << 28, n_tokens=0), path(beams=16)), "lists of 16 beams")


@pytest.mark.parametrize("name", ["_Gaps", "_GapPath"])
def test_structures_have_the_headers_layout(name, tmp_path):
    import subprocess
    import os

    struct = getattr(sequence, name)
    cname = {"_Gaps": "als_gaps", "_GapPath": "als_gap_path"}[name]
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = "#include <stdio.h>\n#include <stddef.h>\n#include \"als.h\"\nint main(void) {\n"
    code += f'  printf("%zu", sizeof({cname}));\n'
    for field, _ in struct._fields_:
        code += f'  printf(" %zu", offsetof({cname}, {field}));\n'
    (tmp_path / "a.c").write_text(code + "  return 0;\n}\n")
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(tmp_path / "a.c"), "-o", str(tmp_path / "a")],
                   check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "a")], capture_output=True, text=True,
                                          check=True).stdout.split()]
    assert got == [ctypes.sizeof(struct)] + [getattr(struct, f).offset for f, _ in struct._fields_]


def test_binding_refuses_host_tensors():
    q, k = torch.zeros(4, 2, 8), torch.zeros(4, 1, 8)
    args = (q, k, k, torch.zeros(2, 3), torch.tensor([1, 2], dtype=torch.int32), torch.zeros(4, dtype=torch.int32),
            torch.tensor([0, 4]))
    with pytest.raises(TypeError, match="q must be"):
        sequence.gap_attention(*args)
    with pytest.raises(TypeError, match="q must be"):
        sequence.gap_attention_step(*args[:5], torch.zeros(4, dtype=torch.int32), *args[5:])

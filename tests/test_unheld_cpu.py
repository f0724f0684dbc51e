"""Refusals of als_clear_unheld, which are made before any device call. Pointers of tensors are made up and never
followed."""
import ctypes

import pytest

from paper_1108_2580_amd import lib
from paper_1108_2580_amd import sequence  # noqa: F401 (declares the arguments)

A, B, C = 0x10000000, 0x20000000, 0x30000000


def call(n_tokens=100, n_rows=3, row_ptr=A, n=2, tensors=(B, C), sizes=(64, 32)):
    at = None if tensors is None else (ctypes.c_void_p * len(tensors))(*tensors)
    of = None if sizes is None else (ctypes.c_int64 * len(sizes))(*sizes)
    status = lib.als_clear_unheld(n_tokens, n_rows, row_ptr, n, at, of, None)
    return status, lib.als_last_error(None).decode()


@pytest.mark.parametrize("change,word", [
    (dict(n_tokens=-1), "n_tokens"), (dict(n_tokens=1 << 31), "n_tokens"), (dict(n_rows=-1), "n_rows"),
    (dict(n_rows=(1 << 30) + 1), "n_rows"), (dict(row_ptr=None), "row_ptr"), (dict(row_ptr=A + 4), "row_ptr"),
    (dict(n=0), "tensors"), (dict(n=5), "tensors"), (dict(tensors=None), "NULL"), (dict(sizes=None), "NULL"),
    (dict(tensors=(B, None)), "tensors[1]"), (dict(sizes=(64, 0)), "token_bytes[1]"),
    (dict(sizes=((1 << 20) + 1, 1)), "token_bytes[0]"), (dict(tensors=(B, A - 8)), "overlaps row_ptr"),
    (dict(tensors=(A + 16, B)), "overlaps row_ptr")])
def test_refusals(change, word):
    status, message = call(**change)
    assert status == 1 and word in message, (status, message)


def test_no_tokens():
    assert call(n_tokens=0, tensors=(None, None))[0] == 0

"""Refusals of the decoding operators that need no GPU and no rows."""

import ctypes as C

import pytest

from paper_2307_04963_amd import _lib

P = C.c_void_p


@pytest.mark.parametrize("keys, values, dim, word", [
    (P((1 << 20) + 8), P(2 << 20), 64, "aligned"), (P(1 << 20), P((2 << 20) + 2), 64, "aligned"), (P(1 << 20), P(1 << 20), 64, "the values"),
    (P(1 << 20), P(2 << 20), 20, "dim not"), (P(1 << 20), None, 64, "together"),
])
def test_fork_of_no_rows_checks_the_cache(keys, values, dim, word):
    rc = _lib.lib.dycl_op_fork(P(1 << 12), 8, P(2 << 12), 4, 8, P(3 << 12), P(4 << 12), 0, None, 8, None, keys, values, 100, 2, 16, dim, None)
    assert rc == -1 and word in _lib.last_error() and "dycl_op_fork" in _lib.last_error()


def test_fork_of_no_rows():
    assert _lib.lib.dycl_op_fork(None, 8, None, 4, 8, None, None, 0, None, 8, None, P(1 << 20), P(2 << 20), 100, 2, 16, 64, None) == 0
    assert _lib.lib.dycl_op_fork(None, 8, None, 4, 8, None, None, 0, None, 8, None, None, None, 0, 0, 16, 0, None) == 0

"""Which kernel a product of the token operators takes: every tile shape is
taken somewhere, a launch holds the tiles, and more than it holds is refused
before anything is launched."""

import ctypes as C

import pytest

from paper_2307_04963_amd import _lib

lib = _lib.lib
P = C.c_void_p
A, B, D = P(1 << 12), P(2 << 12), P(3 << 12)       # aligned addresses that no refused call touches


def tile(rows, n, k, gated=0, experts=0):
    t = (C.c_int32 * 3)()
    _lib.check(lib.dycl_op_linear_tile(rows, n, k, gated, experts, t))
    return tuple(t)


@pytest.mark.parametrize("rows, n, k", [(1, 1, 1), (1 << 20, 1 << 20, 64), ((1 << 31) - 257, 8, 8), (1 << 29, 1000, 8), (1 << 26, 30000, 8)])
@pytest.mark.parametrize("gated", [0, 1])
@pytest.mark.parametrize("experts", [0, 64, 1024])
def test_a_launch_holds_the_tiles(rows, n, k, gated, experts):
    largest = ((rows + 255) // 256 + min(experts, rows)) * ((n + 255 - 128 * gated) // (256 - 128 * gated))
    t = (C.c_int32 * 3)()
    rc = lib.dycl_op_linear_tile(rows, n, k, gated, experts, t)
    if largest >= (1 << 23) - 1:
        assert rc == -1 and "launch" in _lib.last_error()
        return
    assert rc == 0
    tiles = ((rows + t[0] - 1) // t[0] + min(experts, rows)) * ((n + t[1] - 1) // t[1])
    assert tiles * 512 < 1 << 32


def test_more_than_a_launch_holds_is_refused_before_any():
    m = (1 << 31) - 1
    assert lib.dycl_op_linear(A, 8, m, 8, B, 8, 0, None, None, 0, None, 0, D, 0, 8, None, 0, None) == -1
    assert "dycl_op_linear: more tiles" in _lib.last_error()
    # the second product alone has too many
    assert lib.dycl_op_experts(A, 8, 1 << 30, 1 << 20, 8, 1, 1, B, 0, None, None, 0, B, None, A, A, A, A, None, 0, D, 1 << 20, A,
                               (1 << 63) - 1, None) == -1
    assert "dycl_op_experts" in _lib.last_error()


def test_tile_refusals():
    t = (C.c_int32 * 3)()
    for args in ((0, 8, 8, 0, 0), (1 << 31, 8, 8, 0, 0), (8, 0, 8, 0, 0), (8, 8, 0, 0, 0), (8, 8, 8, 0, 1025), (8, 8, 8, 0, -1)):
        assert lib.dycl_op_linear_tile(*args, t) == -1
    assert lib.dycl_op_linear_tile(8, 8, 8, 0, 0, None) == -1

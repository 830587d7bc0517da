"""Token operators without a GPU: the header's exports, the size functions and
the refusals, which all come before the first HIP call."""

import ctypes as C

import pytest

from paper_2307_04963_amd import _lib
from tests.test_abi_cpu import _declared

lib = _lib.lib
P = C.c_void_p
A, B, D = P(1 << 12), P(2 << 12), P(3 << 12)       # aligned addresses that no refused call touches


def test_exports_match_the_header():
    assert _declared("dycl_tokens.h") == sorted(_lib.TOKENS_EXPORTS)
    for n in _lib.TOKENS_EXPORTS:
        assert hasattr(lib, n), n


def _norm(**kw):
    a = dict(x=A, xt=0, ldx=64, y=None, yt=0, ldy=64, gate=None, ldg=64, gact=0, row=None, chan=None, rs=1.0, post=0, pw=None, pb=None,
             pre=1, qw=None, qb=None, eps=1e-6, n=4, d=64, h=None, ldh=64, u=B, ut=0, ldu=64)
    a.update(kw)
    return lib.dycl_op_norm(*a.values(), None)


@pytest.mark.parametrize("bad, word", [
    (dict(n=-1), "n outside"), (dict(n=1 << 31), "n outside"), (dict(d=0), "d outside"), (dict(d=32769, ldx=32769), "d outside"),
    (dict(xt=2), "element type"), (dict(ut=5), "element type"), (dict(y=D, yt=-1), "element type"), (dict(post=3, y=D), "unknown norm"),
    (dict(pre=-1), "unknown norm"), (dict(gact=3), "activation"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"),
    (dict(post=1), "without y"), (dict(gate=D), "without y"), (dict(row=D), "without y"), (dict(chan=D), "without y"),
    (dict(y=D, pw=D), "without a post norm"), (dict(pre=0, qw=D), "without a pre norm"), (dict(u=None), "without u"),
    (dict(u=None, pre=0), "neither"), (dict(x=None), "null x"), (dict(ldx=63), "pitch"), (dict(ldu=1), "pitch"),
    (dict(h=D, ldh=8), "pitch"), (dict(x=P(4097)), "aligned"), (dict(ut=1, u=P(4098)), "aligned"), (dict(qw=P(4098)), "aligned"),
    (dict(h=A, ldh=72), "h is x"), (dict(u=A), "u is another"), (dict(y=D, h=D, ldh=65), "h is y"), (dict(y=D, gate=B), "u is another"),
])
def test_norm_refuses(bad, word):
    assert _norm(**bad) == -1
    assert word in _lib.last_error() and "dycl_op_norm" in _lib.last_error()


def test_no_rows_is_no_work():
    assert _norm(n=0, x=None, u=B) == 0
    assert lib.dycl_op_linear(None, 64, 0, 64, None, 8, 0, None, None, 0, None, 0, None, 0, 8, None, 0, None) == 0
    assert lib.dycl_op_experts(None, 64, 0, 64, 32, 4, 2, None, 0, None, None, 0, None, None, None, None, None, None, None, 0, None, 64,
                               None, 0, None) == 0
    assert lib.dycl_op_route(None, 0, 8, None, None, 0, 8, 1, 1, 2, 0, 1, 1.0, None, None, None, None, None, None, 0, None) == 0


def _route(**kw):
    a = dict(l=A, lt=1, ldl=64, bias=None, mask=None, n=100, E=64, G=1, T=1, k=4, score=0, renorm=1, scale=1.0, ids=B, w=D, off=A,
             order=B, slots=D, ws=A, wsb=1 << 20)
    a.update(kw)
    return lib.dycl_op_route(*a.values(), None)


@pytest.mark.parametrize("bad, word", [
    (dict(E=0), "experts outside"), (dict(E=1025, ldl=1025), "experts outside"), (dict(k=0), "k outside"), (dict(k=65), "k outside"),
    (dict(E=64, k=33), "k outside"), (dict(G=0), "groups outside"), (dict(G=5), "groups outside"), (dict(G=128, E=128, ldl=128), "groups outside"),
    (dict(G=4, T=5), "top_groups"), (dict(T=0), "top_groups"), (dict(score=2), "score"), (dict(lt=2), "element type"),
    (dict(n=-1), "n * k"), (dict(n=1 << 30), "n * k"), (dict(off=None), "together"), (dict(slots=None), "together"),
    (dict(l=None), "null"), (dict(ids=None), "null"), (dict(ldl=63), "pitch"), (dict(ws=None), "workspace"), (dict(wsb=8), "workspace"),
    (dict(ids=P(4098)), "aligned"), (dict(l=P(4098)), "aligned"),
])
def test_route_refuses(bad, word):
    assert _route(**bad) == -1
    assert word in _lib.last_error() and "dycl_op_route" in _lib.last_error()


def test_sizes():
    assert lib.dycl_op_linear_packed_bytes(1, 1, 1, 0) == 32 * 64 * 2           # one strip of 32 outputs, 64 inputs
    assert lib.dycl_op_linear_packed_bytes(3, 33, 65, 1) == 3 * 64 * 128 * 2 * 2
    for bad in ((0, 1, 1), (1025, 1, 1), (1, 0, 1), (1, 1, 0), (1, (1 << 20) + 1, 1)):
        assert lib.dycl_op_linear_packed_bytes(*bad, 0) == 0
    assert lib.dycl_op_linear_workspace(A, 64, 5, 64, 8, 0) == 0                # aligned rows need none
    for x, ldx, k in ((P(4098), 64, 64), (A, 65, 64), (A, 64, 63)):
        assert lib.dycl_op_linear_workspace(x, ldx, 5, k, 8, 0) >= 5 * ((k + 7) // 8 * 8) * 2
    assert lib.dycl_op_experts_workspace(A, 64, 0, 4, 2, 64, 32) == 0
    assert lib.dycl_op_experts_workspace(A, 64, 10, 4, 2, 64, 33) >= 20 * (64 + 64) * 2
    assert lib.dycl_op_route_workspace(0, 8, 2) == 0 and lib.dycl_op_route_workspace(100, 8, 2) >= 0


def _linear(**kw):
    a = dict(x=A, ldx=64, m=4, k=64, w=B, n=8, gated=0, bias=None, gbias=None, act=0, res=None, ldr=8, y=D, yt=0, ldy=8, ws=None, wsb=0)
    a.update(kw)
    return lib.dycl_op_linear(*a.values(), None)


@pytest.mark.parametrize("bad, word", [
    (dict(n=0), "n or k"), (dict(k=0), "n or k"), (dict(m=-1), "m outside"), (dict(act=4), "activation"), (dict(yt=3), "element type"),
    (dict(gbias=A), "gate bias"), (dict(x=None), "null"), (dict(w=None), "null"), (dict(y=None), "null"), (dict(ldx=63), "pitch"),
    (dict(ldy=7), "pitch"), (dict(res=A, ldr=1), "pitch"), (dict(w=P(4104)), "aligned"), (dict(yt=1, y=P(4098)), "aligned"),
    (dict(y=A), "y is x"), (dict(res=D, yt=1), "residual"), (dict(k=63), "workspace"), (dict(x=P(4098), ws=A, wsb=8), "workspace"),
])
def test_linear_refuses(bad, word):
    assert _linear(**bad) == -1
    assert word in _lib.last_error() and "dycl_op_linear" in _lib.last_error()


def test_pack_refuses():
    for args, word in (((None, None, 1, 8, 64, B, 1 << 20), "null"), ((A, None, 1, 8, 64, None, 1 << 20), "null"),
                       ((A, None, 0, 8, 64, B, 1 << 20), "experts"), ((A, None, 1, 8, 64, B, 16), "too small"),
                       ((A, None, 1, 8, 64, P(4104), 1 << 20), "aligned")):
        assert lib.dycl_op_linear_pack(*args, None) == -1
        assert word in _lib.last_error()


def _experts(**kw):
    a = dict(x=A, ldx=64, n=4, d=64, f=32, E=8, k=2, w1=B, gated=0, b1=None, g1=None, act=1, w2=B, b2=None, w=A, off=A, order=A, slots=A,
             res=None, ldr=64, out=D, ldo=64, ws=A, wsb=1 << 20)
    a.update(kw)
    return lib.dycl_op_experts(*a.values(), None)


@pytest.mark.parametrize("bad, word", [
    (dict(E=0), "experts outside"), (dict(d=0), "experts outside"), (dict(f=0), "experts outside"), (dict(k=0), "k outside"),
    (dict(k=9), "k outside"), (dict(n=-1), "n * k"), (dict(n=1 << 30), "n * k"), (dict(act=9), "activation"), (dict(g1=A), "gate bias"),
    (dict(x=None), "null"), (dict(order=None), "null"), (dict(out=None), "null"), (dict(ldx=1), "pitch"), (dict(ldo=63), "pitch"),
    (dict(ws=None), "workspace"), (dict(wsb=64), "workspace"), (dict(w2=P(4104)), "aligned"), (dict(res=D, ldr=72), "residual"),
])
def test_experts_refuses(bad, word):
    assert _experts(**bad) == -1
    assert word in _lib.last_error() and "dycl_op_experts" in _lib.last_error()

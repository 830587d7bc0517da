"""Decoding operators without a GPU: the header's exports, the size functions,
the frequencies, and the refusals, which all come before the first HIP call."""

import ctypes as C
import math
from types import SimpleNamespace

import pytest
import torch

from paper_2307_04963_amd import _lib, decoding as de
from tests.test_abi_cpu import _declared

lib = _lib.lib
P = C.c_void_p
A, B, D, E, F = (P(i << 12) for i in range(1, 6))       # aligned addresses that no refused call touches


def test_exports_match_the_header():
    assert _declared("dycl_decode.h") == sorted(_lib.DECODE_EXPORTS)
    for n in _lib.DECODE_EXPORTS:
        assert hasattr(lib, n), n


def _rotate(**kw):
    a = dict(x=A, type=0, ldx=256, pos=B, freq=D, pairs=32, layout=0, mag=1.0, adj=0, n=4, heads=4, dim=64, y=E, ldy=256)
    a.update(kw)
    return lib.dycl_op_rotate(*a.values(), None)


@pytest.mark.parametrize("bad, word", [
    (dict(n=-1), "n outside"), (dict(n=1 << 31), "n outside"), (dict(heads=0), "heads below"), (dict(dim=1), "dim below"),
    (dict(heads=1025, ldx=1 << 20, ldy=1 << 20), "above 65536"), (dict(type=2), "element type"), (dict(pairs=0), "no pairs"),
    (dict(pairs=33), "pairs outside"), (dict(pairs=2049, dim=8192, heads=1), "pairs outside"), (dict(freq=None), "null frequencies"),
    (dict(freq=P(4100)), "8 bytes"), (dict(layout=2), "layout"), (dict(mag=float("nan")), "magnitude"), (dict(mag=float("inf")), "magnitude"),
    (dict(x=None), "null"), (dict(y=None), "null"), (dict(pos=None), "null"), (dict(ldx=255), "pitch"), (dict(ldy=8), "pitch"),
    (dict(x=P(4097)), "aligned"), (dict(type=1, y=P(4098)), "aligned"), (dict(pos=P(4098)), "aligned"), (dict(y=A, ldy=264), "another pitch"),
])
def test_rotate_refuses(bad, word):
    assert _rotate(**bad) == -1
    assert word in _lib.last_error() and "dycl_op_rotate" in _lib.last_error()


def _append(**kw):
    a = dict(k=A, ldk=128, v=B, ldv=128, q=None, ldq=0, qo=None, ldo=0, type=0, pos=D, seq=None, freq=E, pairs=32, layout=0, mag=1.0, n=4,
             qh=0, heads=2, dim=64, tables=F, ldt=8, sequences=4, max_pages=8, keys=P(1 << 20), values=P(2 << 20), pages=100, page=16)
    a.update(kw)
    return lib.dycl_op_append(*a.values(), None)


SIZES = [
    (dict(heads=0), "heads outside"), (dict(dim=60), "dim not"), (dict(dim=264), "dim not"), (dict(dim=0), "dim not"), (dict(page=4), "page not"),
    (dict(page=24), "page not"), (dict(page=2048), "page not"), (dict(max_pages=0), "max_pages"), (dict(max_pages=1 << 28, page=16), "max_pages"),
    (dict(pages=0), "pages outside"), (dict(pages=1 << 31), "pages outside"), (dict(sequences=-1), "sequences outside"),
]


@pytest.mark.parametrize("bad, word", SIZES + [
    (dict(n=-1), "n outside"), (dict(heads=2000), "above 65536"), (dict(type=3), "element type"), (dict(pairs=33), "pairs outside"),
    (dict(pairs=-1), "pairs outside"), (dict(freq=None), "null frequencies"), (dict(layout=-1), "layout"), (dict(q=A), "together"),
    (dict(qo=A), "together"), (dict(q=A, qo=B), "q_heads"), (dict(q=A, qo=B, qh=2000), "q_heads"), (dict(n=5), "as many rows"),
    (dict(k=None), "null"), (dict(v=None), "null"), (dict(pos=None), "null"), (dict(tables=None), "null"), (dict(keys=None), "null"),
    (dict(ldk=127), "pitch"), (dict(ldt=7), "pitch"), (dict(q=A, qo=B, qh=4, ldq=256, ldo=255), "pitch"), (dict(keys=P((1 << 20) + 8)), "aligned"),
    (dict(type=1, k=P(4098)), "aligned"), (dict(seq=P(4097)), "aligned"), (dict(values=P(1 << 20)), "the same"),
    (dict(q=A, qo=A, qh=4, ldq=256, ldo=264), "another pitch"),
])
def test_append_refuses(bad, word):
    assert _append(**bad) == -1
    assert word in _lib.last_error() and "dycl_op_append" in _lib.last_error()


def _attend(**kw):
    a = dict(q=A, ldq=512, n=4, qh=8, heads=2, dim=64, scale=0.125, keys=P(1 << 20), values=P(2 << 20), pages=100, page=16, tables=F, ldt=8,
             sequences=4, max_pages=8, lengths=B, seq=None, max_length=128, window=0, mask=None, ldm=0, out=D, ldo=512, ws=None, wsb=0)
    a.update(kw)
    return lib.dycl_op_attend(*a.values(), None)


@pytest.mark.parametrize("bad, word", SIZES + [
    (dict(n=-1), "n outside"), (dict(qh=7), "multiple of heads"), (dict(qh=1), "multiple of heads"), (dict(n=1 << 30, sequences=1 << 30), "n * q_heads"),
    (dict(max_length=129), "max_length"), (dict(max_length=-1), "max_length"), (dict(window=-1), "window"), (dict(scale=float("nan")), "scale"),
    (dict(scale=float("inf")), "scale"), (dict(scale=-2e38), "scale"),
    (dict(n=3), "as many rows"), (dict(q=None), "null"), (dict(lengths=None), "null"), (dict(out=None), "null"), (dict(ldq=511), "pitch"),
    (dict(ldo=8), "pitch"), (dict(mask=A, ldm=127), "pitch"), (dict(keys=P((1 << 20) + 2)), "aligned"), (dict(out=P(4097)), "aligned"),
    (dict(out=A), "out is q"), (dict(max_pages=1 << 16, max_length=1 << 20, ldt=1 << 16), "workspace"),
    (dict(max_pages=1 << 16, max_length=1 << 20, ldt=1 << 16, ws=A, wsb=1000), "workspace"),
])
def test_attend_refuses(bad, word):
    assert _attend(**bad) == -1
    assert word in _lib.last_error() and "dycl_op_attend" in _lib.last_error()


def _beam(**kw):
    a = dict(logits=A, type=0, ldl=1000, scores=B, ended=None, end=-1, sequences=2, beams=4, words=1000, k=4, parents=D, tokens=E, new=F,
             over=P(6 << 12), ws=P(7 << 12), wsb=1 << 20)
    a.update(kw)
    return lib.dycl_op_beam(*a.values(), None)


@pytest.mark.parametrize("bad, word", [
    (dict(beams=0), "beams outside"), (dict(beams=65), "beams outside"), (dict(k=0), "k outside"), (dict(k=65), "k outside"),
    (dict(words=0), "words outside"), (dict(words=(1 << 20) + 1), "words outside"), (dict(sequences=-1), "sequences * beams"),
    (dict(sequences=1 << 22), "sequences * beams"), (dict(type=7), "element type"), (dict(ended=A), "end token"), (dict(ended=A, end=1000), "end token"),
    (dict(logits=None), "null"), (dict(over=None), "null"), (dict(ldl=999), "pitch"), (dict(type=1, logits=P(4098)), "aligned"),
    (dict(ws=P(4104)), "aligned"), (dict(new=B), "old ones"), (dict(ended=P(6 << 12), end=1), "old ones"), (dict(ws=None), "workspace"),
    (dict(wsb=10), "workspace"),
])
def test_beam_refuses(bad, word):
    assert _beam(**bad) == -1
    assert word in _lib.last_error() and "dycl_op_beam" in _lib.last_error()


def _fork(**kw):
    a = dict(tables=A, ldt=8, lengths=B, rows=4, max_pages=8, parents=D, fresh=E, n=4, nt=F, ldn=8, nl=P(6 << 12), keys=P(1 << 20),
             values=P(2 << 20), pages=100, heads=2, page=16, dim=64)
    a.update(kw)
    return lib.dycl_op_fork(*a.values(), None)


@pytest.mark.parametrize("bad, word", [(b, w) for b, w in SIZES if "sequences" not in b] + [
    (dict(rows=-1), "sequences outside"), (dict(n=-1), "n outside"), (dict(values=None), "together"), (dict(nl=None), "together"),
    (dict(keys=None, values=None, nt=None, nl=None), "neither"), (dict(tables=None), "null"), (dict(fresh=None), "null"), (dict(ldt=7), "pitch"),
    (dict(ldn=7), "pitch"), (dict(parents=P(4098)), "aligned"), (dict(keys=P((1 << 20) + 4)), "aligned"), (dict(nt=A), "old ones"),
    (dict(nl=B), "old ones"), (dict(values=P(1 << 20)), "the values"),
])
def test_fork_refuses(bad, word):
    assert _fork(**bad) == -1
    assert word in _lib.last_error() and "dycl_op_fork" in _lib.last_error()


def test_no_rows_is_no_work():
    assert _rotate(n=0, x=None, y=None, pos=None) == 0
    assert _append(n=0, sequences=0, k=None, v=None) == 0
    assert _attend(n=0, sequences=0, q=None, out=None) == 0
    assert _beam(sequences=0, logits=None, ws=None) == 0
    assert _fork(n=0, tables=None) == 0


def test_sizes():
    assert lib.dycl_op_attend_workspace(4, 8, 2, 64, 64, 0) == 0                 # one part: nothing to join
    for n in (0, -1, 1 << 31):
        assert lib.dycl_op_attend_workspace(n, 8, 2, 64, 1 << 16, 0) == 0
    long, windowed = (lib.dycl_op_attend_workspace(4, 8, 2, 64, 1 << 20, w) for w in (0, 2000))
    assert long > windowed > 0
    for all_of_it in (1 << 20, (1 << 63) - 1):                                   # a window that is none
        assert lib.dycl_op_attend_workspace(4, 8, 2, 64, 1 << 20, all_of_it) == long
    assert lib.dycl_op_attend_workspace(8, 8, 2, 64, 1 << 20, 0) == 2 * long
    assert lib.dycl_op_beam_workspace(0, 4, 1000, 4) == lib.dycl_op_beam_workspace(2, 65, 1000, 4) == 0
    assert lib.dycl_op_beam_workspace(2, 4, 1000, 4) >= 8 * (4 * 8 + 8)


def test_frequencies():
    f = de.frequencies(64, 10000.0, device="cpu")
    assert f.dtype == torch.float64 and len(f) == 32 and float(f[0]) == 1.0
    assert abs(float(f[31]) - 10000.0 ** (-62 / 64)) < 1e-18
    near = lambda a, b: abs(float(a) - float(b)) <= 1e-14 * abs(float(b))  # noqa: E731
    g = de.frequencies(64, scaling="linear", factor=4.0, device="cpu")
    assert all(near(a, b / 4) for a, b in zip(g, f))
    g = de.frequencies(64, scaling="base", factor=8.0, device="cpu")
    assert near(g[0], f[0]) and near(g[31], f[31] / 8)
    for scaling in ("turns", "pairs"):
        g = de.frequencies(64, scaling=scaling, factor=8.0, trained=4096, slow=2.0, fast=16.0, device="cpu")
        turns = 4096 * f / (2 * math.pi)
        for i in range(32):
            if turns[i] >= 16:
                assert near(g[i], f[i]), i
            elif turns[i] <= 2 and (scaling == "turns" or turns[i - 1] <= 2):
                assert near(g[i], f[i] / 8), i
            else:
                assert f[i] / 8 <= g[i] <= f[i] * (1 + 1e-14)
        if scaling == "turns":
            i = int((turns > 2).sum()) - 1
            keep = (turns[i] - 2) / 14
            assert near(g[i], f[i] * (keep + (1 - keep) / 8))


@pytest.mark.parametrize("bad", [
    dict(dims=63), dict(dims=0), dict(dims=64, base=0.0), dict(dims=64, factor=-1.0), dict(dims=64, scaling="other"), dict(dims=2, scaling="base"),
    dict(dims=64, scaling="turns", factor=4.0), dict(dims=64, scaling="pairs", trained=4096, slow=4.0, fast=1.0), dict(dims=64, base=math.inf),
])
def test_frequencies_refuse(bad):
    with pytest.raises(ValueError):
        de.frequencies(device="cpu", **bad)


def test_a_stream_of_another_device():
    stream = SimpleNamespace(device=torch.device("cuda", 1))
    x, i, c = torch.zeros((4, 64)), torch.zeros(4, dtype=torch.int32), de.cache(2, 1, 8, 64, device="cpu")
    t, f = torch.zeros((4, 2), dtype=torch.int32), torch.zeros(4, dtype=torch.float64)
    for call in (lambda: de.rotate(x, i, f, dim=64, stream=stream), lambda: de.append(c, x, x, i, t, stream=stream),
                 lambda: de.attend(x, c, t, i, stream=stream), lambda: de.beam(x, x[:, 0], 4, stream=stream),
                 lambda: de.fork(c, t, i, i, i, stream=stream)):
        with pytest.raises(ValueError, match="stream belongs to cuda:1"):
            call()


def test_tensors_on_the_cpu():
    x, i, c = torch.zeros((4, 64)), torch.zeros(4, dtype=torch.int32), de.cache(2, 1, 8, 64, device="cpu")
    t, f = torch.zeros((4, 2), dtype=torch.int32), torch.zeros(4, dtype=torch.float64)
    for call in (lambda: de.rotate(x, i, f, dim=64), lambda: de.append(c, x, x, i, t), lambda: de.attend(x.bfloat16(), c, t, i),
                 lambda: de.beam(x, x[:, 0], 4), lambda: de.fork(c, t, i, i, i)):
        with pytest.raises(ValueError, match="on a GPU"):
            call()

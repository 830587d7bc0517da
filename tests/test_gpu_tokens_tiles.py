"""Every tile shape of the products, plain and gated, of one layer and of a
partition, against 64 bits.  The sizes are checked (without a GPU) to select the
shapes, so a change of the selection cannot leave one untested."""

import ctypes as C
import math

import pytest
import torch

from paper_2307_04963_amd import _lib

# rows and outputs of a tile, workgroups per CU
PLAIN = [(256, 256, 1), (128, 256, 2), (64, 128, 2), (64, 128, 1), (64, 64, 1), (32, 64, 1), (32, 32, 1), (16, 32, 4), (16, 32, 1)]
GATED = [(256, 128, 1), (128, 128, 2), (64, 64, 2), (64, 64, 1), (64, 32, 1), (32, 32, 1), (16, 32, 5), (16, 32, 2), (16, 32, 1)]

# (rows, outputs, inputs): last tiles of 1, 128, 129 and 255 rows, outputs that end inside a strip, inputs inside a step
LINEAR = {
    False: [(1025, 8200, 520), (1152, 8200, 520), (1153, 8200, 520), (1279, 8200, 520), (4097, 2056, 520), (3000, 8200, 1032),
            (513, 8200, 72), (1300, 3100, 64), (1025, 4104, 520), (8193, 200, 72), (700, 4104, 264), (65, 8200, 72), (300, 4104, 264),
            (33, 8200, 72), (1025, 777, 200), (1, 8200, 264), (100, 3100, 520), (17, 4104, 72), (33, 3100, 520), (1300, 33, 64),
            (5, 4104, 136), (1, 33, 264), (65, 200, 1032)],
    True: [(513, 8200, 520), (640, 8200, 520), (641, 8200, 520), (767, 8200, 520), (1300, 3100, 520), (200, 8200, 64), (2177, 4104, 136),
           (65, 8200, 72), (2049, 777, 200), (17, 8200, 1032), (2177, 330, 200), (4097, 33, 72), (300, 1500, 200), (17, 4104, 200),
           (33, 3100, 1032), (4097, 33, 136), (100, 4104, 64), (17, 8200, 64), (1, 33, 64), (33, 2056, 64), (65, 330, 200)],
}

# (pairs of all 8 experts, d, f): the first layer has f outputs on d inputs, the second d on f
EXPERTS = {
    False: [(8200, 1032, 1032), (2300, 2056, 2056), (700, 264, 264), (513, 777, 72), (2049, 33, 520), (300, 520, 264), (40, 520, 520),
            (130, 200, 136), (17, 3100, 72), (700, 3100, 264), (200, 1032, 520)],
    True: [(8200, 1032, 520), (4200, 2056, 520), (1025, 200, 1032), (700, 264, 264), (2049, 264, 200), (4097, 72, 33), (300, 520, 520),
           (300, 136, 520), (9, 100, 330), (200, 72, 1032), (2177, 520, 200), (300, 64, 330)],
}


def tile(rows, n, k, gated=False, experts=0):
    t = (C.c_int32 * 3)()
    _lib.check(_lib.lib.dycl_op_linear_tile(rows, n, k, int(gated), experts, t))
    return tuple(t)


def test_every_tile_is_run():
    assert {tile(*c) for c in LINEAR[False]} == set(PLAIN)
    assert {tile(*c, True) for c in LINEAR[True]} == set(GATED)
    first = {tile(n, f, d, True, 8) for n, d, f in EXPERTS[True]}
    second = {tile(n, d, f, False, 8) for n, d, f in EXPERTS[True] + EXPERTS[False]}
    second |= {tile(n, f, d, False, 8) for n, d, f in EXPERTS[False]}
    assert first == set(GATED), set(GATED) - first
    assert second == set(PLAIN), set(PLAIN) - second


def test_no_other_tile_is_selected():
    for gated, known in ((False, PLAIN), (True, GATED)):
        for experts in (0, 1, 8, 128):
            for rows in (1, 16, 17, 60, 250, 1000, 5000, 100000):
                for n in (1, 32, 100, 500, 2048, 10000):
                    for k in (1, 64, 300, 2048, 10000):
                        assert tile(rows, n, k, gated, experts) in known


@pytest.fixture(scope="module")
def ex():
    assert torch.cuda.is_available()
    from paper_2307_04963_amd import experts
    return experts


@pytest.mark.gpu
@pytest.mark.parametrize("gated", [False, True])
def test_linear_tiles(ex, gated):
    from tests.test_gpu_tokens import check_linear
    for i, (m, n, k) in enumerate(LINEAR[gated]):
        print("[tiles] linear", m, n, k, gated, tile(m, n, k, gated), flush=True)
        check_linear(ex, m, k, n, ("silu", "gelu", "none")[i % 3], gated, bias=i % 2 == 0, residual=i % 3 != 1,
                     out=(torch.bfloat16, torch.float32)[i % 2])


def counts(n):
    """Rows of 8 experts that add up to n: none, one, tiles' ends and one past them where n has room, the rest on one."""
    c = [0, 1, 128, 129, 255, 256, 65]
    while sum(c) > n:
        c = [v // 2 for v in c]
    return c + [n - sum(c)]


@pytest.mark.gpu
@pytest.mark.parametrize("gated", [False, True])
def test_experts_tiles(ex, gated):
    from tests.test_gpu_tokens import check_experts
    for i, (n, d, f) in enumerate(EXPERTS[gated]):
        print("[tiles] experts", n, d, f, gated, tile(n, f, d, gated, 8), tile(n, d, f, False, 8), flush=True)
        ids = torch.repeat_interleave(torch.arange(8), torch.tensor(counts(n)))
        ids = ids[torch.randperm(n, generator=torch.Generator().manual_seed(n))]
        check_experts(ex, n, 8, 1, d, f, ("silu", "relu", "gelu")[i % 3], gated, bias=i % 2 == 0, residual=i % 3 != 1, ids=ids[:, None].cuda())


def spaced(rows, width, pitch, seed):
    """rows of `width` random values, `pitch` apart in memory that is otherwise untouched."""
    room = torch.empty((rows - 1) * pitch + width, dtype=torch.bfloat16, device="cuda")
    view = room.as_strided((rows, width), (pitch, 1))
    view.copy_(torch.randn((rows, width), device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)))
    return view


@pytest.mark.gpu
@pytest.mark.parametrize("m, n, k, gated", [(1025, 8200, 520, False), (513, 8200, 520, True), (513, 8200, 72, False), (300, 4104, 264, False),
                                            (100, 3100, 520, False), (65, 330, 200, True)])
def test_linear_rows_beyond_32_bits(ex, m, n, k, gated):
    """256 rows at this pitch are 2^32 bytes: offsets of 64 bits in a tile."""
    print("[tiles] far", m, n, k, gated, tile(m, n, k, gated), flush=True)
    g = torch.Generator(device="cuda").manual_seed(m)
    mk = lambda: (torch.randn((n, k), generator=g, device="cuda") / math.sqrt(k)).bfloat16()  # noqa: E731
    w = ex.pack(mk(), mk() if gated else None)
    x = spaced(m, k, 1 << 23, m)
    assert torch.equal(ex.linear(x, w, act="relu"), ex.linear(x.contiguous(), w, act="relu"))


@pytest.mark.gpu
@pytest.mark.parametrize("n, d, f", [(8200, 1032, 520), (4200, 2056, 520), (700, 264, 264)])
def test_experts_rows_beyond_32_bits(ex, n, d, f):
    print("[tiles] far experts", n, d, f, flush=True)
    g = torch.Generator(device="cuda").manual_seed(n)
    mk = lambda a, b: (torch.randn((8, a, b), generator=g, device="cuda") / math.sqrt(b)).bfloat16()  # noqa: E731
    w, w2 = ex.pack(mk(f, d), mk(f, d)), ex.pack(mk(d, f))
    pitch = -(-(1 << 31) // n + 8) // 8 * 8 + 4096
    x = spaced(n, d, pitch, n)
    assert n * pitch * 2 >= 1 << 32
    r = ex.route(torch.randn((n, 8), generator=g, device="cuda"), 1)
    assert torch.equal(ex.experts(x, r, w, w2), ex.experts(x.contiguous(), r, w, w2))

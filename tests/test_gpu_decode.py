"""The decoding operators on the GPU against their definitions in 64 bits (tests/_decode.py has the bounds)."""

import math

import pytest
import torch

from tests._decode import ROUND, UNIT, attended64, chosen64, dense, gen, paged, put, turned64, within

pytestmark = pytest.mark.gpu

B, F = torch.bfloat16, torch.float32
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def de():
    assert torch.cuda.is_available()
    from paper_2307_04963_amd import decoding
    return decoding


def normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def rows_of(g, n, width, dtype, pad=0, skew=0):
    return normal(g, n, width + pad + skew).to(dtype)[:, skew:skew + width]


# ---- rotate --------------------------------------------------------------------

def check_rotate(de, n, heads, dim, pairs, layout, dtype, adjoint=False, magnitude=1.0, far=5000, pad=0, skew=0, inplace=False):
    g = gen(n * 31 + heads * dim + pairs)
    x = rows_of(g, n, heads * dim, dtype, pad, skew)
    positions = torch.randint(-3, far, (n,), generator=g, device="cuda").int()
    f = de.frequencies(2 * pairs)
    want, err = turned64(x, positions, f, layout, dim, adjoint, magnitude)
    y = de.rotate(x, positions, f, dim=dim, layout=layout, adjoint=adjoint, magnitude=magnitude, out=x if inplace else None)
    if inplace:
        assert y.data_ptr() == x.data_ptr()
    within(y, want, err + (ROUND * want.abs() if dtype == B else UNIT * want.abs()), f"{n} {heads} {dim} {pairs} {layout} {dtype}")
    rest = lambda t: t.reshape(n, heads, dim)[..., 2 * pairs:]  # noqa: E731
    if not inplace:
        assert torch.equal(rest(y), rest(x))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dim, pairs", [(2, 1), (3, 1), (8, 4), (10, 3), (64, 32), (64, 8), (80, 20), (96, 48), (128, 64), (128, 30), (256, 128), (513, 129),
                                        (4096, 2048)])
def test_rotate_dims(de, dim, pairs, layout):
    for dtype in (B, F):
        check_rotate(de, 13, 3, dim, pairs, layout, dtype)
        check_rotate(de, 7, 2, dim, pairs, layout, dtype, adjoint=True, magnitude=1.25, pad=3, skew=1)


@pytest.mark.parametrize("n, heads", [(1, 1), (1, 32), (2, 512), (1023, 5), (1024, 1), (2049, 1), (4100, 3), (65537, 1), (70000, 8)])
def test_rotate_rows(de, n, heads):
    for layout in ("half", "interleaved"):
        check_rotate(de, n, heads, 64, 32, layout, B)
        check_rotate(de, min(n, 3000), heads, 72, 12, layout, F, inplace=True)


def test_rotate_far_positions(de):
    """Angles keep 64 bits: a position of 2^31 - 1 is turned as exactly as the first."""
    g = gen(5)
    f = de.frequencies(128)
    x = normal(g, 6, 128)
    positions = torch.tensor([0, 1, -1, 1 << 20, 2**31 - 1, -2**31], dtype=torch.int32, device="cuda")
    want, err = turned64(x, positions, f, "half", 128)
    within(de.rotate(x, positions, f, dim=128), want, err + UNIT * want.abs())
    assert torch.equal(de.rotate(x, positions, f, dim=128)[0], x[0])


def test_rotate_gradient(de):
    """The adjoint is the gradient of the formula, and of differences of the operator itself."""
    g = gen(6)
    n, heads, dim, f = 9, 2, 24, de.frequencies(16)
    positions = torch.arange(n, dtype=torch.int32, device="cuda") * 7
    for layout in ("half", "interleaved"):
        x, dy = normal(g, n, heads * dim), normal(g, n, heads * dim)
        dx = de.rotate(dy, positions, f, dim=dim, layout=layout, adjoint=True, magnitude=0.75)
        leaf = x.double().requires_grad_()
        half = len(f)
        h = leaf.view(n, heads, dim)
        t = (positions.double()[:, None] * f)[:, None]
        a, b = (h[..., :half], h[..., half:2 * half]) if layout == "half" else (h[..., 0:2 * half:2], h[..., 1:2 * half:2])
        ya, yb = 0.75 * (a * t.cos() - b * t.sin()), 0.75 * (b * t.cos() + a * t.sin())
        y = torch.cat([ya, yb], -1) if layout == "half" else torch.stack([ya, yb], -1).flatten(-2)
        torch.cat([y, h[..., 2 * half:]], -1).reshape(n, -1).backward(dy.double())
        _, err = turned64(dy, positions, f, layout, dim, True, 0.75)
        within(dx, leaf.grad, err + UNIT * leaf.grad.abs())
        # a linear map: the difference along d is the map of d, up to the roundings of two results
        d = normal(g, n, heads * dim)
        of = lambda v: de.rotate(v, positions, f, dim=dim, layout=layout, magnitude=0.75).double()  # noqa: E731
        diff = ((of(x + d) - of(x - d)) * dy.double()).sum() / 2
        size = ((x.abs() + d.abs()).double().sum() * 4 * float(dy.abs().max()))
        assert abs(float(diff - (d.double() * dx.double()).sum())) <= float(size) * 2.0 ** -19


def test_rotate_nan_stays_in_its_pair(de):
    x = torch.ones((2, 64), device="cuda")
    x[0, 3] = NAN
    y = de.rotate(x, torch.tensor([5, 6], dtype=torch.int32, device="cuda"), de.frequencies(32), dim=64)
    assert torch.isnan(y).nonzero().tolist() == [[0, 3], [0, 19]]


# ---- append --------------------------------------------------------------------

def check_append(de, lengths, held, q_heads, heads, dim, pairs, layout, page, dtype, pad=0, magnitude=1.0, shuffle=True):
    """Sequences that hold `held` tokens receive the rest of `lengths`, rows in a random order with padding among them."""
    g = gen(sum(lengths) + dim)
    cache, tables = paged(g, lengths, heads, page, dim, max_pages=max(-(-n // page) for n in lengths) + 1, garbage=7.0)
    pairs_of = [(s, p) for s, (h, n) in enumerate(zip(held, lengths)) for p in range(h, n)] + [(0, -1), (len(lengths) - 1, -5)]
    order = torch.randperm(len(pairs_of), generator=g, device="cuda").tolist() if shuffle else range(len(pairs_of))
    sequence = torch.tensor([pairs_of[i][0] for i in order], dtype=torch.int32, device="cuda")
    positions = torch.tensor([pairs_of[i][1] for i in order], dtype=torch.int32, device="cuda")
    n = len(pairs_of)
    qkv = rows_of(g, n, (q_heads + 2 * heads) * dim, dtype, pad)
    q, k, v = qkv.split([q_heads * dim, heads * dim, heads * dim], 1)
    f = de.frequencies(2 * pairs) if pairs else None
    want = [c.clone() for c in cache]
    got_q = de.append(cache, k, v, positions, tables, sequence=sequence, frequencies=f, layout=layout, q=q, magnitude=magnitude)
    nothing = torch.zeros(0, dtype=torch.float64, device="cuda")
    turn = lambda t: turned64(t, positions, f if pairs else nothing, layout, dim, magnitude=magnitude)  # noqa: E731
    q64, qe = turn(q)
    padding = positions < 0
    q64[padding], qe[padding] = 0, 0
    last = ROUND if dtype == B else UNIT
    within(got_q, q64, qe + last * q64.abs(), "q")
    k64, ke = turn(k)
    for r in (~padding).nonzero()[:, 0].tolist():
        at = int(positions[r])
        place = int(tables[sequence[r], at // page]), slice(None), at % page
        within(cache.keys[place], k64[r].view(heads, dim), (ke[r] + ROUND * k64[r].abs()).view(heads, dim), "keys")
        assert torch.equal(cache.values[place], v[r].view(heads, dim).to(B))
        want[0][place], want[1][place] = cache.keys[place], cache.values[place]
    assert torch.equal(cache.keys, want[0]) and torch.equal(cache.values, want[1])     # nothing else is touched


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dim, pairs, page", [(8, 4, 8), (64, 32, 16), (72, 12, 8), (128, 64, 16), (128, 0, 32), (256, 64, 1024)])
def test_append_sizes(de, dim, pairs, page, layout, dtype):
    check_append(de, [1, 17, 40, 9], [0, 16, 3, 8], 6, 3, dim, pairs, layout, page, dtype, pad=5)


def test_append_heads_and_rows(de):
    check_append(de, [1], [0], 1, 1, 64, 32, "half", 8, B)
    check_append(de, [300, 211], [0, 100], 64, 8, 128, 64, "half", 64, B, magnitude=1.1)
    check_append(de, [1100, 13], [0, 0], 2, 1, 64, 16, "interleaved", 16, B, shuffle=False)


@pytest.mark.parametrize("heads", [8152, 8192])
def test_append_widest(de, heads):
    """Rows of 97824 and 98304 units of two values: the last ones belong to the same row."""
    for dtype in (B, F):
        check_append(de, [1, 2], [0, 7], heads, heads, 8, 1, "interleaved", 8, dtype)


def test_append_one_token_per_sequence(de):
    """Without `sequence` row r is sequence r; without q nothing is returned; q_out may be q."""
    g = gen(9)
    cache, tables = paged(g, [20, 33, 8], 2, 16, 64, garbage=0.0)
    k, v, q = normal(g, 3, 128).to(B), normal(g, 3, 128).to(B), normal(g, 3, 256).to(B)
    at = torch.tensor([19, 32, 0], dtype=torch.int32, device="cuda")
    f = de.frequencies(64)
    assert de.append(cache, k, v, at, tables) is None
    for r, p in enumerate([19, 32, 0]):
        assert torch.equal(dense(cache.keys, tables[r], p + 1)[:, p], k[r].view(2, 64))
        assert torch.equal(dense(cache.values, tables[r], p + 1)[:, p], v[r].view(2, 64))
    want = de.append(cache, k, v, at, tables, frequencies=f, q=q)
    out = de.append(cache, k, v, at, tables, frequencies=f, q=q, q_out=q)
    assert out.data_ptr() == q.data_ptr() and torch.equal(out, want)
    assert torch.equal(dense(cache.keys, tables[0], 20)[:, 19].reshape(1, -1), de.rotate(k[:1], at[:1], f, dim=64))


def test_append_bad_places(de):
    """Pages outside the cache, places past the table and sequences that do not exist: nothing is written, other rows are."""
    g = gen(10)
    cache, tables = paged(g, [32, 32], 2, 16, 64, garbage=3.0)
    before = [c.clone() for c in cache]
    tables[1, 0], tables[1, 1] = 1 << 20, -7
    positions = torch.tensor([0, 31, 32, 2**31 - 1, 5, 5, 5], dtype=torch.int32, device="cuda")
    sequence = torch.tensor([1, 1, 0, 0, 2, -1, 0], dtype=torch.int32, device="cuda")
    k, v = normal(g, 7, 128).to(B), normal(g, 7, 128).to(B)
    de.append(cache, k, v, positions, tables, sequence=sequence)
    page = int(tables[0, 0])
    before[0][page, :, 5], before[1][page, :, 5] = k[6].view(2, 64), v[6].view(2, 64)
    assert torch.equal(cache.keys, before[0]) and torch.equal(cache.values, before[1])


# ---- attend --------------------------------------------------------------------

def check_attend(de, lengths, q_heads, heads, dim, page, window=0, holes=0.0, max_length=None, scale=None, pad=0, big=1.0, rows=64):
    g = gen(sum(lengths) + q_heads * dim + window % 2**31)
    cache, tables = paged(g, lengths, heads, page, dim)
    n, cap = len(lengths), tables.shape[1] * page
    for r in range(n):
        for t in cache:
            put(t, tables[r], normal(g, heads, lengths[r], dim).to(B))
    q = (big * rows_of(g, n, q_heads * dim, F, pad, 1 if pad else 0)).to(B)
    mask = None
    if holes:
        mask = torch.rand((n, (max_length or cap) + 3), generator=g, device="cuda") >= holes
        mask[0] = False                                    # a row without any key
        for r in range(1, n):                              # what holes hold is nobody's
            for t in cache:
                d = dense(t, tables[r], lengths[r]).clone()
                d[:, :mask.shape[1]][:, ~mask[r, :lengths[r]]] = NAN if r % 2 else INF
                put(t, tables[r], d)
    out = de.attend(q, cache, tables, torch.tensor(lengths, dtype=torch.int32, device="cuda"), window=window, mask=mask,
                    max_length=max_length, scale=scale)
    assert out.shape == q.shape and out.dtype == B
    for r in range(0, n, max(1, n // rows)):
        m = min(lengths[r], max_length if max_length is not None else cap)
        here = torch.arange(m, device="cuda") >= (m - window if window else 0)
        if mask is not None:
            here &= mask[r, :m]
        want, bound = attended64(q[r].view(q_heads, dim), dense(cache.keys, tables[r], m), dense(cache.values, tables[r], m),
                                 1 / math.sqrt(dim) if scale is None else scale, here)
        within(out[r].view(q_heads, dim), want, bound, f"row {r} of {lengths[r]}")


LENGTHS = [0, 1, 2, 7, 8, 9, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200]


@pytest.mark.parametrize("page", [8, 16, 64, 1024])
@pytest.mark.parametrize("dim", [8, 32, 64, 72, 96, 128, 136, 192, 256])
def test_attend_dims_and_pages(de, dim, page):
    check_attend(de, LENGTHS, 4, 2, dim, page)
    check_attend(de, LENGTHS, 4, 2, dim, page, holes=0.4)


@pytest.mark.parametrize("q_heads, heads", [(1, 1), (3, 3), (16, 16), (5, 1), (32, 8), (16, 1), (17, 1), (40, 1), (64, 2), (128, 1)])
def test_attend_heads(de, q_heads, heads):
    check_attend(de, [100, 0, 700], q_heads, heads, 256, 16)
    check_attend(de, [0, 1, 33, 150], q_heads, heads, 64, 16)
    check_attend(de, [300, 1, 33, 900], q_heads, heads, 128, 32, holes=0.2, pad=3)


@pytest.mark.parametrize("length", [255, 256, 257, 511, 512, 513, 1000, 2047, 2049, 4095, 4096, 4097, 4608, 5000, 16384, 20011])
def test_attend_lengths(de, length):
    check_attend(de, [length, 3, length // 2, 0], 8, 2, 64, 16)
    check_attend(de, [length, length - 1], 4, 1, 128, 64, holes=0.1)


@pytest.mark.parametrize("window", [1, 7, 32, 33, 100, 128, 1000, 4096, 5000, 100000, 2**63 - 1])
def test_attend_window(de, window):
    check_attend(de, [0, 1, 31, 100, 500, 3000, 6001], 4, 2, 64, 16, window=window)
    check_attend(de, [5, 777], 2, 2, 128, 8, window=window, holes=0.3)


def test_attend_max_length(de):
    """Lengths above max_length count as it, below 0 as 0; the mask then has max_length columns."""
    check_attend(de, [100, 64, 65, 3], 4, 2, 64, 16, max_length=64)
    check_attend(de, [100, 64, 65, 3], 4, 2, 64, 16, max_length=50, holes=0.2)
    check_attend(de, [100, 9], 4, 2, 64, 16, max_length=0)
    g = gen(3)
    cache, tables = paged(g, [40], 1, 8, 64)
    q = normal(g, 1, 64).to(B)
    assert not de.attend(q, cache, tables, torch.tensor([-3], dtype=torch.int32, device="cuda")).any()


def test_attend_scales(de):
    """Large scores (one key takes all), a scale of 0 (all take the same), a negative one."""
    check_attend(de, [40, 300, 1000], 8, 2, 64, 16, big=30.0)
    check_attend(de, [40, 300, 1000], 8, 2, 64, 16, scale=0.0)
    check_attend(de, [40, 300, 1000], 8, 2, 64, 16, scale=-0.3)


def test_attend_many_rows(de):
    lengths = [(37 * i) % 700 for i in range(300)]
    check_attend(de, lengths, 4, 1, 64, 16, rows=40)


def test_attend_rows_of_one_sequence(de):
    """A prompt's tokens as rows of one sequence, each with its own length; sequences that do not exist have no keys."""
    g = gen(12)
    cache, tables = paged(g, [90, 20], 2, 16, 64)
    for r, n in ((0, 90), (1, 20)):
        for t in cache:
            put(t, tables[r], normal(g, 2, n, 64).to(B))
    rows = [(0, i + 1) for i in range(90)] + [(1, 20), (2, 5), (-1, 5)]
    q = normal(g, len(rows), 4 * 64).to(B)
    out = de.attend(q, cache, tables, torch.tensor([n for _, n in rows], dtype=torch.int32, device="cuda"),
                    sequence=torch.tensor([s for s, _ in rows], dtype=torch.int32, device="cuda"))
    for r, (s, n) in enumerate(rows):
        if s not in (0, 1):
            assert not out[r].any()
            continue
        want, bound = attended64(q[r].view(4, 64), dense(cache.keys, tables[s], n), dense(cache.values, tables[s], n), 0.125)
        within(out[r].view(4, 64), want, bound, f"row {r}")


def test_attend_bad_pages(de):
    """Keys on pages outside the cache, and past the table's end, are no keys."""
    g = gen(13)
    cache, tables = paged(g, [64, 64], 1, 16, 64)
    for r in range(2):
        for t in cache:
            put(t, tables[r], normal(g, 1, 64, 64).to(B))
    bad = tables.clone()
    bad[0, 1], bad[1, 0], bad[1, 3] = cache.keys.shape[0], -1, 2**31 - 1
    q = normal(g, 2, 64).to(B)
    out = de.attend(q, cache, bad, torch.tensor([64, 60], dtype=torch.int32, device="cuda"))
    for r, (n, gone) in enumerate(((64, [1]), (60, [0, 3]))):
        here = torch.ones(n, dtype=torch.bool, device="cuda")
        for p in gone:
            here[16 * p:16 * p + 16] = False
        want, bound = attended64(q[r].view(1, 64), dense(cache.keys, tables[r], n), dense(cache.values, tables[r], n), 0.125, here)
        within(out[r].view(1, 64), want, bound, f"row {r}")


def test_attend_infinite_values(de):
    """An infinite value of a key that is seen is infinite in its column alone; a key of -inf score has no weight."""
    g = gen(14)
    cache, tables = paged(g, [40], 1, 8, 64)
    k, v = normal(g, 1, 40, 64).to(B), normal(g, 1, 40, 64).to(B)
    v[0, 5, 7], v[0, 39, 9] = INF, -INF
    k[0, 11] = 0
    k[0, 11, 0] = -INF
    q = normal(g, 1, 64).to(B)
    q[0, 0] = 1.0
    put(cache.keys, tables[0], k)
    put(cache.values, tables[0], v)
    out = de.attend(q, cache, tables, torch.tensor([40], dtype=torch.int32, device="cuda"))[0]
    assert float(out[7]) == INF and float(out[9]) == -INF
    fine = torch.ones(64, dtype=torch.bool, device="cuda")
    fine[[7, 9]] = False
    here = torch.ones(40, dtype=torch.bool, device="cuda")
    here[11] = False
    v[0, 5, 7] = v[0, 39, 9] = 0
    want, bound = attended64(q.view(1, 64), k, v, 0.125, here)
    within(out[fine], want[0][fine], bound[0][fine])


@pytest.mark.parametrize("n, heads, q_heads, dim, most, page, window", [
    (40, 2, 8, 128, 100, 16, 0), (40, 2, 8, 128, 5000, 64, 0), (400, 1, 2, 64, 5000, 64, 0), (700, 2, 2, 64, 700, 8, 0), (90, 4, 20, 256, 7000, 32, 0),
    (300, 2, 2, 72, 4500, 128, 4200), (48, 8, 8, 64, 33000, 256, 0), (64, 2, 66, 128, 9000, 64, 0),
    (64, 1, 32, 256, 9000, 64, 0), (70, 1, 16, 200, 33000, 1024, 0)])
def test_attend_company_leaves_bits(de, n, heads, q_heads, dim, most, page, window):
    """A row's bits do not depend on the other rows, on the page order or on what is behind its keys."""
    g = gen(15 + n)
    per = -(-most // page)
    pages = max(4 * per, 64)
    cache = de.Cache(*(normal(g, pages, heads, page, dim).to(B) for _ in range(2)))
    tables = torch.randint(0, pages, (n, per), generator=g, device="cuda").int()       # (rows may share pages)
    q = normal(g, n, q_heads * dim).to(B)
    lengths = torch.randint(1, most + 1, (n,), generator=g, device="cuda").int()
    lengths[0], lengths[n // 2] = most, 0
    all_rows = de.attend(q, cache, tables, lengths, window=window)
    assert torch.equal(de.attend(q, cache, tables, lengths, window=window), all_rows)
    for first, last in ((0, 1), (n // 3, n // 3 + 1), (n - 1, n), (n // 2, n // 2 + 2), (1, 1 + n // 5)):
        some = de.attend(q[first:last], cache, tables[first:last], lengths[first:last], window=window)
        assert torch.equal(some, all_rows[first:last]), (first, last)
    swapped = torch.randperm(pages, generator=g, device="cuda")
    moved = de.Cache(*(torch.empty_like(t) for t in cache))
    for a, b in zip(moved, cache):
        a[swapped] = b
    assert torch.equal(de.attend(q, moved, swapped[tables.long()].int(), lengths, window=window), all_rows)


def test_attend_far_offsets(de):
    """A cache of more than 2^31 values: the pages of a sequence lie at its two ends."""
    g = gen(16)
    pages = (1 << 31) // (4 * 1024 * 128) + 4
    cache = de.cache(pages, 4, 1024, 128)
    tables = torch.tensor([[pages - 1, 0], [1, pages - 2]], dtype=torch.int32, device="cuda")
    k, v = normal(g, 1500, 512).to(B), normal(g, 1500, 512).to(B)
    positions = torch.arange(1500, dtype=torch.int32, device="cuda")
    for s in (0, 1):
        de.append(cache, k, v, positions, tables, sequence=torch.full((1500,), s, dtype=torch.int32, device="cuda"))
    q = normal(g, 1, 512).to(B).repeat(2, 1)
    out = de.attend(q, cache, tables, torch.tensor([1500, 1500], dtype=torch.int32, device="cuda"))
    want, bound = attended64(q[0].view(4, 128), k.view(1500, 4, 128).transpose(0, 1), v.view(1500, 4, 128).transpose(0, 1), 128 ** -0.5)
    for r in (0, 1):
        within(out[r].view(4, 128), want, bound, f"row {r}")


# ---- beam ----------------------------------------------------------------------

def check_beam(de, sequences, beams, words, k, dtype, ended=0.0, closed=0.0, pad=0, spread=3.0, first=False):
    g = gen(sequences * 1000 + beams * 100 + words + k)
    rows = sequences * beams
    end = min(2, words - 1)
    for attempt in range(50):       # rows in which 32 bits decide nothing that 64 bits would decide otherwise
        logits = (spread * rows_of(g, rows, words, F, pad, 1 if pad else 0)).to(dtype)
        if closed:
            shut = torch.rand((rows, words), generator=g, device="cuda") < closed
            logits = torch.where(shut, torch.tensor(-INF, dtype=dtype, device="cuda"), logits)
            logits[shut & (torch.rand((rows, words), generator=g, device="cuda") < 0.3)] = NAN
        scores = -8 * torch.rand(rows, generator=g, device="cuda")
        if first:
            scores.view(sequences, beams)[:, 1:] = -INF
        over = (torch.rand(rows, generator=g, device="cuda") < ended).to(torch.uint8) if ended else None
        parents, tokens, best, now, c = chosen64(logits, scores, beams, k, over, end)
        top = c.sort(dim=1, descending=True).values[:, :k + 1]
        gap = top[:, :-1] - top[:, 1:]
        if not ((gap > 0) & (gap < 1e-4)).any():
            break
    else:
        raise AssertionError("no such rows")
    got = de.beam(logits, scores, beams, k=k, ended=over, end=end)
    label = f"{sequences} x {beams} of {words}, {k}"
    assert torch.equal(got.parents, parents), label
    assert torch.equal(got.tokens, tokens), label
    assert torch.equal(got.ended, now), label
    there = best > -INF
    assert torch.equal(got.scores > -INF, there) and bool((got.scores[~there] == -INF).all())
    # the sum of exponentials to 2^-16, its logarithm, three operations on values up to the scores' and logits' size
    size = float(logits[torch.isfinite(logits)].abs().max()) if bool(torch.isfinite(logits).any()) else 0.0
    within(got.scores[there], best[there], 2.0 ** -16 + 2.0 ** -21 * (best[there].abs() + size + 8))


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("words", [1, 2, 7, 8, 9, 100, 255, 257, 1000, 4095, 4096, 4097, 8192, 20001, 65536, 65537, 100003])
def test_beam_words(de, words, dtype):
    check_beam(de, 2, 3, words, 3, dtype)
    check_beam(de, 1, 1, words, 1, dtype)
    check_beam(de, 3, 4, words, 8, dtype, ended=0.3, closed=0.3, pad=3)


@pytest.mark.parametrize("beams, k", [(1, 64), (64, 1), (64, 64), (2, 4), (5, 5), (8, 16), (16, 33)])
def test_beam_widths(de, beams, k):
    check_beam(de, 2, beams, 5000, k, F)
    check_beam(de, 5, beams, 300, k, F, ended=0.5)
    check_beam(de, 2, beams, 9001, k, F, first=True)


@pytest.mark.parametrize("beams, words, k", [(16, 200000, 32), (64, 70000, 64), (9, 131072, 64), (64, 262144, 3), (33, 5000, 64), (2, 1 << 20, 64)])
def test_beam_many_lists(de, beams, words, k):
    """More lists of candidates than a workgroup keeps at once."""
    check_beam(de, 1, beams, words, k, F)
    check_beam(de, 2, beams, words, k, F, ended=0.3, closed=0.05, spread=1.0)


def test_beam_many_equal_lists(de):
    for beams, words, k in ((64, 70000, 64), (40, 200000, 5)):
        got = de.beam(torch.zeros((beams, words), dtype=B, device="cuda"), torch.zeros(beams, device="cuda"), beams, k=k)
        assert got.parents[0].tolist() == [0] * k and got.tokens[0].tolist() == list(range(k))
        z = torch.zeros((beams, words), device="cuda")
        z[:, 7] = -1.0                                      # (every beam's words weigh the same)
        got = de.beam(z, torch.arange(beams, device="cuda") * 0.5, beams, k=k)
        assert got.parents[0].tolist() == [beams - 1] * k and got.tokens[0].tolist() == [i for i in range(k + 1) if i != 7][:k]


def test_beam_many_sequences(de):
    check_beam(de, 200, 2, 501, 2, F, ended=0.2)
    check_beam(de, 33, 4, 12345, 4, F)


def test_beam_equal_values(de):
    """Ties, in one beam and across beams, go to the lowest beam and word; rows of one value take the slow way."""
    for words, k in ((10, 4), (5000, 4), (5000, 64), (70000, 16)):
        for dtype in (B, F):
            logits = torch.zeros((6, words), dtype=dtype, device="cuda")
            got = de.beam(logits, torch.zeros(6, device="cuda"), 3, k=k)
            for s in range(2):
                want = [divmod(i, words) for i in range(k)]
                assert got.tokens[s].tolist() == [t for _, t in want] and got.parents[s].tolist() == [3 * s + w for w, _ in want]
        logits = torch.full((2, words), -3.0, device="cuda")
        logits[1, words // 2:] = 5.0                        # half a row of one value
        got = de.beam(logits, torch.tensor([0.0, 0.0], device="cuda"), 2, k=min(k, words // 2))
        # (a word of row 0 weighs 1 / words, of row 1 about 2 / words)
        assert got.tokens[0].tolist() == list(range(words // 2, words // 2 + min(k, words // 2)))


def test_beam_extremes(de):
    """+inf counts as the largest finite value, the type's lowest is open, a row of closed words has no candidates."""
    low = torch.finfo(F).min
    z = torch.full((4, 50), -INF, device="cuda")
    z[0, 7], z[0, 3] = INF, torch.finfo(F).max
    z[1, 20] = low
    z[2, :] = NAN
    z[3, 4], z[3, 5] = low, low / 2
    got = de.beam(z, torch.tensor([-1.0, -2.0, 0.0, -3.0], device="cuda"), 4, k=8)
    # rows: two equal words at -1 - log 2 each; one word at -2; none; -3 and one too low to count
    assert got.parents[0].tolist()[:4] == [0, 0, 1, 3] and got.tokens[0].tolist()[:4] == [3, 7, 20, 5]
    within(got.scores[0, :4], torch.tensor([-1 - math.log(2), -1 - math.log(2), -2.0, -3.0], dtype=torch.float64, device="cuda"), 2.0 ** -20)
    for i in range(4, 8):
        assert int(got.parents[0, i]) in (-1, 3)
    none = de.beam(z[2:3], torch.zeros(1, device="cuda"), 1, k=2)
    assert none.parents.tolist() == [[-1, -1]] and none.tokens.tolist() == [[-1, -1]] and none.scores.tolist() == [[-INF, -INF]]
    assert none.ended.tolist() == [[0, 0]]
    for bad in (-INF, NAN):
        got = de.beam(torch.zeros((2, 9), device="cuda"), torch.tensor([bad, -1.0], device="cuda"), 2, k=3)
        assert got.parents.tolist() == [[1, 1, 1]] and got.tokens.tolist() == [[0, 1, 2]]


def test_beam_ended(de):
    """An ended beam goes on as it is, with its score; NaN and anything else in its logits are not looked at."""
    z = torch.zeros((3, 1000), device="cuda")
    z[1] = NAN
    z[0, 5] = 20.0
    over = torch.tensor([False, True, False], device="cuda")
    got = de.beam(z, torch.tensor([-1.0, -1.5, -9.0], device="cuda"), 3, ended=over, end=5)
    assert got.parents.tolist() == [[0, 1, 2]] and got.tokens.tolist() == [[5, 5, 0]] and got.ended.tolist() == [[1, 1, 0]]
    assert float(got.scores[0, 1]) == -1.5


def test_beam_company_leaves_bits(de):
    g = gen(20)
    for words in (3000, 50000, 90000):
        z, s = 2 * normal(g, 24, words), -normal(g, 24).abs()
        got = de.beam(z, s, 4)
        for b in (0, 5):
            one = de.beam(z[4 * b:4 * b + 4], s[4 * b:4 * b + 4], 4)
            assert torch.equal(one.scores[0], got.scores[b]) and torch.equal(one.tokens[0], got.tokens[b])


# ---- fork ----------------------------------------------------------------------

@pytest.mark.parametrize("page, heads, dim, max_pages", [(8, 1, 8, 5), (16, 3, 64, 4), (64, 8, 128, 2), (1024, 2, 256, 1)])
def test_fork(de, page, heads, dim, max_pages):
    g = gen(page)
    cap = max_pages * page
    lengths = [0, 1, page - 1, page, min(page + 1, cap), cap - 1, cap, min(3 * page // 2, cap)]
    rows = len(lengths)
    cache, tables = paged(g, lengths, heads, page, dim, max_pages=max_pages, spare=20)
    second = de.Cache(*(t.clone() for t in cache))
    for c in (cache, second):
        for t in c:
            t.copy_(normal(g, *t.shape).to(B))
    used = set(tables.view(-1).tolist())
    free = [p for p in range(cache.keys.shape[0]) if p not in used]
    parents = [7, 0, 0, 3, 2, -1, 6, 5, 1, 4, rows, 2]
    n = len(parents)
    fresh = torch.tensor(free[:n], dtype=torch.int32, device="cuda")
    before = [t.clone() for c in (cache, second) for t in c]
    got_t, got_l = de.fork([cache, second], tables, torch.tensor(lengths, dtype=torch.int32, device="cuda"),
                           torch.tensor(parents, dtype=torch.int32, device="cuda").view(3, 4), fresh)
    want_t, want_l = torch.full((n, max_pages), -1, dtype=torch.int32), []
    for i, p in enumerate(parents):
        live = 0 <= p < rows
        want_l.append(lengths[p] if live else 0)
        if not live:
            continue
        want_t[i] = tables[p].cpu()
        begun, part = divmod(lengths[p], page)
        if begun < max_pages:
            want_t[i, begun] = int(fresh[i])
            for t in before:
                if part:
                    t[int(fresh[i]), :, :part] = t[int(tables[p, begun]), :, :part]
    assert torch.equal(got_t.cpu(), want_t) and got_l.tolist() == want_l
    for t, want in zip([t for c in (cache, second) for t in c], before):
        assert torch.equal(t, want)
    only = de.fork(None, tables, torch.tensor(lengths, dtype=torch.int32, device="cuda"), torch.tensor(parents, dtype=torch.int32, device="cuda"),
                   fresh, page=page)
    assert torch.equal(only[0], got_t) and torch.equal(only[1], got_l)


def test_fork_bad_pages(de):
    """A begun page outside the cache, or a fresh one, is not copied; lengths outside the table count as its ends."""
    g = gen(2)
    cache, tables = paged(g, [20, 20], 1, 8, 16, garbage=1.0)
    before = [t.clone() for t in cache]
    bad = tables.clone()
    bad[0, 2] = -4
    lengths = torch.tensor([20, 20], dtype=torch.int32, device="cuda")
    fresh = torch.tensor([0, cache.keys.shape[0]], dtype=torch.int32, device="cuda")
    t, length = de.fork(cache, bad, lengths, torch.tensor([0, 1], dtype=torch.int32, device="cuda"), fresh)
    assert length.tolist() == [20, 20] and t[1, 2] == fresh[1] and all(torch.equal(a, b) for a, b in zip(cache, before))
    t, length = de.fork(cache, tables, torch.tensor([-5, 1000], dtype=torch.int32, device="cuda"),
                        torch.tensor([0, 1], dtype=torch.int32, device="cuda"), fresh)
    assert length.tolist() == [0, 24] and torch.equal(t[1], tables[1])

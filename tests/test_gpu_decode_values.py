"""The decoding operators' values where few bits or a number's range decide them: weights that nearly cancel, values near the
type's largest, weights that vanish, large logits."""

import math

import pytest
import torch

from tests._decode import ROUND, UNIT, chosen64, within

pytestmark = pytest.mark.gpu

B, F = torch.bfloat16, torch.float32
INF, MOST = float("inf"), torch.finfo(torch.bfloat16).max


@pytest.fixture(scope="module")
def de():
    assert torch.cuda.is_available()
    from paper_2307_04963_amd import decoding
    return decoding


# Capacities for which a workgroup takes a part, a run and a stretch of the keys where there are a thousand rows.
CAPACITIES = [8, 1024, 2048]


def attend(de, scores, values, dim, capacity):
    """Rows of 8 keys: row r's key j has the score scores[r, j] (bf16 values) and values[r, j] in every column -> [rows, dim]."""
    rows = scores.shape[0]
    assert scores.shape == values.shape == (rows, 8)
    cache = de.Cache(*(torch.zeros((rows, 1, 8, dim), dtype=B, device="cuda") for _ in range(2)))
    cache.keys[:, 0, :, 3] = scores.to(B)
    cache.values[:] = values.to(B)[:, None, :, None]
    tables = torch.full((rows, capacity // 8), -1, dtype=torch.int32, device="cuda")
    tables[:, 0] = torch.arange(rows, dtype=torch.int32, device="cuda")
    q = torch.zeros((rows, dim), dtype=B, device="cuda")
    q[:, 3] = 1
    return de.attend(q, cache, tables, torch.full((rows,), 8, dtype=torch.int32, device="cuda"), scale=1.0)


@pytest.mark.parametrize("capacity", CAPACITIES)
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attend_weights_have_24_bits(de, dim, capacity):
    """Two keys of weights 1 and e^s, values -c and 1 with c next to e^s: what is left is as exact as float32's weights are.

    Off by, in units of 2^-24 of the sum of p |v|: the score in base 2, two roundings of 1.45 |s| at most, 2; the exponential, 2^-22: 4;
    the products' and the weights' sums, the quotient and its product, 8.  The others of the eight keys have no weight."""
    s = torch.cat([torch.arange(128, 256, device="cuda") * -(2.0 ** (e - 8)) for e in range(-6, 1)])
    s = torch.cat([s, s[:128]])                             # a thousand rows
    scores = torch.full((len(s), 8), -INF, device="cuda")
    values = torch.zeros_like(scores)
    c = s.double().exp().to(B)
    scores[:, 0], scores[:, 1], values[:, 0], values[:, 1] = 0, s, -c.float(), 1
    p = s.double().exp()
    want = ((p - c.double()) / (1 + p))[:, None].expand(-1, dim)
    size = ((p + c.double()) / (1 + p))[:, None]
    within(attend(de, scores, values, dim, capacity), want, 14 * UNIT * size + ROUND * want.abs())


@pytest.mark.parametrize("capacity", CAPACITIES)
@pytest.mark.parametrize("dim", [64, 72, 128, 256])
def test_attend_values_without_weight(de, dim, capacity):
    """Finite values as large as they come add what their weights say, and nothing without one; infinite ones are."""
    n, no = 0.0, -INF
    big = torch.tensor(3e38).to(B).item()
    rows = [([n, no, no, no, no, no, no, no], [1, big, 0, 0, 0, 0, 0, 0], 1.0),        # a score of -infinity
            ([n, -200, no, no, no, no, no, -200], [1, big, 0, 0, 0, 0, 0, -big], 1.0),  # e^-200
            ([n, -60, no, no, no, no, no, no], [1, big, 0, 0, 0, 0, 0, 0], (1 + big * math.exp(-60)) / (1 + math.exp(-60))),
            ([no] * 8, [big] * 8, 0.0),
            # an infinite value is one, whatever bits its weight has
            ([n, no, no, no, no, no, no, no], [INF, 0, 0, 0, 0, 0, 0, 0], INF),
            ([n, n, -1, -20, no, no, no, no], [1, -INF, 1, 1, 0, 0, 0, 0], -INF),
            ([n, n, -1, -30, no, no, no, no], [1, 1, 1, INF, 0, 0, 0, 0], INF)]
    times = 1024 // len(rows) + 1
    scores, values = (torch.tensor([r[i] for r in rows], device="cuda").repeat(times, 1) for i in (0, 1))
    got = attend(de, scores, values, dim, capacity)
    assert torch.equal(got, got[:len(rows)].repeat(times, 1))
    for r, (_, _, want) in enumerate(rows):
        # (a score of 60 is off by up to 120 * 2^-24 where it is taken to base 2, and so is its weight)
        bound = 0.0 if want in (1.0, 0.0, INF, -INF) else want * (ROUND + 2.0 ** -15)
        assert all(v == want or abs(v - want) <= bound for v in got[r].tolist()), (r, got[r, 0].item(), want)


@pytest.mark.parametrize("capacity", CAPACITIES)
@pytest.mark.parametrize("dim", [64, 72, 128, 256])
def test_attend_largest_values(de, dim, capacity):
    """Sums of the type's largest values do not pass its range: a mean of equal values is that value."""
    n, no = 0.0, -INF
    rows = [([n] * 8, [MOST] * 8, MOST), ([n, n, no, no, no, no, no, no], [-MOST, -MOST, 0, 0, 0, 0, 0, 0], -MOST),
            ([n] * 8, [MOST, -MOST] * 4, 0.0), ([n, n, n, no, no, no, no, n], [MOST, MOST, -MOST, 0, 0, 0, 0, MOST], MOST / 2)]
    scores, values = (torch.tensor([r[i] for r in rows], device="cuda").repeat(256, 1) for i in (0, 1))
    got = attend(de, scores, values, dim, capacity)
    for r, (_, _, want) in enumerate(rows):
        assert bool((got[r::len(rows)] == want).all()), (r, got[r, 0].item(), want)


@pytest.mark.parametrize("q_heads", [1, 2, 20])
def test_attend_many_largest_values(de, q_heads):
    """5000 and 70000 keys of the largest value, more than a stretch: their mean is that value."""
    for dim, length in ((64, 5000), (128, 5000), (64, 70000)):
        pages = length // 8
        cache = de.Cache(torch.zeros((pages, 1, 8, dim), dtype=B, device="cuda"), torch.full((pages, 1, 8, dim), MOST, dtype=B, device="cuda"))
        tables = torch.arange(pages, dtype=torch.int32, device="cuda").repeat(3, 1)
        lengths = torch.tensor([length, length - 1, 1], dtype=torch.int32, device="cuda")
        assert bool((de.attend(torch.ones((3, q_heads * dim), dtype=B, device="cuda"), cache, tables, lengths) == MOST).all())


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("low, high", [(1e5, 1e6), (1e6, 1e9), (1.4e9, 3e9), (3e9, 1e12), (1e29, 1e31), (1e37, 3e38)])
def test_beam_large_logits(de, low, high, sign, dtype):
    """Rows whose largest logit is far above the others: it alone is likely, its value is the beam's score."""
    g = torch.Generator(device="cuda").manual_seed(int(low) % 1000003 + sign)
    rows, words = 4096, 300
    top = sign * torch.exp(math.log(low) + (math.log(high) - math.log(low)) * torch.rand(rows, generator=g, device="cuda"))
    at = torch.randint(0, words, (rows,), generator=g, device="cuda")
    less = torch.rand((rows, words), generator=g, device="cuda") * 0.4 + 0.05           # by 5 to 45 percent
    logits = (top[:, None] - less * top.abs()[:, None]).to(dtype)
    logits.scatter_(1, at[:, None], top.to(dtype)[:, None])
    scores = -9 * torch.rand(rows, generator=g, device="cuda")
    got = de.beam(logits, scores, 1, k=1)
    assert torch.equal(got.tokens[:, 0].long(), at) and torch.equal(got.parents[:, 0].long(), torch.arange(rows, device="cuda"))
    # The others' exponentials are 0, the logarithm of 1 is.  Where the largest is taken around its rounded product, its own exponential
    # and what puts that right are each 2^-22 off, their product 2^-24, so the logarithm is off by 2^-21 + 2^-24 at most, and
    # the two sums that it enters by a rounding each.
    within(got.scores[:, 0], scores.double(), 2.0 ** -21 + UNIT + 2 * UNIT * scores.double().abs())


@pytest.mark.parametrize("words", [700, 5000, 70001])
@pytest.mark.parametrize("offset", [0.0, -1000.0, 1e5, 3e6])
def test_beam_scores(de, offset, words):
    """Scores to the roundings of 32 bits, also where all of a row's logits are large.

    In units of 2^-24: the exponentials 4, their arguments 0.7 log2(words) on the average: 12, their sum over 32 values of a lane, the lanes,
    the waves and the segments 64; the logarithm and the terms' roundings 2 of the logarithm (24) and 4 of the result and of the
    logit below the largest, which is less: 8 of the result."""
    g = torch.Generator(device="cuda").manual_seed(words)
    beams, k = 4, 6
    for _ in range(50):
        logits = 3 * torch.randn((5 * beams, words), generator=g, device="cuda") + offset
        scores = -8 * torch.rand(5 * beams, generator=g, device="cuda")
        parents, tokens, best, _, c = chosen64(logits, scores, beams, k)
        top = c.sort(dim=1, descending=True).values[:, :k + 1]
        gap = top[:, :-1] - top[:, 1:]
        if not ((gap > 0) & (gap < 1e-4)).any():
            break
    else:
        raise AssertionError("no such rows")
    got = de.beam(logits, scores, beams, k=k)
    assert torch.equal(got.parents, parents) and torch.equal(got.tokens, tokens)
    within(got.scores, best, UNIT * (104 + 8 * best.abs()))

"""Definitions of the decoding operators in 64 bits, and bounds on the kernels' distance from them.

Bounds, from the formulas: a value stored in bf16 is off by at most 2^-8 of itself; one operation in 32 bits by
2^-24 of its result, a hardware exponential in base 2 by 2^-22.  A pair's rotation: the angle is 64 bits up to a
rounding of 2^-24 of at most pi / 4, sine and cosine 2^-22 with their polynomials' roundings, then three operations: TURN = 2^-20 of
|a| + |b|.
"""

import math

import torch

ROUND = 2.0 ** -8
UNIT = 2.0 ** -24
TURN = 2.0 ** -20


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def within(got, want, bound, what=""):
    got = got.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert not torch.isnan(got).any(), what
    off = (got - want).abs() - bound
    assert off.numel() == 0 or float(off.max()) <= 0, (what, float(off.max()), float((got - want).abs().max()))


def turned64(x, positions, f, layout, dim, adjoint=False, magnitude=1.0):
    """(rotation of x [n, heads * dim] in 64 bits, its bound before the last rounding)."""
    x = x.double().reshape(x.shape[0], -1, dim)
    half = len(f)
    t = (positions.double()[:, None] * f.double())[:, None]
    c, s = t.cos(), t.sin() * (-1 if adjoint else 1)
    first, second = (slice(0, half), slice(half, 2 * half)) if layout == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    a, b = x[..., first], x[..., second]
    y, e = x.clone(), torch.zeros_like(x)
    y[..., first], y[..., second] = magnitude * (a * c - b * s), magnitude * (b * c + a * s)
    e[..., first] = e[..., second] = TURN * abs(magnitude) * (a.abs() + b.abs())
    return y.flatten(1), e.flatten(1)


def paged(g, lengths, heads, page, dim, max_pages=None, spare=2, garbage=float("nan")):
    """(cache filled with `garbage`, tables): pages of sequences of `lengths` tokens, shuffled."""
    from paper_2307_04963_amd import decoding as de
    need = [-(-n // page) for n in lengths]
    pages = sum(need) + spare
    order = torch.randperm(pages, generator=g, device="cuda").int()
    tables = torch.full((len(lengths), max_pages or max(1, max(need))), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, k in enumerate(need):
        tables[i, :k] = order[at:at + k]
        at += k
    return de.Cache(*(torch.full((pages, heads, page, dim), garbage, dtype=torch.bfloat16, device="cuda") for _ in range(2))), tables


def dense(t, table, n):
    """The first n tokens [heads, n, dim] of a table's pages."""
    page = t.shape[2]
    pages = table[:-(-n // page)].long() if n else table[:0].long()
    return t[pages].transpose(0, 1).reshape(t.shape[1], -1, t.shape[3])[:, :n]


def put(t, table, values):
    """values [heads, n, dim] into the first places of a table's pages."""
    page = t.shape[2]
    for i in range(0, values.shape[1], page):
        part = values[:, i:i + page]
        t[int(table[i // page]), :, :part.shape[1]] = part


def attended64(q, k, v, scale, here=None):
    """One row: q [q_heads, dim], k, v [heads, n, dim], here [n] bool -> (out [q_heads, dim], bound)."""
    heads, n, dim = k.shape
    q = q.double().view(heads, -1, dim)
    if here is not None:
        k, v = k[:, here], v[:, here]
    k, v = k.double(), v.double()
    if not k.shape[1]:
        return torch.zeros_like(q).flatten(0, 1), torch.zeros_like(q).flatten(0, 1)
    z = torch.matmul(q, k.transpose(1, 2).contiguous()) * scale
    p = torch.softmax(z, 2)
    out = torch.matmul(p, v)
    # A score: dim products summed in 32 bits, scaled and taken to base 2 (three roundings of a value up to 3 / 2 of it); what it is
    # off by is the weight's relative error.  The weight: its exponential, 16 bits in two terms.  Sums: at most n roundings, which
    # do not all fall one way (2^-16 up to 2^14 keys, more with their number).
    size = torch.matmul(q.abs(), k.abs().transpose(1, 2).contiguous()) * abs(scale)
    off = (size * (dim + 3) * UNIT * 1.5).amax(2, keepdim=True) + 2.0 ** -22 + 2.0 ** -15 + 2.0 ** -16 * max(1.0, k.shape[1] / 2 ** 14)
    bound = torch.matmul(p, v.abs()) * 2 * off
    return out.flatten(0, 1), bound.flatten(0, 1) + ROUND * out.abs().flatten(0, 1)


def chosen64(logits, scores, beams, k, ended=None, end=-1):
    """(parents, tokens, scores, ended) by the definition; logits [rows, words], +inf as the largest finite value."""
    z = logits.double()
    z = torch.where(torch.isnan(z), -math.inf, z).clamp(max=3.4028234663852886e38)
    rows, words = z.shape
    live = (scores == scores) & (scores > -math.inf)
    c = scores.double()[:, None] + torch.log_softmax(z, 1)
    c = torch.where(torch.isnan(c) | ~live[:, None], -math.inf, c)
    if ended is not None:
        kept = torch.full_like(c, -math.inf)
        kept[:, end] = torch.where(live, scores.double(), -math.inf)
        c = torch.where(ended[:, None] != 0, kept, c)
    c = c.view(rows // beams, beams * words)
    order = torch.argsort(c, dim=1, descending=True, stable=True)[:, :k]
    best = c.gather(1, order)
    if order.shape[1] < k:
        pad = k - order.shape[1]
        order = torch.cat([order, order.new_zeros(order.shape[0], pad)], 1)
        best = torch.cat([best, best.new_full((best.shape[0], pad), -math.inf)], 1)
    none = best == -math.inf
    parents = torch.where(none, -1, order // words + beams * torch.arange(rows // beams, device=c.device)[:, None])
    tokens = torch.where(none, -1, order % words)
    over = ~none & ((tokens == end) if ended is None else ((tokens == end) | (ended[parents.clamp(min=0)] != 0)))
    return parents.int(), tokens.int(), best, over.to(torch.uint8), c

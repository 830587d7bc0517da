"""The token operators on the GPU against their definitions in 64 bits.

Bounds, from the formulas: a value stored in bf16 is off by at most 2^-8 of
itself (half a unit in the last of 8 significant bits, against the least value
of a binade); a 32-bit sum of K products by SUM of the sum of their magnitudes, SUM =
2^-16 (K up to 2^14 roundings of 2^-24 that do not all fall one way); functions
of one value by FN = 2^-20 of its magnitude.  An intermediate's bound travels
through what follows by the largest slope of it (1.13 for GELU, 1.1 for SiLU).
"""

import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

ROUND = 2.0 ** -8
SUM = 2.0 ** -16
FN = 2.0 ** -20


@pytest.fixture(scope="module")
def ex():
    assert torch.cuda.is_available()
    from paper_2307_04963_amd import experts
    return experts


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def within(got, want, bound, what=""):
    got = got.double()
    assert got.shape == want.shape
    assert torch.equal(torch.isfinite(got), torch.isfinite(want)), what
    fine = torch.isfinite(want)
    off = ((got - want).abs() - bound)[fine]
    assert off.numel() == 0 or float(off.max()) <= 0, (what, float(off.max()), float((got - want).abs()[fine].max()))


# ---- norm ---------------------------------------------------------------------

def norm64(v, kind, w, b, eps, err):
    """The norm of v in 64 bits, and how far 32 bits may be off for v known to within err."""
    if kind == "none":
        return v, err
    w = 1.0 if w is None else w.double()
    b = 0.0 if b is None else b.double()
    mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    c = v - mean
    inv = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + eps)
    out = c * inv * w + b
    big = (v.abs() + v.abs().mean(1, keepdim=True)) * inv
    # the statistics of values that are off by err, and 16 roundings on the way
    return out, (16 * 2.0 ** -24) * (big * abs(w) + abs(b)) + (err + err.mean(1, keepdim=True) * (1 + (c * inv).abs())) * inv * abs(w) * 2


def check_norm(ex, n, d, xt, yt, ut, post, pre, gate_act, rows, chan, bias, alpha, pad=0, skew=0, eps=1e-6, seed=0):
    g = gen(seed + n * 131 + d)
    def mat(dtype):
        full = normal(g, n, d + pad + skew) * 2 + 0.5
        return full.to(dtype)[:, skew:skew + d]
    vec = lambda on: 1 + 0.3 * normal(g, d) if on else None  # noqa: E731
    x = mat(xt)
    y = mat(yt) if post is not None else None
    gate = mat(yt) if gate_act else None
    row = None
    if rows:
        row = torch.rand(n, generator=g, device="cuda")
        row[torch.rand(n, generator=g, device="cuda") < 0.4] = 0
        y[row == 0] = float("nan")
        if gate is not None:
            gate[row == 0] = float("inf")
    cs = 0.2 * normal(g, d) if chan else None
    pw, pb = (vec(post != "none"), vec(bias and post != "none")) if post else (None, None)
    qw, qb = vec(pre != "none"), vec(bias and pre != "none")
    h, u = ex.norm(x, y, post=post or "none", post_weight=pw, post_bias=pb, gate=gate, gate_act=gate_act or "none", row_gate=row,
                   channel_scale=cs, residual_scale=alpha, pre=pre, pre_weight=qw, pre_bias=qb, eps=eps, u_dtype=ut)
    h64 = x.double() * alpha
    err = 2.0 ** -23 * h64.abs()
    if y is not None:
        z, e = norm64(torch.nan_to_num(y.double()) if rows else y.double(), post, pw, pb, eps, torch.zeros_like(h64))
        f = torch.ones_like(z)
        if gate is not None:
            gd = gate.double() if row is None else torch.where(row[:, None] == 0, torch.zeros_like(gate), gate).double()
            f = {"none": gd, "sigmoid": torch.sigmoid(gd), "silu": gd * torch.sigmoid(gd)}[gate_act]
        if cs is not None:
            f = f * cs.double()
        if row is not None:
            f = f * row.double()[:, None]
        z, e = z * f, (e + z.abs() * FN) * f.abs()
        if row is not None:
            z, e = torch.where(row[:, None] == 0, 0.0, z), torch.where(row[:, None] == 0, 0.0, e)
        h64, err = h64 + z, err + e + 2.0 ** -23 * z.abs()
    label = f"n={n} d={d}"
    within(h, h64, err + (ROUND * h64.abs() if xt == torch.bfloat16 else 0), "h " + label)
    if pre == "none":
        assert u is None
        return
    u64, uerr = norm64(h64, pre, qw, qb, eps, err)
    within(u, u64, uerr + (ROUND * u64.abs() if ut == torch.bfloat16 else 0), "u " + label)


B, F = torch.bfloat16, torch.float32


@pytest.mark.parametrize("d", [1, 7, 8, 64, 65, 512, 520, 1003, 1024, 2048, 2056, 4096, 5000, 8192, 8200, 16384, 20001, 32768])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_norm_widths(ex, d, kind):
    n = 5 if d > 4096 else 37
    check_norm(ex, n, d, B, B, B, kind, kind, None, False, False, False, 1.0)
    check_norm(ex, n, d, F, B, F, kind, kind, "sigmoid", True, True, True, 0.5)


@pytest.mark.parametrize("xt, yt, ut", [(B, B, B), (B, B, F), (F, F, B), (B, F, F), (F, B, B)])
@pytest.mark.parametrize("post, pre", [("none", "rms"), ("rms", "none"), ("layer", "rms"), ("none", "none")])
def test_norm_types_and_parts(ex, xt, yt, ut, post, pre):
    for gate_act, rows, chan in ((None, False, True), ("silu", True, False), ("none", False, False)):
        check_norm(ex, 19, 640, xt, yt, ut, post, pre, gate_act, rows, chan, True, 0.75)


@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 1535, 1536, 1537, 6200])
def test_norm_rows(ex, n):
    check_norm(ex, n, 256, B, B, B, "rms", "layer", None, True, False, False, 1.0)
    if n < 2000:
        check_norm(ex, n, 2304, B, B, B, "layer", "rms", None, False, False, False, 1.0)


@pytest.mark.parametrize("pad, skew", [(8, 0), (3, 0), (8, 1), (0, 8)])
def test_norm_strided_and_misaligned_rows(ex, pad, skew):
    check_norm(ex, 29, 512, B, B, B, "rms", "rms", "silu", True, True, True, 1.0, pad=pad, skew=skew)
    check_norm(ex, 29, 1024, F, B, F, "layer", "layer", None, False, False, False, 1.0, pad=pad, skew=skew)


def test_norm_without_a_block(ex):
    check_norm(ex, 21, 768, B, B, B, None, "rms", None, False, False, False, 1.0)
    check_norm(ex, 21, 768, B, B, B, None, "layer", None, False, False, True, 0.5)
    x = normal(gen(1), 4, 64).bfloat16()
    h, u = ex.norm(x)
    assert h is x and u is None
    h, u = ex.norm(x, pre="rms")
    assert h is x and u.shape == x.shape


def test_norm_in_place_and_empty(ex):
    g = gen(3)
    x, y = normal(g, 3000, 1024).bfloat16(), normal(g, 3000, 1024).bfloat16()
    want = ex.norm(x, y, post="rms", pre="rms")
    for h in ("x", "y"):
        a, b = x.clone(), y.clone()
        got = ex.norm(a, b, post="rms", pre="rms", h=a if h == "x" else b)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    h, u = ex.norm(x[:0], y[:0], post="rms", pre="rms")
    assert h.shape == u.shape == (0, 1024)


def test_norm_of_constant_and_huge_rows(ex):
    # a constant row's layer norm is its bias; all values far from zero: the variance comes from the centred values
    x = torch.full((3, 512), 1000.0, device="cuda")
    b = normal(gen(5), 512)
    _, u = ex.norm(x, pre="layer", pre_bias=b, u_dtype=F)
    assert torch.allclose(u, b.expand(3, 512), rtol=0, atol=1e-6)
    v = (normal(gen(6), 64, 512) + 4096).float()
    _, u = ex.norm(v, pre="layer", u_dtype=F)
    w = v.double()
    w = w - w.mean(1, keepdim=True)
    w = w / torch.sqrt((w * w).mean(1, keepdim=True) + 1e-6)
    assert float((u.double() - w).abs().max()) < 4096 * 2.0 ** -22


# ---- route ----------------------------------------------------------------------

def route_by_hand(logits, k, score, bias, groups, top_groups, mask, renorm, scale):
    """Row by row on the host, in 64 bits from 32-bit logits."""
    z = logits.float().cpu().numpy().astype(np.float64)
    n, E = z.shape
    b = np.zeros(E) if bias is None else bias.cpu().numpy().astype(np.float64)
    ids, w = np.full((n, k), -1, np.int64), np.zeros((n, k))
    for r in range(n):
        if mask is not None and not mask[r]:
            continue
        up = ~(np.isnan(z[r]) | (z[r] == -np.inf)) & ~(np.isnan(b) | (b == -np.inf))
        row = np.where(np.isposinf(z[r]), 3.4028234663852886e38, np.where(np.isnan(z[r]) | (z[r] == -np.inf), -np.inf, z[r]))
        with np.errstate(over="ignore", invalid="ignore"):
            if score == "sigmoid":
                p = 1 / (1 + np.exp(-row))
            else:
                e = np.where(row == -np.inf, 0, np.exp(row - row.max()))
                p = e / e.sum() if e.sum() > 0 else e
        v = np.where(up, p + b, -np.inf)
        if groups > 1:
            size, best = E // groups, []
            for q in range(groups):
                s = np.sort(v[q * size:(q + 1) * size])[::-1]
                best.append(s[0] if len(s) < 2 or s[1] == -np.inf else s[0] + s[1])
            kept = sorted(range(groups), key=lambda q: (-best[q], q))[:top_groups]
            for q in range(groups):
                if q not in kept:
                    v[q * size:(q + 1) * size] = -np.inf
        order = sorted((e for e in range(E) if v[e] > -np.inf), key=lambda e: (-v[e], e))[:k]
        for j, e in enumerate(order):
            ids[r, j], w[r, j] = e, p[e]
        if renorm:
            w[r] = w[r] / w[r].sum() if w[r].sum() > 0 else 0
        w[r] *= scale
    return ids, w


def partition_by_hand(ids, E):
    n, k = ids.shape
    order, offsets, slots = [], [0], np.full(n * k, -1, np.int64)
    flat = ids.reshape(-1)
    for e in range(E):
        order += list(np.flatnonzero(flat == e))
        offsets.append(len(order))
    slots[order] = np.arange(len(order))
    return np.array(offsets), np.array(order + [-1] * (n * k - len(order))), slots.reshape(n, k)


def check_route(ex, logits, k, score="softmax", bias=None, groups=1, top_groups=1, mask=None, renorm=True, scale=1.0):
    got = ex.route(logits, k, score=score, bias=bias, groups=groups, top_groups=top_groups, mask=mask, renormalise=renorm, scale=scale)
    ids, w = route_by_hand(logits, k, score, bias, groups, top_groups, None if mask is None else mask.cpu().numpy(), renorm, scale)
    np.testing.assert_array_equal(got.ids.cpu().numpy(), ids)
    np.testing.assert_allclose(got.weights.cpu().numpy(), w, rtol=4e-6, atol=1e-30)
    offsets, order, slots = partition_by_hand(ids, logits.shape[1])
    np.testing.assert_array_equal(got.offsets.cpu().numpy(), offsets)
    np.testing.assert_array_equal(got.order.cpu().numpy(), order)
    np.testing.assert_array_equal(got.slots.cpu().numpy(), slots)
    return got


def apart(n, E, seed, top=4.0):
    """Logits whose every row is a shuffle of values at least top / E apart, not symmetric about 0 (sigmoids of opposite
    values add up to 1, a tie of group scores): no choice hangs on a rounding."""
    rng = np.random.default_rng(seed)
    step = np.linspace(-top, 1.13 * top, E)
    return torch.from_numpy(np.stack([rng.permutation(step) for _ in range(n)]).astype(np.float32)).cuda()


@pytest.mark.parametrize("E, k", [(1, 1), (2, 2), (7, 3), (16, 16), (60, 4), (64, 8), (65, 2), (128, 6), (160, 8), (256, 8), (257, 5),
                                  (512, 8), (1000, 32), (1024, 8)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_sizes(ex, E, k, score):
    for n in (1, 63, 64, 65, 200):
        check_route(ex, apart(n, E, n + E), k, score, renorm=n != 63, scale=2.5)


@pytest.mark.parametrize("E, groups, top_groups, k", [(8, 4, 2, 3), (64, 8, 3, 6), (256, 8, 4, 8), (60, 4, 1, 15), (160, 10, 3, 6),
                                                      (64, 64, 5, 4), (1024, 16, 7, 8)])
def test_route_groups(ex, E, groups, top_groups, k):
    k = min(k, top_groups * (E // groups))
    logits = apart(130, E, E + groups)
    # a bias on the same grid, half a step aside, keeps the values apart for group sums too
    bias = torch.from_numpy(np.random.default_rng(groups).permutation(np.linspace(-0.3, 0.3, E)).astype(np.float32)).cuda()
    check_route(ex, logits, k, "sigmoid", bias, groups, top_groups)
    check_route(ex, logits, k, "softmax", None, groups, top_groups)


def test_route_ties_go_to_the_lowest_index(ex):
    z = torch.zeros((70, 48), device="cuda")
    got = check_route(ex, z, 5)
    assert got.ids[0].tolist() == [0, 1, 2, 3, 4]
    z[:, 40] = 1.0
    z[:, 17] = 1.0
    assert check_route(ex, z.bfloat16(), 4, "sigmoid").ids[3].tolist() == [17, 40, 0, 1]
    # equal groups: the first ones
    assert check_route(ex, torch.zeros((3, 64), device="cuda"), 4, groups=8, top_groups=2).ids[2].tolist() == [0, 1, 2, 3]


def test_route_masked_rows_and_closed_experts(ex):
    inf = float("inf")
    for E, groups, top_groups in ((32, 1, 1), (32, 4, 2), (256, 8, 4)):
        z = apart(150, E, 5)
        rng = np.random.default_rng(E)
        z[torch.from_numpy(rng.random((150, E)) < 0.5).cuda()] = -inf
        z[3] = -inf                                   # no expert is open
        z[4, 1:] = -inf                               # one is
        z[4, 0] = 0.25
        z[5] = float("nan")
        z[6, 7] = float("nan")
        z[7, E - 1] = inf                             # the largest finite value
        mask = torch.from_numpy((rng.random(150) < 0.7).astype(np.uint8)).cuda()
        mask[2:9] = 1
        for score in ("softmax", "sigmoid"):
            got = check_route(ex, z, 4, score, None, groups, top_groups, mask)
            assert got.ids[3].tolist() == [-1] * 4 and got.weights[3].tolist() == [0.0] * 4
            assert got.ids[4].tolist() == [0, -1, -1, -1]
            assert got.ids[7, 0] == E - 1
    # every row masked: an empty partition
    got = check_route(ex, apart(100, 8, 1), 2, mask=torch.zeros(100, dtype=torch.uint8, device="cuda"))
    assert got.offsets.tolist() == [0] * 9
    # the type's lowest value is not closed: it is chosen after all others
    z = torch.full((2, 8), torch.finfo(torch.float32).min, device="cuda")
    z[:, 3] = 0.0
    assert check_route(ex, z, 3).ids[1].tolist() == [3, 0, 1]
    # sigmoids that are all 0 have no weights to renormalise
    got = ex.route(z.clamp(max=-200.0), 2, score="sigmoid")
    assert got.ids.tolist() == [[0, 1], [0, 1]] and got.weights.abs().max() == 0


def test_route_strides_types_and_closed_bias(ex):
    wide = apart(90, 70, 9).repeat(1, 2)
    check_route(ex, wide[:, 5:69], 4)
    check_route(ex, wide.bfloat16()[:, 5:69].float().bfloat16(), 1, "sigmoid")
    bias = torch.zeros(64, device="cuda")
    bias[10] = -float("inf")
    bias[11] = float("nan")
    got = check_route(ex, apart(90, 64, 2), 8, "softmax", bias)
    assert not ((got.ids == 10) | (got.ids == 11)).any()


def test_route_many_rows(ex):
    # thousands of blocks of rows, a crowded and an empty expert
    n, E, k = 70001, 32, 4
    z = normal(gen(8), n, E).bfloat16().float()
    z = z + torch.arange(E, device="cuda") * 2.0 ** -12          # no ties
    z[:, 5] = 30.0
    z[:, 9] = -float("inf")
    got = ex.route(z, k)
    ids = z.sort(dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(got.ids.long(), ids)
    flat = ids.reshape(-1)
    order = torch.argsort(flat, stable=True)
    assert torch.equal(got.order.long(), order)
    counts = torch.bincount(flat, minlength=E)
    assert torch.equal(got.offsets[1:].long(), counts.cumsum(0)) and counts[5] == n and counts[9] == 0
    assert torch.equal(got.slots.reshape(-1).long()[order], torch.arange(n * k, device="cuda"))


def test_route_without_a_partition_and_without_rows(ex):
    z = apart(100, 16, 3)
    a, b = ex.route(z, 3), ex.route(z, 3, partition=False)
    assert torch.equal(a.ids, b.ids) and torch.equal(a.weights, b.weights) and b.order is None
    e = ex.route(z[:0], 3)
    assert e.ids.shape == (0, 3) and e.offsets.tolist() == [0] * 17


# ---- linear -----------------------------------------------------------------------

ACT64 = {"none": lambda v: v, "relu": lambda v: v.clamp(min=0), "gelu": lambda v: v * 0.5 * torch.special.erfc(-v / math.sqrt(2)),
         "silu": lambda v: v * torch.sigmoid(v)}
SLOPE = {"none": 1.0, "relu": 1.0, "gelu": 1.13, "silu": 1.1}


def layer64(x, err, w, b, gw, gb, act):
    """One layer in 64 bits of inputs known to within err, and its own bound in 32 bits."""
    def product(w, b):
        wd = w.double().t().contiguous()
        v = x @ wd + (0.0 if b is None else b.double())
        return v, SUM * (x.abs() @ wd.abs() + (0.0 if b is None else b.double().abs())) + err @ wd.abs()
    v, e = product(w, b)
    if gw is None:
        return ACT64[act](v), SLOPE[act] * e + FN * v.abs() + 1e-6 * (act != "none")
    q, eq = product(gw, gb)
    a = ACT64[act](q)
    ea = SLOPE[act] * eq + FN * q.abs() + 1e-6 * (act != "none")
    return v * a, v.abs() * ea + a.abs() * e + e * ea


def check_linear(ex, m, K, N, act="none", gated=False, bias=False, residual=False, out=B, pad=0, skew=0, seed=0, in_place=False):
    g = gen(seed + m * 7 + K * 3 + N)
    x = normal(g, m, K + pad + skew).bfloat16()[:, skew:skew + K]
    w, gw = (normal(g, N, K) / math.sqrt(K)).bfloat16(), (normal(g, N, K) / math.sqrt(K)).bfloat16() if gated else None
    b, gb = (0.3 * normal(g, N) if bias else None), (0.3 * normal(g, N) if bias and gated else None)
    r = normal(g, m, N + pad).bfloat16()[:, :N] if residual else None
    want, err = layer64(x.double(), torch.zeros((m, K), dtype=torch.float64, device="cuda"), w, b, gw, gb, act)
    if r is not None:
        want = want + r.double()
        err = err + 2.0 ** -23 * want.abs()
    got = ex.linear(x, ex.pack(w, gw), bias=b, gate_bias=gb, act=act, residual=r, out_dtype=out, out=r if in_place else None)
    assert got.dtype == out
    within(got, want, err + (ROUND * want.abs() if out == B else 2.0 ** -23 * want.abs()), f"m={m} K={K} N={N}")


@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 32, 33, 64, 65, 127, 128, 129, 256, 257, 511, 513, 1000])
def test_linear_rows(ex, m):
    check_linear(ex, m, 192, 160, "gelu", bias=True, residual=True)
    check_linear(ex, m, 192, 160, "silu", gated=True, bias=True)


@pytest.mark.parametrize("K", [1, 7, 8, 31, 32, 33, 63, 64, 65, 72, 127, 128, 136, 200, 1000, 1003, 4096])
@pytest.mark.parametrize("m", [3, 40, 600])
def test_linear_inputs(ex, K, m):
    check_linear(ex, m, K, 96, "relu", bias=True)


@pytest.mark.parametrize("N", [1, 3, 8, 31, 32, 33, 100, 127, 128, 255, 256, 257, 777])
@pytest.mark.parametrize("m", [5, 300, 700])
def test_linear_outputs(ex, N, m):
    check_linear(ex, m, 128, N, "silu", bias=True, residual=True, out=F)
    check_linear(ex, m, 128, N, "gelu", gated=True, residual=True)


@pytest.mark.parametrize("m", [2, 24, 100, 900])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
def test_linear_epilogues(ex, m, act):
    for gated in (False, True):
        for out in (B, F):
            check_linear(ex, m, 264, 136, act, gated, bias=True, residual=True, out=out)
            check_linear(ex, m, 264, 136, act, gated, out=out)


@pytest.mark.parametrize("m", [4, 130, 600])
def test_linear_strides_alignment_and_in_place(ex, m):
    for pad, skew in ((8, 0), (5, 0), (0, 8), (7, 1)):
        check_linear(ex, m, 256, 192, "gelu", residual=True, pad=pad, skew=skew)
        check_linear(ex, m, 256, 192, "gelu", residual=True, out=F, pad=pad, skew=skew)
    check_linear(ex, m, 256, 192, "relu", residual=True, in_place=True, pad=8)


def test_linear_large(ex):
    check_linear(ex, 2049, 2056, 1032, "silu", gated=True, bias=True, residual=True)
    check_linear(ex, 4096, 1024, 4096, "gelu", bias=True)


def test_linear_does_not_touch_what_lies_around(ex):
    g = gen(4)
    x, w = normal(g, 70, 128).bfloat16(), normal(g, 45, 128).bfloat16()
    for m in (9, 70):
        for dtype in (B, F):
            y = torch.full((m + 2, 64), 7.0, dtype=dtype, device="cuda")
            ex.linear(x[:m], ex.pack(w), out=y[1:m + 1, 3:48])
            y[1:m + 1, 3:48] = 7.0
            assert bool((y == 7.0).all())


def test_linear_infinite_inputs_stay_in_their_rows(ex):
    g = gen(11)
    w = normal(g, 50, 100).bfloat16()
    for m in (6, 300):
        x = normal(g, m, 100).bfloat16()
        want = ex.linear(x, ex.pack(w))
        x[2, 99], x[4, 3] = float("inf"), float("nan")
        got = ex.linear(x, ex.pack(w))
        rest = torch.ones(m, dtype=torch.bool, device="cuda")
        rest[2] = rest[4] = False
        assert torch.equal(got[rest], want[rest])
        assert bool(torch.isinf(got[2]).all()) and bool(torch.isnan(got[4]).all())


# ---- experts ------------------------------------------------------------------------

def check_experts(ex, n, E, k, d, f, act="silu", gated=True, bias=False, residual=True, skew=0.0, masked=0.0, pad=0, seed=0, ids=None):
    g = gen(seed + n * 11 + E * 5 + d + f)
    x = normal(g, n, d + pad).bfloat16()[:, :d]
    mk = lambda a, b: (normal(g, E, a, b) / math.sqrt(b)).bfloat16()  # noqa: E731
    w, gw, w2 = mk(f, d), mk(f, d) if gated else None, mk(d, f)
    b, gb, b2 = (0.3 * normal(g, E, f), 0.3 * normal(g, E, f) if gated else None, 0.3 * normal(g, E, d)) if bias else (None, None, None)
    r = normal(g, n, d + pad).bfloat16()[:, :d] if residual else None
    if ids is None:
        ids = torch.topk(normal(g, n, E) + skew * normal(g, E), k).indices
        ids[torch.rand(n, generator=g, device="cuda") < masked] = -1
    weights = torch.where(ids < 0, 0.0, torch.rand((n, k), generator=g, device="cuda") + 0.1)
    off, order, slots = (torch.from_numpy(v.astype(np.int32)).cuda() for v in partition_by_hand(ids.cpu().numpy(), E))
    routing = ex.Routing(ids.int(), weights, off, order, slots)
    got = ex.experts(x, routing, ex.pack(w, gw), ex.pack(w2), act=act, bias=b, gate_bias=gb, bias2=b2, residual=r)
    want = torch.zeros((n, d), dtype=torch.float64, device="cuda") if r is None else r.double()
    err = torch.zeros_like(want)
    of = lambda t, e: None if t is None else t[e]  # noqa: E731
    for e in range(E):
        t, j = torch.where(ids == e)
        if len(t) == 0:
            continue
        v, ve = layer64(x[t].double(), torch.zeros((len(t), d), dtype=torch.float64, device="cuda"), w[e], of(b, e), of(gw, e), of(gb, e), act)
        v, ve = layer64(v, ve + ROUND * v.abs(), w2[e], of(b2, e), None, None, "none")
        ve = ve + ROUND * v.abs()
        c = weights[t, j].double()[:, None]
        want.index_add_(0, t, c * v)
        err.index_add_(0, t, c * ve + 2.0 ** -22 * c * v.abs())
    within(got, want, err + ROUND * (want.abs() + err), f"n={n} E={E} k={k} d={d} f={f}")
    return got


@pytest.mark.parametrize("n", [1, 2, 3, 16, 17, 40, 100, 257, 600])
def test_experts_rows(ex, n):
    check_experts(ex, n, 8, 2, 128, 96)
    check_experts(ex, n, 4, 1, 64, 160, "gelu", gated=False, bias=True, masked=0.3)


@pytest.mark.parametrize("E, k", [(1, 1), (2, 2), (8, 8), (60, 4), (64, 8), (65, 3), (128, 6), (300, 32)])
def test_experts_numbers(ex, E, k):
    check_experts(ex, 33, E, k, 64, 32, masked=0.1)
    check_experts(ex, 500, E, k, 64, 32, skew=2.0)


@pytest.mark.parametrize("d, f", [(8, 8), (1, 1), (33, 65), (100, 30), (167, 168), (1003, 200), (256, 1000)])
def test_experts_widths(ex, d, f):
    for n in (1, 20, 400):
        check_experts(ex, n, 6, 2, d, f, bias=True)
        check_experts(ex, n, 6, 2, d, f, "relu", gated=False, residual=False)


def test_experts_all_rows_on_one_and_none_at_all(ex):
    one = torch.full((700, 1), 3, device="cuda")
    check_experts(ex, 700, 5, 1, 128, 64, ids=one)
    none = torch.full((50, 2), -1, device="cuda")
    got = check_experts(ex, 50, 5, 2, 128, 64, ids=none, residual=False)
    assert float(got.abs().max()) == 0
    some = torch.full((90, 2), -1, device="cuda")
    some[::7, 0] = 4
    check_experts(ex, 90, 5, 2, 128, 64, ids=some)


def test_experts_strides_and_in_place(ex):
    for n in (5, 130):
        for pad in (8, 3):
            check_experts(ex, n, 8, 2, 128, 96, pad=pad)
    g = gen(2)
    x = normal(g, 40, 64).bfloat16()
    mk = lambda a, b: ex.pack(normal(g, 4, a, b).bfloat16())  # noqa: E731
    w, w2 = mk(32, 64), mk(64, 32)
    routing = ex.route(apart(40, 4, 1), 2)
    r = normal(g, 40, 64).bfloat16()
    want = ex.experts(x, routing, w, w2, act="relu", residual=r)
    got = ex.experts(x, routing, w, w2, act="relu", residual=r, out=r)
    assert got is r and torch.equal(got, want)


def test_experts_large(ex):
    check_experts(ex, 2050, 16, 4, 512, 384, skew=0.5, masked=0.05)


def test_a_row_alone_and_among_others(ex):
    """A row's result does not depend on the rows beside it beyond the order of its sums."""
    g = gen(12)
    x = normal(g, 300, 256).bfloat16()
    w, gw, w2 = ((normal(g, 8, a, b) / 16).bfloat16() for a, b in ((128, 256), (128, 256), (256, 128)))
    p1, p2 = ex.pack(w, gw), ex.pack(w2)
    logits = apart(300, 8, 4)
    whole = ex.experts(x, ex.route(logits, 2), p1, p2).double()
    for t in (0, 17, 299):
        one = ex.experts(x[t:t + 1], ex.route(logits[t:t + 1], 2), p1, p2).double()
        assert float((one - whole[t]).norm()) <= 4 * ROUND * float(whole[t].norm())


# ---- together ---------------------------------------------------------------------------

def block(ex, x, y, p):
    h, u = ex.norm(x, y, post="rms", pre="rms")
    logits = ex.linear(u, p["router"], out_dtype=F)
    routing = ex.route(logits, 2, score="sigmoid")
    return h, routing, ex.experts(u, routing, p["w1"], p["w2"], residual=h)


def parameters(ex, g, E=8, d=256, f=192):
    mk = lambda *s: (normal(g, *s) / math.sqrt(s[-1])).bfloat16()  # noqa: E731
    return {"router": ex.pack(mk(E, d)), "w1": ex.pack(mk(E, f, d), mk(E, f, d)), "w2": ex.pack(mk(E, d, f))}


@pytest.mark.parametrize("n", [1, 100, 1500])
def test_captured_and_replayed(ex, n):
    g = gen(21)
    p = parameters(ex, g)
    x, y = normal(g, n, 256).bfloat16(), normal(g, n, 256).bfloat16()
    block(ex, x, y, p)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        block(ex, x, y, p)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = block(ex, x, y, p)
    for i in range(4):
        x.copy_(normal(g, n, 256).bfloat16())
        y.copy_(normal(g, n, 256).bfloat16())
        graph.replay()
        torch.cuda.synchronize()
        want = block(ex, x, y, p)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2]), i
        assert all(torch.equal(a, b) for a, b in zip(got[1], want[1])), i


def test_on_another_stream(ex):
    g = gen(22)
    p = parameters(ex, g)
    x, y = normal(g, 700, 256).bfloat16(), normal(g, 700, 256).bfloat16()
    want = block(ex, x, y, p)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    h, u = ex.norm(x, y, post="rms", pre="rms", stream=s)
    routing = ex.route(ex.linear(u, p["router"], out_dtype=F, stream=s), 2, score="sigmoid", stream=s)
    out = ex.experts(u, routing, p["w1"], p["w2"], residual=h, stream=s)
    s.synchronize()
    assert torch.equal(h, want[0]) and torch.equal(out, want[2])


def test_the_same_bits_every_time(ex):
    g = gen(23)
    p = parameters(ex, g)
    x, y = normal(g, 900, 256).bfloat16(), normal(g, 900, 256).bfloat16()
    want = block(ex, x, y, p)
    for _ in range(3):
        got = block(ex, x, y, p)
        assert torch.equal(got[2], want[2]) and all(torch.equal(a, b) for a, b in zip(got[1], want[1]))


# ---- refusals of the Python entry points --------------------------------------------------

def test_refusals(ex):
    x = torch.zeros((4, 64), dtype=B, device="cuda")
    w = ex.pack(torch.zeros((8, 64), dtype=B, device="cuda"))
    w1, w2 = (ex.pack(torch.zeros(s, dtype=B, device="cuda")) for s in ((4, 32, 64), (4, 64, 32)))
    r = ex.route(torch.zeros((4, 4), device="cuda"), 2)
    bad = [
        lambda: ex.norm(x.cpu(), pre="rms"), lambda: ex.norm(x[0], pre="rms"), lambda: ex.norm(x.half(), pre="rms"),
        lambda: ex.norm(x.t(), pre="rms"), lambda: ex.norm(x, pre="batch"), lambda: ex.norm(x, x[:, :32], post="rms"),
        lambda: ex.norm(x, gate=x), lambda: ex.norm(x, x, gate=x.float()), lambda: ex.norm(x, x, row_gate=torch.zeros(5, device="cuda")),
        lambda: ex.norm(x, x, channel_scale=torch.zeros(64, device="cuda", dtype=B)), lambda: ex.norm(x, u=x.clone()),
        lambda: ex.norm(x, pre="rms", eps=-1.0), lambda: ex.norm(x[:1].expand(4, 64), pre="rms"),
        lambda: ex.route(x, 65), lambda: ex.route(x, 0), lambda: ex.route(x, 2, score="tanh"), lambda: ex.route(x, 2, groups=5),
        lambda: ex.route(x, 2, groups=4, top_groups=5), lambda: ex.route(x, 2, mask=torch.zeros(3, dtype=torch.uint8, device="cuda")),
        lambda: ex.route(x, 2, bias=torch.zeros(64, dtype=B, device="cuda")), lambda: ex.route(x.long(), 2),
        lambda: ex.pack(x.float()), lambda: ex.pack(x, x[:2]), lambda: ex.pack(x.cpu()),
        lambda: ex.linear(x[:, :32], w), lambda: ex.linear(x.float(), w), lambda: ex.linear(x, w1), lambda: ex.linear(x, w, act="tanh"),
        lambda: ex.linear(x, w, bias=torch.zeros(9, device="cuda")), lambda: ex.linear(x, w, gate_bias=torch.zeros(8, device="cuda")),
        lambda: ex.linear(x, w, residual=x), lambda: ex.linear(x, w, out=torch.zeros((4, 9), dtype=B, device="cuda")),
        lambda: ex.linear(x, w, out_dtype=torch.float16), lambda: ex.linear(x[:, 1:], ex.pack(x[:, 1:].clone()), workspace=None),
        lambda: ex.experts(x, r, w2, w1), lambda: ex.experts(x, r, w1, w1), lambda: ex.experts(x[:3], r, w1, w2),
        lambda: ex.experts(x, r._replace(offsets=None), w1, w2), lambda: ex.experts(x, r._replace(order=r.order.long()), w1, w2),
        lambda: ex.experts(x, r, w1, w2, bias2=torch.zeros(64, device="cuda")), lambda: ex.experts(x, r, w1, w2, workspace=None),
    ]
    from paper_2307_04963_amd._lib import DyclError
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, DyclError)):
            call()
            print("accepted:", i)

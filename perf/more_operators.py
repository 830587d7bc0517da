"""Timed cases of the decoding operators: what a network that emits a token at a
time needs around its layers.

Four operators: the rotation of heads by their positions, the entry of new
tokens' keys and values into a paged cache (with that rotation on the way), the
attention of one new token to such a cache, and the choice of the next tokens
over beams and vocabulary with the reordering of the cache behind it.
listed() holds the cases that are always timed, draw(rng) one more of the same
ranges.  run() calls the framework where `own` is true; otherwise it computes
the plain form in 32 bits (angles in 64).  exact() is the definition in 64 bits.
"""

import math

import torch

own = False

BF16, F32 = "bf16", "f32"
DTYPE = {BF16: torch.bfloat16, F32: torch.float32}


def rotate_case(name, n, heads, dim, dims, layout, x=BF16, far=8192, adjoint=False, factor=1.0, pad=0):
    return {"name": name, "op": "rotate", "n": n, "heads": heads, "dim": dim, "dims": dims, "layout": layout, "x": x, "far": far,
            "adjoint": adjoint, "factor": factor, "pad": pad}


def append_case(name, sequences, new, held, heads, kv, dim, dims, layout, page, x=BF16, idle=0.0):
    return {"name": name, "op": "append", "sequences": sequences, "new": new, "held": held, "heads": heads, "kv": kv, "dim": dim,
            "dims": dims, "layout": layout, "page": page, "x": x, "idle": idle}


def attend_case(name, n, low, high, heads, kv, dim, page, window=0, holes=0.0, empty=0.0):
    return {"name": name, "op": "attend", "n": n, "low": low, "high": high, "heads": heads, "kv": kv, "dim": dim, "page": page,
            "window": window, "holes": holes, "empty": empty}


def beam_case(name, sequences, beams, words, k, kv, dim, page, held, logits=BF16, ended=0.0, closed=0.0, first=False):
    return {"name": name, "op": "beam", "sequences": sequences, "beams": beams, "words": words, "k": k, "kv": kv, "dim": dim,
            "page": page, "held": held, "logits": logits, "ended": ended, "closed": closed, "first": first}


def listed():
    return [
        # the queries of one token: the latency of one small pass
        rotate_case("rotate_1x32x128", 1, 32, 128, 128, "half"),
        # the gradient of a long batch's rotated heads in 32 bits: part of the head, positions far out, rows of a wider tensor
        rotate_case("rotate_back_16383x20x96", 16383, 20, 96, 64, "interleaved", x=F32, far=1000000, adjoint=True, factor=8.0, pad=5),
        # one token each of 64 sequences
        append_case("append_64x1", 64, 1, 1000, 32, 8, 128, 128, "half", 16),
        # the prompts of five sequences at once
        append_case("append_5_prompts", 5, 1700, 0, 32, 8, 128, 128, "half", 64),
        # later parts of prompts behind what is cached already, in 32 bits, odd widths, part of the head, padding between them
        append_case("append_odd_13x97", 13, 97, 300, 6, 3, 72, 24, "interleaved", 8, x=F32, idle=0.1),
        # one sequence's next token: latency, the cache split over the whole card
        attend_case("attend_1x4095", 1, 4095, 4095, 32, 8, 128, 16),
        # many long sequences of unequal length: bound by reading the cache
        attend_case("attend_64x8192", 64, 4096, 8192, 32, 8, 128, 64),
        # heads of their own, a window, tokens that skipped this block (holes), sequences with nothing in the cache yet
        attend_case("attend_holes_37x3001", 37, 1, 3001, 16, 16, 64, 8, window=2048, holes=0.3, empty=0.1),
        # two very long sequences, wide heads that share two of the cache's
        attend_case("attend_2x131072", 2, 131000, 131072, 16, 2, 256, 128),
        # four beams of one sequence: latency
        beam_case("beam_1x4_of_32000", 1, 4, 32000, 4, 8, 128, 16, 777),
        # an odd vocabulary, twice as many choices as beams, some beams ended and some words closed
        beam_case("beam_13x5_of_50021", 13, 5, 50021, 10, 4, 64, 32, 300, ended=0.2, closed=0.1),
        # the largest choice, logits in 32 bits
        beam_case("beam_64x8_of_131072", 64, 8, 131072, 8, 8, 128, 64, 1000, logits=F32),
    ]


MOST_BYTES = 1.7e9      # of one drawn case: at most the largest listed one's


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rotate", "append", "attend", "attend", "beam", "beam"])
    coin = lambda p=0.5: rng.random() < p  # noqa: E731
    while True:
        dim = rng.choice([64, 64, 72, 80, 96, 128, 128, 128, 192, 256])
        dims = rng.choice([dim, dim, dim, dim // 2 // 2 * 2, dim // 4 // 2 * 2])
        layout = rng.choice(["half", "interleaved"])
        kv, page = rng.choice([1, 2, 3, 4, 8, 8, 16]), rng.choice([8, 16, 16, 32, 64, 128])
        heads = kv * rng.choice([1, 1, 2, 4, 4, 5, 8, 16])
        if op == "rotate":
            c = rotate_case("", _log_int(rng, 1, 32768), rng.choice([1, 3, 8, 16, 32]), dim, dims, layout, x=rng.choice([BF16, BF16, F32]),
                            far=_log_int(rng, 100, 1000000), adjoint=coin(0.3), factor=rng.choice([1.0, 4.0, 8.0]), pad=rng.choice([0, 0, 8, 3]))
        elif op == "append":
            c = append_case("", _log_int(rng, 1, 128), 1 if coin() else _log_int(rng, 2, 2000), rng.choice([0, _log_int(rng, 1, 1000)]), heads,
                            kv, dim, dims, layout, page, x=rng.choice([BF16, BF16, F32]), idle=rng.choice([0.0, 0.0, 0.2]))
            if c["sequences"] * (c["new"] + c["held"]) * kv * dim * 4 > 5e8:
                continue
        elif op == "attend":
            high = _log_int(rng, 1, 131072)
            c = attend_case("", _log_int(rng, 1, 256), rng.randrange(1, high + 1), high, heads, kv, dim, page,
                            window=rng.choice([0, 0, 0, _log_int(rng, 1, 4096)]), holes=rng.choice([0.0, 0.0, 0.2]),
                            empty=rng.choice([0.0, 0.0, 0.1]))
            if c["n"] * high * kv * dim * 4 > MOST_BYTES:
                continue
        else:
            beams = rng.choice([1, 2, 3, 4, 5, 8, 16])
            c = beam_case("", _log_int(rng, 1, 64), beams, _log_int(rng, 1000, 200000), rng.choice([beams, beams, 2 * beams]), rng.choice([1, 4, 8]),
                          rng.choice([64, 128]), page, rng.randrange(1, 1000), logits=rng.choice([BF16, F32]), ended=rng.choice([0.0, 0.2]),
                          closed=rng.choice([0.0, 0.0, 0.1]), first=coin(0.2))
            if c["sequences"] * beams * c["words"] > 64 * 8 * 131072:
                continue
        if work(c)["bytes"] <= MOST_BYTES:
            del c["name"]
            return c


# ---- what a program has in hand before the call -----------------------------

def _frequencies(dims, factor):
    """Radians per position of each pair, in 64 bits; for a context `factor` times the trained 8192 the slow ones are stretched, the fast ones
    kept and those between blended by their wavelength."""
    f = 10000.0 ** (-torch.arange(0, dims, 2, dtype=torch.float64) / dims)
    if factor != 1:
        keep = ((8192 * f / (2 * math.pi) - 1) / (4 - 1)).clamp(0, 1)
        f = f * (keep + (1 - keep) / factor)
    return f.cuda()


def _tables(g, counts, page, spare=0):
    """Page tables of sequences of `counts` tokens in a shuffled pool with `spare` pages more: (tables [n, most], pages, the spare ones)."""
    need = [-(-c // page) for c in counts]
    total = sum(need) + spare
    shuffled = torch.randperm(max(1, total), generator=g, device="cuda").int()
    tables = torch.full((len(counts), max(1, max(need))), -1, dtype=torch.int32)
    at = torch.tensor([0] + need).cumsum(0)
    place = torch.arange(tables.shape[1])[None, :] + at[:-1, None]
    there = torch.arange(tables.shape[1])[None, :] < torch.tensor(need)[:, None]
    tables = torch.where(there.cuda(), shuffled[torch.where(there, place, 0).cuda()], tables.cuda())
    return tables.contiguous(), max(1, total), shuffled[int(at[-1]):int(at[-1]) + spare].contiguous()


def _inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(1_000_003 * (seed % (1 << 31)) + 31)
    host = torch.Generator().manual_seed(seed % (1 << 31) + 7)
    # a case's lengths are its own, their order the seed's: outputs of all seeds have the same shapes
    sizes = torch.Generator().manual_seed(sum(v * (i + 3) for i, v in enumerate(c.values()) if isinstance(v, int)))
    normal = lambda *shape, dtype=torch.float32: torch.randn(shape, generator=g, device="cuda", dtype=dtype)  # noqa: E731
    uniform = lambda *shape: torch.rand(shape, generator=g, device="cuda")  # noqa: E731
    whole = lambda lo, hi, n: torch.randint(lo, hi + 1, (n,), generator=sizes)  # noqa: E731
    shuffled = lambda n: torch.randperm(n, generator=host)  # noqa: E731

    if c["op"] == "rotate":
        width = c["heads"] * c["dim"]
        return {"x": normal(c["n"], width + c["pad"]).to(DTYPE[c["x"]])[:, :width], "positions": torch.randint(0, c["far"] + 1, (c["n"],), generator=host).int().cuda(),
                "frequencies": _frequencies(c["dims"], c["factor"])}
    if c["op"] == "append":
        B, new, kv, dim = c["sequences"], c["new"], c["kv"], c["dim"]
        order = shuffled(B)
        held, fresh = whole(c["held"] // 2, c["held"], B)[order], whole(max(1, new // 2), new, B)[order]
        tables, pages, _ = _tables(g, (held + fresh).tolist(), c["page"])
        # rows in the sequences' order; a padding row holds no token (position -1)
        sequence = torch.arange(B).repeat_interleave(fresh)
        begin = torch.cat([torch.zeros(1, dtype=torch.int64), fresh.cumsum(0)[:-1]])
        positions = (torch.arange(len(sequence)) - begin[sequence] + held[sequence]).int().cuda()
        n = len(sequence)
        if c["idle"]:
            positions[uniform(n) < c["idle"]] = -1
        width = (c["heads"] + 2 * kv) * dim
        qkv = normal(n, width).to(DTYPE[c["x"]])        # one product's output: queries, keys, values side by side
        return {"q": qkv[:, :c["heads"] * dim], "k": qkv[:, c["heads"] * dim:(c["heads"] + kv) * dim], "v": qkv[:, (c["heads"] + kv) * dim:],
                "positions": positions, "sequence": sequence.int().cuda(), "tables": tables, "frequencies": _frequencies(c["dims"], 1.0),
                "keys": normal(pages, kv, c["page"], dim, dtype=torch.bfloat16), "values": normal(pages, kv, c["page"], dim, dtype=torch.bfloat16)}
    if c["op"] == "attend":
        n, kv, dim = c["n"], c["kv"], c["dim"]
        lengths = whole(c["low"], c["high"], n)
        if c["empty"]:
            lengths[torch.rand(n, generator=sizes) < c["empty"]] = 0
        lengths = lengths[shuffled(n)]
        tables, pages, _ = _tables(g, lengths.tolist(), c["page"])
        s = {"q": (1.5 * normal(n, c["heads"] * dim)).bfloat16(), "tables": tables, "lengths": lengths.int().cuda(), "mask": None,
             "keys": normal(pages, kv, c["page"], dim, dtype=torch.bfloat16), "values": normal(pages, kv, c["page"], dim, dtype=torch.bfloat16)}
        if c["holes"]:
            s["mask"] = uniform(n, tables.shape[1] * c["page"]) >= c["holes"]
        return s
    B, W, V, k = c["sequences"], c["beams"], c["words"], c["k"]
    rows = B * W
    ended = (uniform(rows) < c["ended"]).to(torch.uint8)
    scores = -12 * uniform(rows)
    if c["first"]:
        scores.view(B, W)[:, 1:] = -math.inf        # before the first token all beams are one
        ended.zero_()
    s = {"scores": scores, "ended": ended}
    logits = 2.5 * normal(rows, V)
    if c["closed"]:
        logits = torch.where(uniform(rows, V) < c["closed"], torch.full_like(logits, -math.inf), logits)
    # a choice that hangs on the rounding of a score is no choice that 32 bits define: such sequences are made anew
    for _ in range(12):
        s["logits"] = logits.to(DTYPE[c["logits"]])
        bad = _close_calls(c, s)
        if not bad.any():
            break
        logits.view(B, W, V)[bad] = 2.5 * normal(int(bad.sum()), W, V)
    held = whole(max(1, c["held"] // 2), c["held"], rows)[shuffled(rows)]
    tables, pages, spare = _tables(g, held.tolist(), c["page"], B * k)
    s.update(tables=tables, lengths=held.int().cuda(), fresh=spare, keys=normal(pages, c["kv"], c["page"], c["dim"], dtype=torch.bfloat16),
             values=normal(pages, c["kv"], c["page"], c["dim"], dtype=torch.bfloat16))
    return s


def _close_calls(c, s):
    """Sequences among whose best candidates two unequal ones, in 64 bits, lie within a few roundings of 32 bits."""
    B, W, V = c["sequences"], c["beams"], c["words"]
    top = min(V, c["k"] + 1)
    z = s["logits"].double()
    best = z.topk(top, 1).values + (s["scores"].double() - torch.logsumexp(z, 1))[:, None]
    kept = torch.full_like(best, -math.inf)
    kept[:, 0] = s["scores"].double()
    ranked = torch.where(s["ended"][:, None] != 0, kept, best).view(B, -1).sort(dim=1, descending=True).values[:, :c["k"] + 1]
    gap = ranked[:, :-1] - ranked[:, 1:]
    return ((gap > 0) & (gap < 4e-5)).any(1)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = dict(case)
    return s


# ---- one pass -----------------------------------------------------------------

END = 2


def run(s):
    return (_OWN if own else _PLAIN)[s["case"]["op"]](s)


def _own_rotate(s):
    from paper_2307_04963_amd import decoding as de
    c = s["case"]
    return de.rotate(s["x"], s["positions"], s["frequencies"], dim=c["dim"], layout=c["layout"], adjoint=c["adjoint"])


def _own_append(s):
    from paper_2307_04963_amd import decoding as de
    q = de.append(de.Cache(s["keys"], s["values"]), s["k"], s["v"], s["positions"], s["tables"], sequence=s["sequence"],
                  frequencies=s["frequencies"], layout=s["case"]["layout"], q=s["q"])
    return {"keys": s["keys"], "values": s["values"], "q": q}


def _own_attend(s):
    from paper_2307_04963_amd import decoding as de
    return de.attend(s["q"], de.Cache(s["keys"], s["values"]), s["tables"], s["lengths"], window=s["case"]["window"], mask=s["mask"])


def _own_beam(s):
    from paper_2307_04963_amd import decoding as de
    c = s["case"]
    b = de.beam(s["logits"], s["scores"], c["beams"], k=c["k"], ended=s["ended"], end=END)
    tables, lengths = de.fork(de.Cache(s["keys"], s["values"]), s["tables"], s["lengths"], b.parents, s["fresh"])
    return {"parents": b.parents, "tokens": b.tokens, "scores": b.scores, "ended": b.ended, "tables": tables, "lengths": lengths,
            "keys": s["keys"], "values": s["values"]}


_OWN = {"rotate": _own_rotate, "append": _own_append, "attend": _own_attend, "beam": _own_beam}


def _turn(x, positions, frequencies, layout, sign=1.0):
    """x [n, heads, dim] in 32 bits, its first pairs turned by position * frequency (an angle of 64 bits)."""
    angle = positions.double()[:, None] * frequencies
    cos, sin = angle.cos().float()[:, None], sign * angle.sin().float()[:, None]
    half = frequencies.numel()
    out = x.clone()
    a, b = (x[..., :half], x[..., half:2 * half]) if layout == "half" else (x[..., 0:2 * half:2], x[..., 1:2 * half:2])
    first, second = (slice(0, half), slice(half, 2 * half)) if layout == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    out[..., first] = a * cos - b * sin
    out[..., second] = b * cos + a * sin
    return out


def _plain_rotate(s):
    c = s["case"]
    x = s["x"].float().reshape(c["n"], c["heads"], c["dim"])
    y = _turn(x, s["positions"], s["frequencies"], c["layout"], -1.0 if c["adjoint"] else 1.0)
    return y.reshape(c["n"], -1).to(s["x"].dtype)


def _plain_append(s):
    c = s["case"]
    n = len(s["positions"])
    heads = lambda t: t.float().reshape(n, -1, c["dim"])  # noqa: E731
    q = _turn(heads(s["q"]), s["positions"], s["frequencies"], c["layout"])
    k = _turn(heads(s["k"]), s["positions"], s["frequencies"], c["layout"])
    live = s["positions"] >= 0
    at = s["positions"].long()[live]
    page = s["tables"][s["sequence"].long()[live], at // c["page"]].long()
    s["keys"][page, :, at % c["page"]] = k[live].bfloat16()
    s["values"][page, :, at % c["page"]] = heads(s["v"])[live].bfloat16()
    q = torch.where(live[:, None, None], q, torch.zeros_like(q)).reshape(n, -1)
    return {"keys": s["keys"], "values": s["values"], "q": q.to(s["q"].dtype)}


def _plain_attend(s):
    c = s["case"]
    n, kv, dim = c["n"], c["kv"], c["dim"]
    most = s["tables"].shape[1] * c["page"]
    at = torch.arange(most, device=s["q"].device)
    length = s["lengths"].long()[:, None]
    here = at < length
    if c["window"]:
        here = here & (at >= length - c["window"])
    if s["mask"] is not None:
        here = here & s["mask"]
    pages = s["tables"].long().clamp(min=0)
    laid = lambda t: t[pages].float().permute(0, 2, 1, 3, 4).reshape(n * kv, most, dim)  # noqa: E731
    q = s["q"].float().view(n * kv, c["heads"] // kv, dim)
    z = torch.bmm(q, laid(s["keys"]).transpose(1, 2).contiguous()).view(n, c["heads"], most) / math.sqrt(dim)
    here = here[:, None]
    z = torch.where(here, z, torch.full_like(z, -math.inf))
    top = z.amax(2, keepdim=True)
    e = torch.where(here, torch.exp(z - top), torch.zeros_like(z))
    total = e.sum(2, keepdim=True)
    p = torch.where(total > 0, e / total, torch.zeros_like(e))
    return torch.bmm(p.view(n * kv, -1, most), laid(s["values"])).view(n, -1).bfloat16()


def _plain_beam(s):
    c = s["case"]
    B, W, V, k = c["sequences"], c["beams"], c["words"], c["k"]
    z = s["logits"].float()
    top = z.amax(1, keepdim=True)
    total = torch.exp(z - top).sum(1, keepdim=True)
    scores = s["scores"][:, None]
    v = z + (scores - top - torch.log(total))
    ended = s["ended"][:, None] != 0
    word = torch.arange(V, device=z.device)
    v = torch.where(ended, torch.where(word == END, scores, torch.full_like(v, -math.inf)), v)
    ranked, index = v.view(B, W * V).sort(dim=1, descending=True, stable=True)
    ranked, index = ranked[:, :k], index[:, :k]
    none = ranked == -math.inf
    gone = torch.full_like(index, -1)
    parents = torch.where(none, gone, index // V + W * torch.arange(B, device=z.device)[:, None])
    tokens = torch.where(none, gone, index % V)
    # the cache behind them: a parent's table and length, its last page's tokens in a page of the row's own
    of = parents.view(-1)
    live, of = of >= 0, of.clamp(min=0)
    lengths = torch.where(live, s["lengths"].long()[of], torch.zeros_like(of))
    tables = torch.where(live[:, None], s["tables"][of], torch.full_like(s["tables"][of], -1))
    full = lengths // c["page"]
    place = torch.arange(tables.shape[1], device=z.device)
    tables = torch.where(live[:, None] & (place == full[:, None]), s["fresh"][:, None], tables)
    part = live & (lengths % c["page"] > 0)
    source, target = s["tables"][of[part], full[part]].long(), s["fresh"].long()[part]
    slot = torch.arange(c["page"], device=z.device)[None, None, :, None] < (lengths % c["page"])[part][:, None, None, None]
    s["keys"][target] = torch.where(slot, s["keys"][source], s["keys"][target])
    s["values"][target] = torch.where(slot, s["values"][source], s["values"][target])
    over = live & (ended[of, 0] | (tokens.view(-1) == END))
    return {"parents": parents.int(), "tokens": tokens.int(), "scores": ranked, "ended": over.view(B, k).to(torch.uint8),
            "tables": tables, "lengths": lengths.int(), "keys": s["keys"], "values": s["values"]}


_PLAIN = {"rotate": _plain_rotate, "append": _plain_append, "attend": _plain_attend, "beam": _plain_beam}


# ---- what a pass cannot do without ----------------------------------------------

def work(c):
    size = {BF16: 2, F32: 4}
    if c["op"] == "rotate":
        values = c["n"] * c["heads"] * c["dim"]
        return {"bytes": 2 * values * size[c["x"]] + 4 * c["n"], "flops": 3 * values}
    if c["op"] == "append":
        n = c["sequences"] * (max(1, c["new"] // 2) + c["new"]) / 2
        q, kv = n * c["heads"] * c["dim"], n * (1 - c["idle"]) * 2 * c["kv"] * c["dim"]
        return {"bytes": int(2 * q * size[c["x"]] + kv * (size[c["x"]] + 2) + 12 * n), "flops": int(3 * (q + kv))}
    if c["op"] == "attend":
        seen = (c["low"] + c["high"]) / 2
        if c["window"]:
            lo, hi, w = c["low"], c["high"], c["window"]
            seen = w if w <= lo else seen if w >= hi else ((w * w - lo * lo) / 2 + w * (hi - w)) / (hi - lo)
        seen *= c["n"] * (1 - c["empty"])
        return {"bytes": int(4 * seen * (1 - c["holes"]) * c["kv"] * c["dim"] + (seen if c["holes"] else 0) + 4 * c["n"] * c["heads"] * c["dim"]),
                "flops": int(4 * seen * (1 - c["holes"]) * c["heads"] * c["dim"])}
    rows, out = c["sequences"] * c["beams"], c["sequences"] * c["k"]
    values = rows * (1 - c["ended"]) * c["words"]
    return {"bytes": int(values * size[c["logits"]] + out * (c["kv"] * c["page"] // 2 * c["dim"] * 8 + 8 * -(-c["held"] // c["page"]))),
            "flops": int(4 * values)}


# ---- the definition in 64 bits ------------------------------------------------------

def exact(case, seed):
    return _EXACT[case["op"]](case, _inputs(case, seed))


def _exact_turn(x, positions, frequencies, layout, back=False):
    """Each pair as a complex number, times e^(i angle) (its conjugate for the gradient)."""
    half = frequencies.numel()
    angle = positions.double()[:, None] * frequencies[None, :]
    spin = torch.polar(torch.ones_like(angle), -angle if back else angle)[:, None]
    x = x.double()
    turned, rest = x[..., :2 * half], x[..., 2 * half:]
    if layout == "half":
        z = torch.complex(turned[..., :half], turned[..., half:]) * spin
        turned = torch.cat([z.real, z.imag], -1)
    else:
        z = torch.view_as_complex(turned.reshape(*turned.shape[:-1], half, 2).contiguous()) * spin
        turned = torch.view_as_real(z).flatten(-2)
    return torch.cat([turned, rest], -1)


def _exact_rotate(c, s):
    x = s["x"].reshape(c["n"], c["heads"], c["dim"])
    return _exact_turn(x, s["positions"], s["frequencies"], c["layout"], c["adjoint"]).reshape(c["n"], -1)


def _exact_append(c, s):
    n, dim = len(s["positions"]), c["dim"]
    q = _exact_turn(s["q"].reshape(n, -1, dim), s["positions"], s["frequencies"], c["layout"])
    k = _exact_turn(s["k"].reshape(n, -1, dim), s["positions"], s["frequencies"], c["layout"])
    live = torch.nonzero(s["positions"] >= 0)[:, 0]
    at = s["positions"].long()[live]
    page = s["tables"].long()[s["sequence"].long()[live], torch.div(at, c["page"], rounding_mode="floor")]
    row = page * c["page"] + at % c["page"]

    def entered(cache, new):
        flat = cache.double().transpose(1, 2).reshape(-1, c["kv"], dim)
        flat[row] = new.double()[live]
        return flat.view(-1, c["page"], c["kv"], dim).transpose(1, 2)

    q[s["positions"] < 0] = 0
    return {"keys": entered(s["keys"], k), "values": entered(s["values"], s["v"].reshape(n, -1, dim)), "q": q.reshape(n, -1)}


def _exact_attend(c, s):
    """Sequence by sequence, over the keys that it sees and no others."""
    group, dim, page = c["heads"] // c["kv"], c["dim"], c["page"]
    out = torch.zeros((c["n"], c["heads"], dim), dtype=torch.float64, device="cuda")
    for r, length in enumerate(s["lengths"].tolist()):
        at = torch.arange(max(0, length - c["window"]) if c["window"] else 0, length, device="cuda")
        if s["mask"] is not None:
            at = at[s["mask"][r, at]]
        if len(at):
            where = s["tables"][r].long()[torch.div(at, page, rounding_mode="floor")]
            k, v = (s[t][where, :, at % page].double().transpose(0, 1).contiguous() for t in ("keys", "values"))
            q = s["q"][r].double().view(c["kv"], group, dim)
            z = torch.matmul(q, k.transpose(1, 2).contiguous()) * dim ** -0.5
            out[r] = torch.matmul(torch.softmax(z, 2), v).reshape(c["heads"], dim)
    return out.view(c["n"], -1)


def _exact_beam(c, s):
    """Round by round: the best candidate that is left, the lowest beam and word among equals."""
    B, W, V, k, page = c["sequences"], c["beams"], c["words"], c["k"], c["page"]
    v = torch.log_softmax(s["logits"].double(), 1) + s["scores"].double()[:, None]
    for r in torch.nonzero(s["ended"])[:, 0].tolist():
        v[r] = -math.inf
        v[r, END] = s["scores"][r].double()
    v = torch.nan_to_num(v.view(B, W * V), neginf=-1e30)
    place = torch.arange(W * V, device=v.device)
    parents, tokens, scores = [], [], []
    for _ in range(k):
        best = v.amax(1, keepdim=True)
        i = torch.where(v == best, place, W * V).amin(1, keepdim=True)
        there = best > -1e29
        parents.append(torch.where(there, torch.div(i, V, rounding_mode="floor") + torch.arange(0, B * W, W, device=v.device)[:, None], -1))
        tokens.append(torch.where(there, i % V, -1))
        scores.append(torch.where(there, best, -math.inf))
        v.scatter_(1, i, -1e30)
    parents, tokens, scores = torch.cat(parents, 1), torch.cat(tokens, 1), torch.cat(scores, 1)
    tables = torch.full((B * k, s["tables"].shape[1]), -1, dtype=torch.int32, device=v.device)
    lengths = torch.zeros(B * k, dtype=torch.int32, device=v.device)
    over = torch.zeros(B * k, dtype=torch.uint8, device=v.device)
    keys, values = s["keys"].double(), s["values"].double()
    held, before, fresh, ended = s["lengths"].tolist(), s["tables"].tolist(), s["fresh"].tolist(), s["ended"].tolist()
    for i, (r, t) in enumerate(zip(parents.view(-1).tolist(), tokens.view(-1).tolist())):
        if r >= 0:
            full, rest = divmod(held[r], page)
            tables[i] = s["tables"][r]
            lengths[i] = held[r]
            over[i] = int(ended[r] != 0 or t == END)
            if full < tables.shape[1]:
                tables[i, full] = fresh[i]
            if rest:
                keys[fresh[i], :, :rest] = s["keys"][before[r][full], :, :rest].double()
                values[fresh[i], :, :rest] = s["values"][before[r][full], :, :rest].double()
    return {"parents": parents, "tokens": tokens, "scores": scores, "ended": over.view(B, k), "tables": tables, "lengths": lengths,
            "keys": keys, "values": values}


_EXACT = {"rotate": _exact_rotate, "append": _exact_append, "attend": _exact_attend, "beam": _exact_beam}

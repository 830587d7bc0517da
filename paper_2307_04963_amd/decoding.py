"""The decoding operators of include/dycl_decode.h on torch tensors: heads turned
by their positions, a paged cache of keys and values, the attention of single
tokens to it, the choice of the next tokens over beams, and the cache's
reordering behind it.  This file gives the arguments names and defaults;
_tokens.so (csrc/binding) checks the tensors and calls libdycl.so, where every
kernel is.

A row is one token; its heads lie side by side in a 2-D tensor whose last
dimension is contiguous (rows may be strided: a slice of a wider product is
taken as it is).  Work is queued on ``stream`` (default: the current one); what
a call allocates belongs to that stream.  Wrong tensors raise ValueError, other
refusals DyclError.  Nothing here records gradients (tensors that require
grad are refused where gradients are recorded, and those that carry a
forward-mode tangent); rotate's ``adjoint`` is its gradient, and rotate of a
tangent its tangent.
"""

from __future__ import annotations

import math
from typing import NamedTuple

import torch

from .experts import _call, _of, _room, _tokens

LAYOUTS = {"half": 0, "interleaved": 1}


class Cache(NamedTuple):
    """One layer's keys and values, [pages, heads, page, dim] bf16."""
    keys: torch.Tensor
    values: torch.Tensor


def cache(pages: int, heads: int, page: int, dim: int, device="cuda") -> Cache:
    """An empty cache (its values are whatever the memory held)."""
    return Cache(*(torch.empty((pages, heads, page, dim), dtype=torch.bfloat16, device=device) for _ in range(2)))


def frequencies(dims: int, base: float = 10000.0, *, scaling: str = "none", factor: float = 1.0, trained: int | None = None,
                slow: float = 1.0, fast: float = 4.0, device="cuda") -> torch.Tensor:
    """Radians per position of the dims / 2 pairs, float64: f_i = base^(-2 i / dims), scaled for contexts `factor`
    times as long as the `trained` one:

    "linear"   f / factor: positions closer together
    "base"     base * factor^(dims / (dims - 2)): the slowest pair divided by factor, the fastest kept
    "turns"    by the turns t = trained * f / (2 pi) that a pair makes in the trained context: f from `fast` turns on,
               f / factor up to `slow`, between them the blend of the two, linear in t
    "pairs"    the same with the blend linear in i, from the pair that makes `fast` turns (rounded down) to the one that makes
               `slow` (rounded up), wherever these lie, also outside the dims / 2 pairs
    """
    if dims < 2 or dims % 2:
        raise ValueError("dims must be even and at least 2")
    if not (base > 0 and math.isfinite(base) and factor > 0 and math.isfinite(factor)):
        raise ValueError("base and factor must be positive and finite")
    i = torch.arange(dims // 2, dtype=torch.float64)
    if scaling == "base":
        if dims == 2:
            raise ValueError("a single pair has no slower one: dims must be at least 4")
        base = base * factor ** (dims / (dims - 2))
    f = base ** (-2 * i / dims)
    if scaling == "linear":
        f = f / factor
    elif scaling in ("turns", "pairs"):
        if trained is None or trained < 1 or not 0 < slow < fast:
            raise ValueError(f'scaling "{scaling}" needs the trained context and 0 < slow < fast')
        if scaling == "turns":
            keep = (trained * f / (2 * math.pi) - slow) / (fast - slow)
        else:
            if base <= 1:
                raise ValueError('scaling "pairs" needs a base above 1')
            # the pair that makes t turns: trained * base^(-2 i / dims) = 2 pi t; it may lie before the first pair or past the last
            of = lambda t: dims * math.log(trained / (2 * math.pi * t)) / (2 * math.log(base))  # noqa: E731
            first, last = math.floor(of(fast)), math.ceil(of(slow))
            keep = 1 - (i - first) / max(last - first, 1e-3)
        keep = keep.clamp(0, 1)
        f = f * (keep + (1 - keep) / factor)
    elif scaling not in ("none", "base"):
        raise ValueError("scaling must be one of ['none', 'linear', 'base', 'turns', 'pairs']")
    return f.to(device)


def rotate(x: torch.Tensor, positions: torch.Tensor, frequencies: torch.Tensor, *, dim: int, layout: str = "half", magnitude: float = 1.0,
           adjoint: bool = False, out=None, stream=None) -> torch.Tensor:
    """dycl_op_rotate: the first 2 * len(frequencies) values of each head of `dim` in x [n, heads * dim] (bf16 or float32),
    turned by positions [n] int32 * frequencies (float64); layout "half" pairs value i with i + len(frequencies),
    "interleaved" 2 i with 2 i + 1.  adjoint: turned back, times magnitude: x's gradient for y's.  out may be x."""
    return _call(stream, _tokens.rotate, x, positions, frequencies, dim, _of(LAYOUTS, layout, "layout"), magnitude, adjoint, out)


def append(cache: Cache, k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor, tables: torch.Tensor, *, sequence=None,
           frequencies=None, layout: str = "half", magnitude: float = 1.0, q=None, q_out=None, stream=None):
    """dycl_op_append: row r of k and v [n, heads * dim] (bf16 or float32) becomes the token at place positions[r] of
    sequence[r] (default r), k turned as by rotate if frequencies are given; returns the turned q (q_out may be q; None
    without q).  tables [sequences, max_pages] int32 names the sequences' pages.  Rows of negative position are
    padding: nothing enters, their q is 0."""
    return _call(stream, _tokens.append, *cache, k, v, positions, tables, sequence, frequencies, _of(LAYOUTS, layout, "layout"), magnitude,
                 q, q_out)


def attend(q: torch.Tensor, cache: Cache, tables: torch.Tensor, lengths: torch.Tensor, *, sequence=None, scale: float | None = None,
           window: int = 0, mask=None, max_length: int | None = None, out=None, workspace="auto", stream=None) -> torch.Tensor:
    """dycl_op_attend: each row of q [n, q_heads * dim] bf16 attends to the first lengths[r] (int32) keys of sequence[r]
    (default r), the last `window` of them if that is not 0, those whose mask [n, max_length] (bool or uint8) is not 0.
    scale defaults to 1 / sqrt(dim), max_length (no length may be above it) to the tables' capacity; the work is divided
    for it, so where tables are much longer than the rows give a tight one (one row of 4095 keys: 10 us, 49 in a table for 131072).  A row without a key is 0.  Returns [n, q_heads * dim] bf16."""
    if max_length is not None and max_length < 0:
        raise ValueError("max_length must not be negative")
    return _call(stream, _tokens.attend, q, *cache, tables, lengths, sequence, scale, window, mask, -1 if max_length is None else max_length,
                 out, *_room(workspace))


class Beams(NamedTuple):
    """What dycl_op_beam writes, [sequences, k]: the rows of logits that go on (-1: fewer than k candidates), their next
    tokens, their scores, and whether they have ended (uint8)."""
    parents: torch.Tensor
    tokens: torch.Tensor
    scores: torch.Tensor
    ended: torch.Tensor


def beam(logits: torch.Tensor, scores: torch.Tensor, beams: int, *, k: int | None = None, ended=None, end: int = -1, workspace="auto",
         stream=None) -> Beams:
    """dycl_op_beam: the k (default: beams) largest of scores + log softmax(logits) over the beams and words of each
    sequence; logits [sequences * beams, words] (bf16 or float32), scores float32, ended (uint8 or bool) the beams that
    hold the token `end` already and go on as they are."""
    return Beams(*_call(stream, _tokens.beam, logits, scores, beams, beams if k is None else k, ended, end, *_room(workspace)))


def fork(cache, tables: torch.Tensor, lengths: torch.Tensor, parents: torch.Tensor, fresh: torch.Tensor, *, page: int | None = None,
         out_tables=None, out_lengths=None, stream=None):
    """dycl_op_fork: (tables, lengths) of rows that go on from rows `parents` (any shape, int32), with fresh[i] as the
    page of row i's next token; what the parent has in that page already is copied there in `cache`: one Cache, a
    list of the layers' (which share the tables), or None with `page` given.  Fresh pages are distinct pages that no
    sequence that goes on reads."""
    layers = [cache] if isinstance(cache, Cache) else list(cache or [])
    if not layers and page is None:
        raise ValueError("without a cache, page (tokens of a page) must be given")
    return _call(stream, _tokens.fork, tables, lengths, parents, fresh, page, out_tables, out_lengths, *(t for c in layers for t in c))

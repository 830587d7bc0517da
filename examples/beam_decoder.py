"""A decoder that emits tokens over beams: the decoding operators with the token
operators, as a serving program runs them.

Each block attends to the tokens so far (a paged cache of its own), to an
encoder's states, and passes through a gated layer.  Every step enters one token
per beam, chooses the next ones over all beams and words, and reorders the
caches: full pages are shared by the beams that go on from the same one, the
begun page is copied to a page of the new beam's own.

    python -m examples.beam_decoder --sequences 8 --beams 4
"""

from __future__ import annotations

import argparse
import math
from typing import NamedTuple

import torch

from paper_2307_04963_amd import decoding as de, experts as ex

PAGE = 16


class Block(NamedTuple):
    """One block's weights (products packed once): norms [d] float32; queries, keys and values of the tokens so far in one
    layer; queries to the encoder's states, and those states' keys and values; the gated layer's two products."""
    norms: list
    qkv: ex.Packed
    out: ex.Packed
    cross_q: ex.Packed
    cross_kv: ex.Packed
    cross_out: ex.Packed
    up: ex.Packed
    down: ex.Packed


class Decoder:
    def __init__(self, embedding, blocks, last_norm, head: ex.Packed, heads: int, kv_heads: int, dim: int, end: int):
        self.embedding, self.blocks, self.last_norm, self.head = embedding, blocks, last_norm, head
        self.heads, self.kv_heads, self.dim, self.end = heads, kv_heads, dim, end
        self.frequencies = de.frequencies(dim, device=embedding.device)

    def encode(self, states: torch.Tensor, lengths: list):
        """The encoder's states [sum(lengths), d] bf16 as every block's keys and values: (caches, tables, lengths)."""
        dev, need = states.device, [-(-n // PAGE) for n in lengths]
        tables = torch.full((len(lengths), max(1, max(need))), -1, dtype=torch.int32)
        for i, k in enumerate(need):
            tables[i, :k] = torch.arange(sum(need[:i]), sum(need[:i]) + k)
        tables = tables.to(dev)
        row = torch.tensor([s for s, n in enumerate(lengths) for _ in range(n)], dtype=torch.int32, device=dev)
        place = torch.tensor([p for n in lengths for p in range(n)], dtype=torch.int32, device=dev)
        caches = []
        for b in self.blocks:
            kv = ex.linear(states, b.cross_kv)
            caches.append(de.cache(max(1, sum(need)), self.kv_heads, PAGE, self.dim, dev))
            de.append(caches[-1], *kv.split(self.kv_heads * self.dim, 1), place, tables, sequence=row)
        return caches, tables, torch.tensor(lengths, dtype=torch.int32, device=dev)

    def step(self, tokens, caches, tables, lengths, encoder, encoder_lengths, sequence, most: int):
        """Logits [rows, words] float32 of one more token per row, which enters the caches."""
        h, y = self.embedding[tokens], None
        wide, narrow = self.heads * self.dim, self.kv_heads * self.dim
        now = lengths + 1
        for b, cache, states in zip(self.blocks, caches, encoder[0]):
            h, u = ex.norm(h, y, pre="rms", pre_weight=b.norms[0])
            q, k, v = ex.linear(u, b.qkv).split([wide, narrow, narrow], 1)
            q = de.append(cache, k, v, lengths, tables, frequencies=self.frequencies, q=q)
            y = ex.linear(de.attend(q, cache, tables, now, max_length=most), b.out)
            h, u = ex.norm(h, y, pre="rms", pre_weight=b.norms[1])
            y = ex.linear(de.attend(ex.linear(u, b.cross_q), states, encoder[1], encoder_lengths, sequence=sequence), b.cross_out)
            h, u = ex.norm(h, y, pre="rms", pre_weight=b.norms[2])
            y = ex.linear(ex.linear(u, b.up, act="silu"), b.down)
        _, u = ex.norm(h, y, pre="rms", pre_weight=self.last_norm)
        return ex.linear(u, self.head, out_dtype=torch.float32)

    def __call__(self, first: torch.Tensor, encoder, beams: int, steps: int):
        """From the first tokens [sequences] (int64): (tokens [sequences, beams, steps], their scores [sequences, beams])."""
        dev, n = first.device, len(first)
        rows, most = n * beams, -(-steps // PAGE)
        pages = torch.arange((most + 2) * rows, dtype=torch.int32, device=dev).view(most + 2, rows)
        caches = [de.cache((most + 2) * rows, self.kv_heads, PAGE, self.dim, dev) for _ in self.blocks]
        tables = torch.full((rows, most), -1, dtype=torch.int32, device=dev)
        tables[:, 0] = pages[0]
        begun, spare, unused = 0, 1, 2                  # sets of a page per row: the begun ones, the next step's, not used yet
        lengths = torch.zeros(rows, dtype=torch.int32, device=dev)
        sequence = torch.arange(n, dtype=torch.int32, device=dev).repeat_interleave(beams)
        encoder_lengths = encoder[2][sequence.long()].contiguous()
        scores = torch.full((n, beams), -math.inf, device=dev)
        scores[:, 0] = 0                                # before the first choice all beams are one
        scores, ended = scores.view(-1), torch.zeros(rows, dtype=torch.uint8, device=dev)
        tokens, said = first.repeat_interleave(beams), torch.empty((rows, 0), dtype=torch.int64, device=dev)
        for i in range(steps):
            logits = self.step(tokens, caches, tables, lengths, encoder, encoder_lengths, sequence, i + 1)
            b = de.beam(logits, scores, beams, ended=ended, end=self.end)
            parents, tokens = b.parents.view(-1), b.tokens.view(-1).long().clamp(min=0)
            scores, ended = b.scores.view(-1), b.ended.view(-1)
            said = torch.cat([said[parents.long().clamp(min=0)], tokens[:, None]], 1)
            full = (i + 1) % PAGE == 0                  # the begun pages are complete: the rows that have them keep them
            tables, lengths = de.fork(caches, tables, lengths + 1, parents, pages[unused if full else spare])
            begun, spare, unused = (unused, spare, unused + 1) if full else (spare, begun, unused)
        return said.view(n, beams, steps), scores.view(n, beams)


def build(blocks=2, d=512, f=1024, heads=8, kv_heads=2, dim=64, words=1000, end=1, seed=0, device="cuda") -> Decoder:
    """A decoder of random weights."""
    g = torch.Generator(device=device).manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=g, device=device)  # noqa: E731
    layer = lambda n, k: (normal(n, k) / math.sqrt(k)).bfloat16()  # noqa: E731
    wide, narrow = heads * dim, kv_heads * dim
    made = [Block([1 + 0.1 * normal(d) for _ in range(3)], ex.pack(layer(wide + 2 * narrow, d)), ex.pack(layer(d, wide)), ex.pack(layer(wide, d)),
                  ex.pack(layer(2 * narrow, d)), ex.pack(layer(d, wide)), ex.pack(layer(f, d), layer(f, d)), ex.pack(layer(d, f)))
            for _ in range(blocks)]
    return Decoder(normal(words, d).bfloat16(), made, 1 + 0.1 * normal(d), ex.pack((3 * layer(words, d).float()).bfloat16()), heads, kv_heads, dim, end)


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, default in (("sequences", 8), ("beams", 4), ("steps", 64), ("blocks", 4), ("d", 1024), ("f", 4096), ("heads", 16), ("words", 32000)):
        p.add_argument(f"--{name}", type=int, default=default)
    a = p.parse_args()
    model = build(a.blocks, a.d, a.f, a.heads, a.heads // 4, 64, a.words)
    lengths = [20 + 7 * i for i in range(a.sequences)]
    states = torch.randn((sum(lengths), a.d), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).bfloat16()
    first = torch.zeros(a.sequences, dtype=torch.int64, device="cuda")
    encoder = model.encode(states, lengths)
    model(first, encoder, a.beams, 4)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    said, scores = model(first, encoder, a.beams, a.steps)
    end.record()
    torch.cuda.synchronize()
    ms = begin.elapsed_time(end)
    print(f"{a.sequences} sequences, {a.beams} beams, {a.steps} steps of {a.blocks} blocks: {ms:.1f} ms, {1000 * ms / a.steps:.0f} us a step;",
          "best scores:", [round(v, 2) for v in scores[:, 0].tolist()])


if __name__ == "__main__":
    main()

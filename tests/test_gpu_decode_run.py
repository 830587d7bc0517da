"""The decoding operators together, as a program that emits tokens over beams uses them: every step enters its tokens into the
caches of two layers, attends to them and to an encoder's states, chooses the next tokens and reorders the caches.

A token's keys, values and queries are rows of tables, so what a beam's cache has to hold follows from its tokens
alone: after every step it holds exactly that.
"""

import math

import pytest
import torch

from tests._decode import attended64, chosen64, dense, gen, turned64, within

pytestmark = pytest.mark.gpu

B = torch.bfloat16
SEQUENCES, BEAMS, WORDS, PAGE, STEPS, END = 3, 4, 61, 8, 45, 7


def test_steps_over_beams():
    from paper_2307_04963_amd import decoding as de
    g = gen(1)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    rows, most = SEQUENCES * BEAMS, -(-STEPS // PAGE)
    shapes = [(4, 2, 64), (6, 1, 40)]                       # query heads, heads, dim of the two layers
    words = [tuple(normal(WORDS, h * d).to(B) for h in (hq, hk, hk)) for hq, hk, d in shapes]
    frequencies = [de.frequencies(64), de.frequencies(24, scaling="linear", factor=2.0)]
    layouts = ["half", "interleaved"]
    # pages of every table's entry, and two sets that the begun pages alternate between
    caches = [de.cache((most + 2) * rows, hk, PAGE, d) for _, hk, d in shapes]
    pages = torch.randperm((most + 2) * rows, generator=g, device="cuda").int().view(most + 2, rows)
    # an encoder's states of the sequences, of lengths of their own
    encoded = [11, 0, 30]
    states = [tuple(normal(sum(encoded), hk * d).to(B) for _ in range(2)) for _, hk, d in shapes]
    of = torch.tensor([s for s, n in enumerate(encoded) for _ in range(n)], dtype=torch.int32, device="cuda")
    place = torch.tensor([p for n in encoded for p in range(n)], dtype=torch.int32, device="cuda")
    encoder = [de.cache(12, hk, PAGE, d) for _, hk, d in shapes]
    encoder_tables = torch.arange(12, dtype=torch.int32, device="cuda").view(3, 4)
    for c, (k, v) in zip(encoder, states):
        de.append(c, k, v, place, encoder_tables, sequence=of)
    sequence = torch.arange(SEQUENCES, dtype=torch.int32, device="cuda").repeat_interleave(BEAMS)
    encoder_lengths = torch.tensor(encoded, dtype=torch.int32, device="cuda")[sequence.long()].contiguous()

    tables = torch.full((rows, most), -1, dtype=torch.int32, device="cuda")
    tables[:, 0] = pages[0]
    current, spare, unused = 0, 1, 2                        # sets: begun pages, those of the next step, not used yet
    lengths = torch.zeros(rows, dtype=torch.int32, device="cuda")
    tokens = torch.randint(0, WORDS, (rows,), generator=g, device="cuda")
    scores = torch.zeros((SEQUENCES, BEAMS), device="cuda")
    scores[:, 1:] = -math.inf
    scores, ended = scores.view(-1), torch.zeros(rows, dtype=torch.uint8, device="cuda")
    history = [[] for _ in range(rows)]
    for step in range(STEPS):
        history = [h + [t] for h, t in zip(history, tokens.tolist())]
        for i, (hq, hk, d) in enumerate(shapes):
            q, k, v = (t[tokens] for t in words[i])
            q = de.append(caches[i], k, v, lengths, tables, frequencies=frequencies[i], layout=layouts[i], q=q)
            a = de.attend(q, caches[i], tables, lengths + 1, max_length=step + 1)
            x = de.attend(q, encoder[i], encoder_tables, encoder_lengths, sequence=sequence)
            q64, err = turned64(words[i][0][tokens], lengths, frequencies[i], layouts[i], d)
            within(q, q64, err + 2.0 ** -8 * q64.abs())
            for r in range(0, rows, 5 if step % 9 else 1):
                at, n = torch.tensor(history[r], device="cuda"), len(history[r])
                held = [dense(t, tables[r], n) for t in caches[i]]
                turned = de.rotate(words[i][1][at], torch.arange(n, dtype=torch.int32, device="cuda"), frequencies[i], dim=d, layout=layouts[i])
                for got, want in zip(held, (turned, words[i][2][at])):
                    assert torch.equal(got, want.view(n, hk, d).transpose(0, 1)), (step, r, i)
                want, bound = attended64(q[r].view(hq, d), *held, d ** -0.5)
                within(a[r].view(hq, d), want, bound, (step, r, i))
                mine = of == sequence[r]
                want, bound = attended64(q[r].view(hq, d), *(t[mine].view(-1, hk, d).transpose(0, 1) for t in states[i]), d ** -0.5)
                within(x[r].view(hq, d), want, bound, (step, r, i))
        # rows in which 32 bits decide nothing that 64 bits would decide otherwise
        for _ in range(50):
            logits = 2.5 * normal(rows, WORDS)
            parents, chosen, best, over, c = chosen64(logits, scores, BEAMS, BEAMS, ended, END)
            top = c.sort(dim=1, descending=True).values[:, :BEAMS + 1]
            gap = top[:, :-1] - top[:, 1:]
            if not ((gap > 0) & (gap < 1e-4)).any():
                break
        b = de.beam(logits, scores, BEAMS, ended=ended, end=END)
        assert torch.equal(b.parents, parents) and torch.equal(b.tokens, chosen) and torch.equal(b.ended, over)
        if step + 1 == STEPS:
            break
        full = (step + 1) % PAGE == 0                       # the begun pages are complete: their rows keep them
        tables, lengths = de.fork(caches, tables, lengths + 1, b.parents, pages[unused if full else spare])
        if full:
            current, unused = unused, unused + 1
        else:
            current, spare = spare, current
        assert lengths.tolist() == [step + 1] * rows
        history = [history[p] for p in b.parents.view(-1).tolist()]
        tokens, scores, ended = b.tokens.view(-1).long(), b.scores.view(-1), b.ended.view(-1)
    assert int(ended.sum()) > 0


def test_example():
    """The example decoder runs, orders its beams, keeps ended ones, and one sequence's beams are the same alone."""
    from examples import beam_decoder as bd
    model = bd.build(blocks=2, d=128, f=192, heads=4, kv_heads=2, dim=32, words=97, end=5)
    lengths, steps = [9, 40, 17], 37
    states = torch.randn((sum(lengths), 128), device="cuda", generator=gen(2)).bfloat16()
    first = torch.zeros(3, dtype=torch.int64, device="cuda")
    said, scores = model(first, model.encode(states, lengths), 4, steps)
    assert said.shape == (3, 4, steps) and bool(torch.isfinite(scores).all())
    assert bool((scores[:, :-1] >= scores[:, 1:]).all()) and int(said.min()) >= 0 and int(said.max()) < 97
    for tokens in said.view(-1, steps).tolist():
        if 5 in tokens:
            assert set(tokens[tokens.index(5):]) == {5}
    for s in range(3):
        assert len({tuple(t) for t in said[s].tolist()}) == 4
        at = sum(lengths[:s])
        alone, alone_scores = model(first[:1], model.encode(states[at:at + lengths[s]], lengths[s:s + 1]), 4, steps)
        assert torch.equal(alone[0], said[s]) and torch.equal(alone_scores[0], scores[s])

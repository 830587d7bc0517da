"""Captured steps of the decoding operators: every output of every replay against the eager step's."""

import pytest
import torch

from tests.test_gpu_decode_calls import Inputs, ints, step

pytestmark = pytest.mark.gpu


def same(got, want, label):
    assert len(got) == len(want), label
    for i, (a, b) in enumerate(zip(got, want)):
        assert a.shape == b.shape and a.dtype == b.dtype and torch.equal(a, b), (label, i)


def test_replays_with_a_shared_workspace():
    """Two graphs, each with calls on one workspace among its own; replays on new inputs, eager steps and synchronizations between."""
    from paper_2307_04963_amd import decoding as de
    step.frequencies = de.frequencies(64)
    most = (5, 16, 700, 1100, 31, 0)
    static, room = Inputs(), torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    mask = torch.rand((6, 1120), device="cuda") < 0.8

    def calls(s, workspace):
        return step(de, s) + [de.attend(s.q, s.cache, s.tables, s.lengths, workspace=workspace),
                              de.attend(s.q, s.cache, s.tables, s.lengths, window=300, mask=mask, workspace=workspace),
                              *de.beam(s.logits, s.scores, 3, workspace=workspace)]

    calls(static, room)
    torch.cuda.synchronize()
    graphs, results = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            results.append(calls(static, room))
        graphs.append(graph)
    for i in range(6):
        for which in (i % 2, 1 - i % 2):
            new = Inputs(100 + 2 * i + which)
            new.lengths.copy_(torch.minimum(ints(*[(1, 15, 16, 17, 900, 3), (0, 0, 0, 0, 0, 0), (1000, 2, 40, 33, 64, 0)][i % 3]), ints(*most)))
            static.copy_(new)
            graphs[which].replay()
            if i % 2:
                torch.cuda.synchronize()
            got = [t.clone() for t in results[which]]
            same(got, calls(new, "auto"), (i, which))

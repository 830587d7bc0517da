"""Refused calls of the decoding operators leave nothing behind, no memory either."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("beams, k, word", [(3, 65, "k outside"), (3, 1 << 30, "k outside"), (65, 1 << 28, "beams outside")])
def test_refused_choice_allocates_nothing(beams, k, word):
    from paper_2307_04963_amd import decoding as de
    from paper_2307_04963_amd._lib import DyclError
    rows = 2 * beams
    logits, scores = torch.zeros((rows, 100), device="cuda"), torch.zeros(rows, device="cuda")
    torch.cuda.reset_peak_memory_stats()
    held = torch.cuda.memory_allocated()
    with pytest.raises(DyclError, match=word):
        de.beam(logits, scores, beams, k=k)
    assert torch.cuda.max_memory_allocated() == held
    none = de.beam(logits[:0], scores[:0], 3, k=5)
    assert [t.shape for t in none] == [(0, 5)] * 4

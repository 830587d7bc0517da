"""The expert stack on rows of a wider tensor, and on rows at any address: as on
the same rows packed."""

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_stack_on_strided_rows():
    from examples import expert_stack as es
    stack = es.build(*es.weights(3, 128, 64, 8, 20, seed=6), tau=0.6)
    g = torch.Generator(device="cuda").manual_seed(7)
    wide = torch.randn((500, 144), device="cuda", generator=g).bfloat16()
    flat = torch.empty(500 * 128 + 1, dtype=torch.bfloat16, device="cuda")
    for x in (wide[:, :128], wide[:, 3:131], wide[::2, 8:136], flat[1:].view(500, 128).copy_(wide[:, :128])):
        want, left = stack(x.clone(memory_format=torch.contiguous_format))
        logits, exits = stack(x)
        assert len(left.unique()) > 1                  # rows stay together past the first exit
        assert torch.equal(exits, left) and torch.equal(logits, want)

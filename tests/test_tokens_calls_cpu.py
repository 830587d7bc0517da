"""Refusals of the token operators' Python calls that need no GPU."""

from types import SimpleNamespace

import pytest
import torch

from paper_2307_04963_amd import experts as ex


def test_a_stream_of_another_device():
    """Work runs on the tensors' device: a stream of another one would be ignored there."""
    stream = SimpleNamespace(device=torch.device("cuda", 1))
    x, r = torch.zeros((4, 8)), ex.Routing(torch.zeros((4, 2)), torch.zeros((4, 2)), None, None, None)
    p = ex.Packed(torch.zeros(1024, dtype=torch.int16), 1, 8, 8, False)
    for call in (lambda: ex.norm(x, pre="rms", stream=stream), lambda: ex.route(x, 2, stream=stream), lambda: ex.pack(x, stream=stream),
                 lambda: ex.linear(x, p, stream=stream), lambda: ex.experts(x, r, p, p, stream=stream)):
        with pytest.raises(ValueError, match="stream belongs to cuda:1"):
            call()

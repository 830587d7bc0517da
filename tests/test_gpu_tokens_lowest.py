"""Experts closed by the type's lowest value instead of an infinity: they stay
open, come last, and do not push their group behind one with none open."""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

LOW = torch.finfo(torch.float32).min


@pytest.fixture(scope="module")
def ex():
    assert torch.cuda.is_available()
    from paper_2307_04963_amd import experts
    return experts


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E, groups, top", [(16, 4, 1), (16, 4, 2), (64, 8, 3), (256, 8, 4), (64, 64, 5), (1024, 16, 3)])
def test_groups_of_lowest_biases(ex, E, groups, top, score):
    from tests.test_gpu_tokens import apart, check_route
    size = E // groups
    z = apart(90, E, E)
    bias = torch.zeros(E, device="cuda")
    bias[size:] = LOW                                  # only the first group has others
    check_route(ex, z, min(8, top * size), score, bias, groups, top)
    z[::2, :size] = -math.inf                          # ... and in every other row it is closed
    got = check_route(ex, z, min(8, top * size), score, bias, groups, top)
    assert bool((got.ids >= 0).all())
    if size > 1:
        bias[size:2 * size] = LOW                      # one open expert beside lowest ones: ahead of a group of lowest ones only
        bias[E - 1] = 0.0
        got = check_route(ex, z[::2].contiguous(), min(8, top * size), score, bias, groups, top)
        assert bool((got.ids[:, 0] == E - 1).all())


def test_lowest_logits_in_groups(ex):
    from tests.test_gpu_tokens import apart, check_route
    z = apart(70, 32, 3)
    z[:, :24] = LOW
    z[::3, 24:] = -math.inf
    check_route(ex, z, 4, "softmax", None, 4, 2)
    check_route(ex, z, 4, "sigmoid", None, 4, 2)

"""The blend of frequencies by pairs, against values worked out by hand from its formula: with
p(t) = dims ln(trained / (2 pi t)) / (2 ln base), the pair that makes t turns, a pair i keeps the share
1 - (i - a) / (b - a), cut to [0, 1], a = p(fast) rounded down and b = p(slow) rounded up."""

import math

import pytest
import torch

from paper_2307_04963_amd import decoding as de


# dims, base, trained, slow, fast, factor; a, b; some pairs' shares
CASES = [
    # p(16) = 12.88, p(2) = 20.11: both within the pairs
    (64, 1e4, 4096, 2.0, 16.0, 8.0, 12, 21, {0: 1.0, 12: 1.0, 13: 8 / 9, 15: 2 / 3, 20: 1 / 9, 21: 0.0, 31: 0.0}),
    # p(32) = 45.03, p(1) = 69.11: every pair makes more than one turn, the last keeps a share
    (128, 1e4, 131072, 1.0, 32.0, 4.0, 45, 70, {44: 1.0, 45: 1.0, 46: 0.96, 63: 0.28}),
    # p(32) = 45.03 - 4.82 = 40.21, p(1) = 64.29
    (128, 1e4, 65536, 1.0, 32.0, 4.0, 40, 65, {40: 1.0, 41: 0.96, 60: 0.2, 63: 0.08}),
    # p(32) = 22.51, p(1) = 34.55
    (64, 1e4, 131072, 1.0, 32.0, 8.0, 22, 35, {22: 1.0, 26: 9 / 13, 31: 4 / 13}),
    # p(32) = -3.98, p(1) = 8.06: no pair makes 32 turns
    (64, 1e4, 64, 1.0, 32.0, 8.0, -4, 9, {0: 9 / 13, 1: 8 / 13, 8: 1 / 13, 9: 0.0, 31: 0.0}),
    # p(32) = -13.61, p(1) = -1.57: none makes one
    (64, 1e4, 4, 1.0, 32.0, 8.0, -14, -1, {0: 0.0, 1: 0.0, 31: 0.0}),
    # p(32) = 49.12, p(1) = 69.12: all make more than 32
    (8, 2.0, 1000000, 1.0, 32.0, 8.0, 49, 70, {0: 1.0, 3: 1.0}),
]


@pytest.mark.parametrize("dims, base, trained, slow, fast, factor, a, b, shares", CASES)
def test_blend_by_pairs(dims, base, trained, slow, fast, factor, a, b, shares):
    got = de.frequencies(dims, base, scaling="pairs", factor=factor, trained=trained, slow=slow, fast=fast, device="cpu")
    f = de.frequencies(dims, base, device="cpu")
    assert got.dtype == torch.float64 and len(got) == dims // 2
    for i in range(dims // 2):
        keep = min(1.0, max(0.0, 1 - (i - a) / (b - a)))
        if i in shares:
            assert abs(keep - shares[i]) < 1e-12
        want = float(f[i]) * (keep + (1 - keep) / factor)
        assert abs(float(got[i]) - want) <= 1e-13 * want, i


def test_blend_by_pairs_between_its_ends():
    """A pair that makes `fast` turns or more is kept, one that makes `slow` or fewer divided, whatever the trained context; the rounding of
    the ends moves them by less than a pair."""
    for dims in (16, 64, 128):
        for trained in (1, 7, 100, 4096, 30000, 1 << 17, 1 << 20, 1 << 30):
            got = de.frequencies(dims, scaling="pairs", factor=8.0, trained=trained, slow=1.0, fast=32.0, device="cpu")
            f = de.frequencies(dims, device="cpu")
            step = 10000.0 ** (2 / dims)                   # between the turns of neighbours
            for i in range(dims // 2):
                turns, kept = trained * float(f[i]) / (2 * math.pi), float(got[i] / f[i])
                if turns >= 32 * step:
                    assert abs(kept - 1) < 1e-12
                elif turns * step <= 1:
                    assert abs(kept - 1 / 8) < 1e-12
                elif 1 < turns < 32:
                    assert 1 / 8 < kept < 1


@pytest.mark.parametrize("base", [1.0, 0.5])
def test_blend_by_pairs_needs_falling_frequencies(base):
    with pytest.raises(ValueError, match="base"):
        de.frequencies(64, base, scaling="pairs", factor=4.0, trained=4096, device="cpu")

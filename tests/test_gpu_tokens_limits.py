"""The token operators where one launch does not hold all their rows."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ex():
    assert torch.cuda.is_available()
    from paper_2307_04963_amd import experts
    return experts


def test_route_more_rows_than_a_launch_holds(ex):
    """Blocks of 64 rows by 512 threads: beyond 2^29 rows they are 2^32 threads, more than a launch takes."""
    n = (1 << 29) + 67
    print(f"[limits] route n={n}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(3)
    z = torch.randint(-3, 4, (n, 2), dtype=torch.int8, device="cuda", generator=g).to(torch.bfloat16)
    r = ex.route(z, 1)
    second = z[:, 1] > z[:, 0]                    # equal ones go to the lowest index
    del z
    assert torch.equal(r.ids[:, 0], second.int())
    assert bool((r.weights == 1.0).all())
    ones = int(second.sum())
    assert r.offsets.tolist() == [0, n - ones, n]
    for flags, lo, hi in ((~second, 0, n - ones), (second, n - ones, n)):
        rows = flags.nonzero()[:, 0].int()
        assert torch.equal(r.order[lo:hi], rows)
        assert torch.equal(r.slots[rows.long(), 0], torch.arange(lo, hi, dtype=torch.int32, device="cuda"))


def test_pack_more_than_a_launch_holds(ex):
    """257 x 2^15 strips of weights: beyond the 2^23 - 1 workgroups of a launch."""
    print("[limits] pack 257 x 2^20 x 1", flush=True)
    g = torch.Generator(device="cuda").manual_seed(4)
    w = torch.randint(-100, 101, (257, 1 << 20, 1), dtype=torch.int8, device="cuda", generator=g).to(torch.bfloat16)
    packed = ex.pack(w).data.view(257, -1)
    for e in (0, 128, 255, 256):
        assert torch.equal(packed[e], ex.pack(w[e]).data)

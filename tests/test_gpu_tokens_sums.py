"""Each output of the experts' layers on its own: what its neighbours hold, large
or not finite, does not take its digits."""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ex():
    assert torch.cuda.is_available()
    from paper_2307_04963_amd import experts
    return experts


@pytest.mark.parametrize("n", [1, 40, 700])
@pytest.mark.parametrize("k", [1, 3])
def test_outputs_beside_much_larger_ones(ex, n, k):
    d, f, E = 72, 40, 4
    g = torch.Generator(device="cuda").manual_seed(n + k)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    size = torch.tensor([2.0 ** -p for p in (0, 12, 20, 3, 40, 1, 10, 70)], device="cuda").repeat(9)
    up, down = normal(E, f, d).bfloat16(), (normal(E, d, f) * size[None, :, None]).bfloat16()
    x, ids = normal(n, d).bfloat16(), torch.topk(normal(n, E), k).indices
    logits = torch.full((n, E), -math.inf, device="cuda").scatter_(1, ids, normal(n, k))
    r = ex.route(logits, k)
    got = ex.experts(x, r, ex.pack(up), ex.pack(down), act="relu").double()
    want, bound = torch.zeros_like(got), torch.zeros_like(got)
    for e in range(E):
        t, j = torch.where(r.ids == e)
        if len(t):
            w = r.weights[t, j].double()[:, None]
            hidden = (x[t].double() @ up[e].double().t().contiguous()).clamp(min=0)
            w2 = down[e].double().t().contiguous()
            want.index_add_(0, t, w * (hidden @ w2))
            # sums in 32 bits are off by at most 2^-16 of their magnitudes' sum; hidden is rounded to bf16, 2^-8 of it
            off = 2.0 ** -16 * (x[t].double().abs() @ up[e].double().abs().t().contiguous())
            bound.index_add_(0, t, w * ((off + (2.0 ** -8 + 2.0 ** -16) * (hidden + off)) @ w2.abs()))
    bound += 2.0 ** -8 * (want.abs() + bound)
    assert bool(((got - want).abs() <= bound).all())


def test_outputs_beside_infinite_ones(ex):
    d, f, n = 64, 32, 50
    g = torch.Generator(device="cuda").manual_seed(9)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    up, down, x = normal(2, f, d).bfloat16(), normal(2, d, f).bfloat16(), normal(n, d).bfloat16()
    r = ex.route(normal(n, 2), 2)
    want = ex.experts(x, r, ex.pack(up), ex.pack(down), act="silu")
    down[1, 13] = math.inf
    down[0, 40] = math.nan
    got = ex.experts(x, r, ex.pack(up), ex.pack(down), act="silu")
    rest = torch.ones(d, dtype=torch.bool, device="cuda")
    rest[13] = rest[40] = False
    assert torch.equal(got[:, rest], want[:, rest])
    assert not bool(torch.isfinite(got[:, ~rest]).any())

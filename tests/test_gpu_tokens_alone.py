"""A row's results do not depend on the rows beside it: every token operator gives
a row the same bits alone, among a few others and among thousands, whichever
kernel their number selects."""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

B, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ex():
    assert torch.cuda.is_available()
    from paper_2307_04963_amd import experts
    return experts


def normal(g, *s):
    return torch.randn(s, generator=g, device="cuda")


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("K, N, out", [(1024, 768, B), (4096, 256, B), (200, 1000, F), (72, 40, F), (2048, 4096, B)])
def test_linear(ex, K, N, out, gated):
    g = torch.Generator(device="cuda").manual_seed(K + N)
    n = 9000
    mk = lambda: (normal(g, N, K) / math.sqrt(K)).bfloat16()  # noqa: E731
    w = ex.pack(mk(), mk() if gated else None)
    bias, gate_bias = normal(g, N), normal(g, N) if gated else None
    x, r = normal(g, n, K).bfloat16(), normal(g, n, N).bfloat16()
    run = lambda rows: ex.linear(x[rows], w, bias=bias, gate_bias=gate_bias, act="silu", residual=r[rows], out_dtype=out)  # noqa: E731
    whole = run(slice(0, n))
    for m in (1, 2, 7, 16, 17, 32, 40, 64, 65, 100, 130, 200, 256, 300, 520, 700, 1030, 1536, 2100, 4100):
        assert torch.equal(run(slice(0, m)), whole[:m]), m
        assert torch.equal(run(slice(n - m, n)), whole[n - m:]), m
    some = torch.randperm(n, generator=g, device="cuda")[:77]
    assert torch.equal(run(some), whole[some])


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("d, f", [(256, 192), (1024, 512), (100, 72)])
def test_experts(ex, d, f, gated):
    E, k, n = 8, 2, 6000
    g = torch.Generator(device="cuda").manual_seed(d + f)
    mk = lambda a, b: (normal(g, E, a, b) / math.sqrt(b)).bfloat16()  # noqa: E731
    w, w2 = ex.pack(mk(f, d), mk(f, d) if gated else None), ex.pack(mk(d, f))
    x, r = normal(g, n, d).bfloat16(), normal(g, n, d).bfloat16()
    logits = normal(g, n, E) + normal(g, E)
    run = lambda rows: ex.experts(x[rows], ex.route(logits[rows], k), w, w2, act="gelu", residual=r[rows])  # noqa: E731
    whole = run(slice(0, n))
    for m in (1, 3, 16, 50, 130, 300, 1000, 3000):
        assert torch.equal(run(slice(0, m)), whole[:m]), m
    some = torch.randperm(n, generator=g, device="cuda")[:99]
    assert torch.equal(run(some), whole[some])


def test_norm_and_route(ex):
    g = torch.Generator(device="cuda").manual_seed(1)
    n, d, E = 5000, 1000, 96
    x, y, logits = normal(g, n, d).bfloat16(), normal(g, n, d).bfloat16(), normal(g, n, E)
    norm = lambda rows: ex.norm(x[rows], y[rows], post="rms", pre="layer")  # noqa: E731
    route = lambda rows: ex.route(logits[rows], 5, groups=6, top_groups=3)  # noqa: E731
    h, u = norm(slice(0, n))
    whole = route(slice(0, n))
    for m in (1, 5, 64, 65, 1024, 3000):
        a, b = norm(slice(0, m))
        assert torch.equal(a, h[:m]) and torch.equal(b, u[:m])
        r = route(slice(0, m))
        assert torch.equal(r.ids, whole.ids[:m]) and torch.equal(r.weights, whole.weights[:m])


def test_a_stack_of_blocks(ex):
    """A row of the expert stack takes the same experts, leaves at the same block and gets the same logits in any company."""
    from examples import expert_stack as es
    stack = es.build(*es.weights(3, 256, 128, 16, 50, seed=2), tau=0.6)
    x = normal(torch.Generator(device="cuda").manual_seed(4), 3000, 256).bfloat16()
    logits, exits = stack(x)
    assert len(exits.unique()) > 2
    for rows in ([0], [7], [2999], list(range(40)), list(range(500, 1700))):
        a, b = stack(x[rows])
        assert torch.equal(b, exits[rows]) and torch.equal(a, logits[rows])

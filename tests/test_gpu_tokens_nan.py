"""NaN and infinities through the layers' activations: what the definition gives,
NaN for NaN, each infinity for itself."""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

ACT64 = {"none": lambda v: v, "relu": lambda v: v.clamp(min=0), "gelu": lambda v: v * 0.5 * torch.special.erfc(-v / math.sqrt(2)),
         "silu": lambda v: v * torch.sigmoid(v)}


@pytest.fixture(scope="module")
def ex():
    assert torch.cuda.is_available()
    from paper_2307_04963_amd import experts
    return experts


def same_kind(got, want):
    got = got.double()
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got == math.inf, want == math.inf) and torch.equal(got == -math.inf, want == -math.inf)


@pytest.mark.parametrize("m", [6, 300, 2100])
@pytest.mark.parametrize("act", list(ACT64))
@pytest.mark.parametrize("gated", [False, True])
def test_linear(ex, m, act, gated):
    # one input and weights of 1: the value itself comes to the activation
    values = torch.tensor([math.nan, math.inf, -math.inf, -3.0, 0.0, 2.5], device="cuda")
    x = values[torch.arange(m, device="cuda") % 6][:, None].bfloat16()
    w = torch.ones((40, 1), device="cuda").bfloat16()
    got = ex.linear(x, ex.pack(w, w if gated else None), act=act, out_dtype=torch.float32)
    v = x.double().expand(m, 40)
    same_kind(got, v * ACT64[act](v) if gated else ACT64[act](v))


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_experts(ex, act):
    g = torch.Generator(device="cuda").manual_seed(1)
    mk = lambda a, b: torch.randn((2, a, b), generator=g, device="cuda").bfloat16()  # noqa: E731
    x = torch.randn((70, 64), generator=g, device="cuda").bfloat16()
    x[5, 3] = math.nan
    r = ex.route(torch.randn((70, 2), generator=g, device="cuda"), 1)
    got = ex.experts(x, r, ex.pack(mk(32, 64)), ex.pack(mk(64, 32)), act=act)
    assert bool(got[5].isnan().all()) and bool(torch.isfinite(got[:5]).all()) and bool(torch.isfinite(got[6:]).all())

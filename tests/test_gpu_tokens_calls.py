"""Python calls of the token operators that must not pass silently."""

import pytest
import torch

pytestmark = pytest.mark.gpu

B = torch.bfloat16


@pytest.fixture(scope="module")
def ex():
    assert torch.cuda.is_available()
    from paper_2307_04963_amd import experts
    return experts


def test_tensors_that_require_grad(ex):
    x = torch.ones((4, 64), dtype=B, device="cuda")
    w = torch.ones((8, 64), dtype=B, device="cuda")
    p, p1, p2 = ex.pack(w), ex.pack(torch.ones((4, 32, 64), dtype=B, device="cuda")), ex.pack(torch.ones((4, 64, 32), dtype=B, device="cuda"))
    logits = torch.zeros((4, 4), device="cuda")
    r = ex.route(logits, 2)
    scale = torch.ones(64, device="cuda")
    want = lambda t: t.detach().clone().requires_grad_()  # noqa: E731
    calls = [lambda f: ex.norm(f(x), pre="rms"), lambda f: ex.norm(x, f(x), post="rms"), lambda f: ex.norm(x, pre="rms", pre_weight=f(scale)),
             lambda f: ex.route(f(logits), 2), lambda f: ex.pack(f(w)), lambda f: ex.linear(f(x), p), lambda f: ex.linear(x, p, bias=f(scale[:8])),
             lambda f: ex.experts(f(x), r, p1, p2), lambda f: ex.experts(x, r._replace(weights=f(r.weights)), p1, p2),
             lambda f: ex.linear(x, p, residual=f(torch.ones((4, 8), dtype=B, device="cuda")))]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError, match="requires grad"):
            call(want)
            print("accepted:", i)
        with torch.no_grad():
            call(want)
        with torch.inference_mode():
            call(lambda t: t)
        call(lambda t: want(t).detach())


def test_a_norm_of_nothing(ex):
    """Without y, a pre norm or a scale x is the result as it is; weights and norms given all the same are a mistake."""
    from paper_2307_04963_amd._lib import DyclError
    x, w, r = torch.ones((4, 64), dtype=B, device="cuda"), torch.ones(64, device="cuda"), torch.ones(4, device="cuda")
    assert ex.norm(x)[0] is x
    for more in ({}, {"pre": "rms"}):
        for bad in ({"post": "rms"}, {"post_weight": w}, {"post_bias": w}, {"channel_scale": w}, {"row_gate": r}, {"gate": x}):
            with pytest.raises((ValueError, DyclError)):
                ex.norm(x, **bad, **more)
                print("accepted:", bad, more)
    for bad in ({"pre_weight": w}, {"pre_bias": w}):
        with pytest.raises((ValueError, DyclError)):
            ex.norm(x, **bad)

"""Tensors that carry a forward-mode tangent are refused by the token and the decoding operators, which would drop it."""

import pytest
import torch
from torch.autograd import forward_ad

from paper_2307_04963_amd import decoding as de, experts as ex

B = torch.bfloat16


def calls(x, k):
    """One call per tensor argument of a floating type, `x` [4, 64] (a dual one) in its place."""
    i, t = torch.zeros(4, dtype=torch.int32), torch.zeros((4, 2), dtype=torch.int32)
    c, f = de.cache(2, 1, 8, 64, device="cpu"), torch.zeros(4, dtype=torch.float64)
    plain = torch.zeros((4, 64), dtype=x.dtype)
    routing = ex.Routing(plain[:, :2], plain[:, :2], i, i, t)
    packed = ex.Packed(torch.zeros(64, dtype=torch.uint8), 1, 64, 64, False)
    return [lambda: de.rotate(x, i, f, dim=64), lambda: de.rotate(plain, i, f, dim=64, out=x), lambda: de.append(c, x, plain, i, t),
            lambda: de.append(c, plain, x, i, t), lambda: de.append(c, plain, plain, i, t, q=x), lambda: de.append(c._replace(keys=k), plain, plain, i, t),
            lambda: de.attend(x, c, t, i), lambda: de.attend(plain, c._replace(values=k), t, i), lambda: de.beam(x, plain[:, 0], 4),
            lambda: de.beam(plain, x[:, 0], 4), lambda: de.fork(c._replace(keys=k), t, i, i, i),
            lambda: ex.norm(x), lambda: ex.norm(plain, x), lambda: ex.route(x, 2), lambda: ex.pack(x), lambda: ex.linear(x, packed),
            lambda: ex.linear(plain, packed, residual=x), lambda: ex.experts(x, routing, packed, packed)]


@pytest.mark.parametrize("dtype", [B, torch.float32])
@pytest.mark.parametrize("no_grad", [False, True])
def test_tangents_are_refused(dtype, no_grad):
    x, k = torch.zeros((4, 64), dtype=dtype), torch.zeros((2, 1, 8, 64), dtype=B)
    with forward_ad.dual_level(), torch.set_grad_enabled(not no_grad):
        dual, dual_k = forward_ad.make_dual(x, torch.ones_like(x)), forward_ad.make_dual(k, torch.ones_like(k))
        for n, call in enumerate(calls(dual, dual_k)):
            with pytest.raises(ValueError, match="tangent"):
                call()
                print("accepted:", n)
        # without its tangent it comes to the next check
        for call in calls(forward_ad.unpack_dual(dual).primal, forward_ad.unpack_dual(dual_k).primal):
            with pytest.raises(ValueError, match="on a GPU"):
                call()
    for call in calls(x, k):
        with pytest.raises(ValueError, match="on a GPU"):
            call()

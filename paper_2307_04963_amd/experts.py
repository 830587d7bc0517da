"""The token operators of include/dycl_tokens.h on torch tensors: the norms
around a block with its gate and residual scale, the choice of experts, a layer
with its epilogue, and the chosen experts' layers.  This file gives the
arguments names and defaults; _tokens.so (csrc/binding) checks the tensors and
calls libdycl.so, where every kernel is.

Matrices are 2-D tensors whose last dimension is contiguous (rows may be
strided).  Work is queued on ``stream`` (default: the current one); what a call
allocates belongs to that stream.  Wrong tensors raise ValueError, other
refusals DyclError.  Nothing here has a backward: tensors that require grad are
refused where gradients are recorded (call under torch.no_grad()).
"""

from __future__ import annotations

from typing import NamedTuple

import torch

from . import _lib

try:
    from . import _tokens
except ImportError as e:
    raise ImportError("_tokens.so is not built; run `python -m paper_2307_04963_amd.build` (needs hipcc and g++)") from e

_tokens.set_error(_lib.DyclError)

NORMS = {"none": 0, "rms": 1, "layer": 2}
GATE_ACTS = {"none": 0, "sigmoid": 1, "silu": 2}
ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
SCORES = {"softmax": 0, "sigmoid": 1}
_F32 = {torch.bfloat16: 0, torch.float32: 1}


def _of(table: dict, key, what: str) -> int:
    try:
        return table[key]
    except (KeyError, TypeError):
        raise ValueError(f"{what} must be one of {[str(k) for k in table]}") from None


def _call(stream, f, *args):
    """f on the given stream; args[0] is the tensor that says where the call runs."""
    if stream is None:
        return f(*args)
    if isinstance(args[0], torch.Tensor) and stream.device != args[0].device:
        raise ValueError(f"the stream belongs to {stream.device}, the tensors to {args[0].device}")
    with torch.cuda.stream(stream):
        return f(*args)


def _room(workspace):
    """workspace: "auto" (allocate what is needed), None or a tensor; returns (tensor or None, allocate)."""
    return (None, 1) if isinstance(workspace, str) else (workspace, 0)


def norm(x: torch.Tensor, y: torch.Tensor | None = None, *, post: str = "none", post_weight=None, post_bias=None, gate=None,
         gate_act: str = "none", row_gate=None, channel_scale=None, residual_scale: float = 1.0, pre: str = "none",
         pre_weight=None, pre_bias=None, eps: float = 1e-6, h: torch.Tensor | None = None, u: torch.Tensor | None = None,
         u_dtype=torch.bfloat16, stream=None):
    """dycl_op_norm: z = post(y) * act(gate) * channel_scale * row_gate, h = residual_scale * x + z, u = pre(h).

    x [n, d] (bf16 or float32) is the residual stream, y and gate [n, d] the
    block's output and gate (both bf16 or both float32), row_gate [n],
    channel_scale and the norms' weights and biases [d] float32.  A row whose
    row_gate is 0 was skipped by the block: its y and gate are not read.
    Returns (h, u): h is x itself where nothing changes it (no y,
    residual_scale 1, no h given), u is None without a pre norm.
    """
    h_out, u_out = _call(stream, _tokens.norm, x, y, _of(NORMS, post, "post"), post_weight, post_bias, gate,
                         _of(GATE_ACTS, gate_act, "gate_act"), row_gate, channel_scale, residual_scale, _of(NORMS, pre, "pre"),
                         pre_weight, pre_bias, eps, h, u, _of(_F32, u_dtype, "u_dtype"))
    return x if h_out is None else h_out, u_out


class Routing(NamedTuple):
    """What dycl_op_route writes: ids and weights [n, k]; offsets [experts + 1],
    order [n * k] and slots [n, k] are the partition of the (row, choice) pairs
    by expert (None where it was not asked for)."""
    ids: torch.Tensor
    weights: torch.Tensor
    offsets: torch.Tensor | None
    order: torch.Tensor | None
    slots: torch.Tensor | None


def route(logits: torch.Tensor, k: int, *, score: str = "softmax", bias=None, groups: int = 1, top_groups: int | None = None,
          mask=None, renormalise: bool = True, scale: float = 1.0, partition: bool = True, workspace="auto",
          stream=None) -> Routing:
    """dycl_op_route: the k best experts of every row of logits [n, experts]
    (bf16 or float32) by softmax or sigmoid score plus bias [experts], within
    the top_groups best of `groups` runs of experts, their weights, and the
    partition of the pairs by expert.  Experts whose logit is -inf or NaN are
    closed to that row; rows with mask [n] (uint8 or bool) 0 choose nothing."""
    return Routing(*_call(stream, _tokens.route, logits, k, _of(SCORES, score, "score"), bias, groups,
                          groups if top_groups is None else top_groups, mask, renormalise, scale, partition, *_room(workspace)))


class Packed(NamedTuple):
    """Weights laid out by dycl_op_linear_pack: `experts` layers of n outputs
    on k inputs, gated or not."""
    data: torch.Tensor
    experts: int
    n: int
    k: int
    gated: bool


def pack(w: torch.Tensor, gate: torch.Tensor | None = None, *, stream=None) -> Packed:
    """dycl_op_linear_pack: w [n, k] (one layer) or [experts, n, k] bf16, and the
    gate's weights of the same shape."""
    data = _call(stream, _tokens.pack, w, gate)
    experts, n, k = (1, *w.shape) if w.dim() == 2 else w.shape
    return Packed(data, experts, n, k, gate is not None)


def linear(x: torch.Tensor, packed: Packed, *, bias=None, gate_bias=None, act: str = "none", residual=None, out=None,
           out_dtype=torch.bfloat16, workspace="auto", stream=None) -> torch.Tensor:
    """dycl_op_linear: act(x W^T + bias) + residual, or with packed gate weights
    (x W^T + bias) * act(x G^T + gate_bias) + residual; x [m, k] and residual
    [m, n] bf16, biases [n] float32; returns y [m, n] in out_dtype."""
    return _call(stream, _tokens.linear, x, *packed, bias, gate_bias, _of(ACTS, act, "act"), residual, out,
                 _of(_F32, out_dtype, "out_dtype"), *_room(workspace))


def experts(x: torch.Tensor, routing: Routing, packed: Packed, packed2: Packed, *, act: str = "silu", bias=None, gate_bias=None,
            bias2=None, residual=None, out=None, workspace="auto", stream=None) -> torch.Tensor:
    """dycl_op_experts: residual + the sum over each row's choices of weight *
    (W2 f(x) + bias2), f the chosen expert's first layer (packed, gated or not,
    bias and gate_bias [experts, f]), packed2 its second; x, residual and the
    result [n, d] bf16."""
    return _call(stream, _tokens.experts, x, routing.weights, routing.offsets, routing.order, routing.slots, *packed, *packed2,
                 _of(ACTS, act, "act"), bias, gate_bias, bias2, residual, out, *_room(workspace))

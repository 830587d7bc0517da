"""The token operators of include/dycl_tokens.h on device tensors (argument
checks and marshalling only): the norms around a block with its gate and
residual scale, the choice of experts, a layer with its epilogue, and the
chosen experts' layers.  Every kernel is in libdycl.so.

Matrices are 2-D tensors whose last dimension is contiguous (rows may be
strided).  Work is queued on ``stream`` (default: the current one); what a call
allocates belongs to that stream.
"""

from __future__ import annotations

import contextlib
from typing import NamedTuple

import torch

from . import _lib

check = _lib.check
lib = _lib.lib

NORMS = {"none": 0, "rms": 1, "layer": 2}
GATE_ACTS = {"none": 0, "sigmoid": 1, "silu": 2}
ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
SCORES = {"softmax": 0, "sigmoid": 1}
TYPES = {torch.bfloat16: 0, torch.float32: 1}


def _ptr(t):
    return None if t is None else t.data_ptr()


def _choice(table: dict, name: str, what: str) -> int:
    if name not in table:
        raise ValueError(f"{what} must be one of {sorted(table)}")
    return table[name]


def _matrix(t: torch.Tensor, what: str, rows: int, cols: int, dtypes, device) -> int:
    """Checks a matrix; returns its row pitch in elements."""
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != cols:
        raise ValueError(f"{what} must be [{rows}, {cols}], not {list(t.shape)}")
    if t.dtype not in dtypes:
        raise ValueError(f"{what} must be {' or '.join(str(d) for d in dtypes)}, not {t.dtype}")
    if t.device != device:
        raise ValueError(f"{what} is on {t.device}, not on {device}")
    if cols > 1 and t.stride(1) != 1:
        raise ValueError(f"{what}: the last dimension must be contiguous")
    if rows <= 1:
        return max(cols, t.stride(0))
    if t.stride(0) < cols:
        raise ValueError(f"{what}: rows overlap")
    return t.stride(0)


def _vector(t, what: str, shape, device, dtype=torch.float32):
    if t is None:
        return None
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{what} must be a contiguous {dtype} tensor {list(shape)} on {device}")
    return t.data_ptr()


def _input(t: torch.Tensor, what: str) -> tuple[int, int]:
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError(f"{what} must be a 2-D tensor")
    if not t.is_cuda:
        raise ValueError(f"{what} must be on a GPU")
    return t.shape[0], t.shape[1]


def _on(stream, device):
    """The stream to queue on, and a context in which allocations belong to it."""
    current = torch.cuda.current_stream(device)
    if stream is None or stream == current:
        return current, contextlib.nullcontext()
    return stream, torch.cuda.stream(stream)


def _workspace(workspace, nbytes: int, device):
    """workspace: "auto" (allocate), or a device tensor of at least nbytes; returns (tensor, bytes)."""
    if not nbytes:
        return None, 0
    if isinstance(workspace, str):
        return torch.empty(nbytes, dtype=torch.uint8, device=device), nbytes
    if workspace is None or workspace.device != device or not workspace.is_contiguous():
        raise ValueError(f"needs a contiguous workspace of {nbytes} bytes on {device}")
    return workspace, workspace.numel() * workspace.element_size()


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
    n, d = _input(x, "x")
    dev = x.device
    post_k, pre_k, act = _choice(NORMS, post, "post"), _choice(NORMS, pre, "pre"), _choice(GATE_ACTS, gate_act, "gate_act")
    ldx = _matrix(x, "x", n, d, TYPES, dev)
    ldy = ldg = d
    if y is not None:
        ldy = _matrix(y, "y", n, d, TYPES, dev)
    if gate is not None:
        if y is None:
            raise ValueError("a gate needs y")
        ldg = _matrix(gate, "gate", n, d, (y.dtype,), dev)
    vectors = [_vector(row_gate, "row_gate", (n,), dev), _vector(channel_scale, "channel_scale", (d,), dev),
               _vector(post_weight, "post_weight", (d,), dev), _vector(post_bias, "post_bias", (d,), dev),
               _vector(pre_weight, "pre_weight", (d,), dev), _vector(pre_bias, "pre_bias", (d,), dev)]
    if u is not None and pre_k == 0:
        raise ValueError("u needs a pre norm")
    s, own = _on(stream, dev)
    with own:
        keep = h is None and y is None and residual_scale == 1.0
        if h is None and not keep:
            h = torch.empty((n, d), dtype=x.dtype, device=dev)
        if u is None and pre_k:
            u = torch.empty((n, d), dtype=u_dtype, device=dev)
    ldh = d if h is None else _matrix(h, "h", n, d, (x.dtype,), dev)
    ldu = d if u is None else _matrix(u, "u", n, d, TYPES, dev)
    if h is not None or u is not None:
        check(lib.dycl_op_norm(x.data_ptr(), TYPES[x.dtype], ldx, _ptr(y), TYPES[y.dtype] if y is not None else 0, ldy, _ptr(gate),
                               ldg, act, vectors[0], vectors[1], float(residual_scale), post_k, vectors[2], vectors[3], pre_k,
                               vectors[4], vectors[5], float(eps), n, d, _ptr(h), ldh, _ptr(u),
                               TYPES[u.dtype] if u is not None else 0, ldu, s.cuda_stream))
    return x if h is None else h, u


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
    n, E = _input(logits, "logits")
    dev = logits.device
    kind = _choice(SCORES, score, "score")
    ldl = _matrix(logits, "logits", n, E, TYPES, dev)
    if mask is not None and mask.dtype == torch.bool:
        mask = mask.view(torch.uint8)
    if k < 1 or k > E:
        raise ValueError(f"k must be between 1 and the {E} experts")
    bias_p, mask_p = _vector(bias, "bias", (E,), dev), _vector(mask, "mask", (n,), dev, torch.uint8)
    s, own = _on(stream, dev)
    with own:
        ids = torch.empty((n, k), dtype=torch.int32, device=dev)
        weights = torch.empty((n, k), dtype=torch.float32, device=dev)
        offsets = order = slots = None
        if partition:
            offsets = torch.empty(E + 1, dtype=torch.int32, device=dev)
            order = torch.empty(n * k, dtype=torch.int32, device=dev)
            slots = torch.empty((n, k), dtype=torch.int32, device=dev)
        ws, wsb = _workspace(workspace, lib.dycl_op_route_workspace(n, E, k) if partition else 0, dev)
    check(lib.dycl_op_route(logits.data_ptr(), TYPES[logits.dtype], ldl, bias_p, mask_p, n, E, groups,
                            groups if top_groups is None else top_groups, k, kind, int(renormalise), float(scale), ids.data_ptr(),
                            weights.data_ptr(), _ptr(offsets), _ptr(order), _ptr(slots), _ptr(ws), wsb, s.cuda_stream))
    return Routing(ids, weights, offsets, order, slots)


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
    if not isinstance(w, torch.Tensor) or w.dim() not in (2, 3) or w.dtype != torch.bfloat16 or not w.is_cuda:
        raise ValueError("w must be a bfloat16 tensor [n, k] or [experts, n, k] on a GPU")
    if gate is not None and (gate.shape != w.shape or gate.dtype != w.dtype or gate.device != w.device):
        raise ValueError("gate must be like w")
    experts, n, k = (1, *w.shape) if w.dim() == 2 else w.shape
    s, own = _on(stream, w.device)
    with own:
        w, gate = w.contiguous(), None if gate is None else gate.contiguous()
        nbytes = lib.dycl_op_linear_packed_bytes(experts, n, k, int(gate is not None))
        data = torch.empty(nbytes // 2, dtype=torch.int16, device=w.device)
    check(lib.dycl_op_linear_pack(w.data_ptr(), _ptr(gate), experts, n, k, data.data_ptr(), nbytes, s.cuda_stream))
    return Packed(data, experts, n, k, gate is not None)


def linear(x: torch.Tensor, packed: Packed, *, bias=None, gate_bias=None, act: str = "none", residual=None, out=None,
           out_dtype=torch.bfloat16, workspace="auto", stream=None) -> torch.Tensor:
    """dycl_op_linear: act(x W^T + bias) + residual, or with packed gate weights
    (x W^T + bias) * act(x G^T + gate_bias) + residual; x [m, k] and residual
    [m, n] bf16, biases [n] float32; returns y [m, n] in out_dtype."""
    m, k = _input(x, "x")
    dev = x.device
    if packed.experts != 1 or packed.k != k or packed.data.device != dev:
        raise ValueError(f"packed must be one layer on {k} inputs on {dev}")
    n = packed.n
    code = _choice(ACTS, act, "act")
    ldx = _matrix(x, "x", m, k, (torch.bfloat16,), dev)
    ldr = n if residual is None else _matrix(residual, "residual", m, n, (torch.bfloat16,), dev)
    bias_p, gbias_p = _vector(bias, "bias", (n,), dev), _vector(gate_bias, "gate_bias", (n,), dev)
    s, own = _on(stream, dev)
    with own:
        y = out if out is not None else torch.empty((m, n), dtype=out_dtype, device=dev)
        ws, wsb = _workspace(workspace, lib.dycl_op_linear_workspace(x.data_ptr(), ldx, m, k, n, int(packed.gated)), dev)
    ldy = _matrix(y, "out", m, n, TYPES, dev)
    check(lib.dycl_op_linear(x.data_ptr(), ldx, m, k, packed.data.data_ptr(), n, int(packed.gated), bias_p, gbias_p, code,
                             _ptr(residual), ldr, y.data_ptr(), TYPES[y.dtype], ldy, _ptr(ws), wsb, s.cuda_stream))
    return y


def experts(x: torch.Tensor, routing: Routing, packed: Packed, packed2: Packed, *, act: str = "silu", bias=None, gate_bias=None,
            bias2=None, residual=None, out=None, workspace="auto", stream=None) -> torch.Tensor:
    """dycl_op_experts: residual + the sum over each row's choices of weight *
    (W2 f(x) + bias2), f the chosen expert's first layer (packed, gated or not,
    bias and gate_bias [experts, f]), packed2 its second; x, residual and the
    result [n, d] bf16."""
    n, d = _input(x, "x")
    dev = x.device
    E, f = packed.experts, packed.n
    if packed.k != d or packed2.experts != E or packed2.n != d or packed2.k != f or packed2.gated:
        raise ValueError(f"packed must be layers of {d} inputs, packed2 ungated layers back of as many experts")
    if packed.data.device != dev or packed2.data.device != dev:
        raise ValueError(f"packed weights must be on {dev}")
    code = _choice(ACTS, act, "act")
    if routing.offsets is None or routing.weights.dim() != 2:
        raise ValueError("routing must hold a partition")
    k = routing.weights.shape[1]
    lists = [_vector(routing.weights, "routing.weights", (n, k), dev), _vector(routing.offsets, "routing.offsets", (E + 1,), dev, torch.int32),
             _vector(routing.order, "routing.order", (n * k,), dev, torch.int32), _vector(routing.slots, "routing.slots", (n, k), dev, torch.int32)]
    ldx = _matrix(x, "x", n, d, (torch.bfloat16,), dev)
    ldr = d if residual is None else _matrix(residual, "residual", n, d, (torch.bfloat16,), dev)
    b1, g1, b2 = _vector(bias, "bias", (E, f), dev), _vector(gate_bias, "gate_bias", (E, f), dev), _vector(bias2, "bias2", (E, d), dev)
    s, own = _on(stream, dev)
    with own:
        y = out if out is not None else torch.empty((n, d), dtype=torch.bfloat16, device=dev)
        ws, wsb = _workspace(workspace, lib.dycl_op_experts_workspace(x.data_ptr(), ldx, n, E, k, d, f), dev)
    ldo = _matrix(y, "out", n, d, (torch.bfloat16,), dev)
    check(lib.dycl_op_experts(x.data_ptr(), ldx, n, d, f, E, k, packed.data.data_ptr(), int(packed.gated), b1, g1, code,
                              packed2.data.data_ptr(), b2, *lists, _ptr(residual), ldr, y.data_ptr(), ldo, _ptr(ws), wsb,
                              s.cuda_stream))
    return y

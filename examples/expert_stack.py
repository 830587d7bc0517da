"""A stack of expert blocks whose rows leave early: the token operators run
together as a serving program runs them, with the routing primitives that the
batched executor uses between its decisions.

Each block normalises the residual stream (with the block before's output, its
post-norm and its scale), scores the experts, sends every row through its own
k of them, and hands the weighted sum on.  In front of each block an exit head
looks at the normalised state: confident rows leave with its logits
(dycl_op_compact splits the rows, dycl_op_move_rows brings those that stay
together), so later blocks run on fewer rows, down to one.

    python -m examples.expert_stack --rows 4096 --blocks 4
"""

from __future__ import annotations

import argparse
import math
from typing import NamedTuple

import torch

from paper_2307_04963_amd import _lib, experts as ex


class Block(NamedTuple):
    """One block's weights as the operators take them (products packed once)."""
    pre_weight: torch.Tensor       # [d] float32, the norm before the block
    post_weight: torch.Tensor      # [d] float32, the norm after it
    scale: torch.Tensor            # [d] float32, its residual scale
    router: ex.Packed              # d -> experts
    balance: torch.Tensor          # [experts] float32, added to the scores that are compared
    up: ex.Packed                  # experts layers d -> f, gated
    down: ex.Packed                # experts layers f -> d


class Stack:
    def __init__(self, blocks, last_weight, head: ex.Packed, k: int, groups: int, top_groups: int, tau: float):
        self.blocks, self.last_weight, self.head = blocks, last_weight, head
        self.k, self.groups, self.top_groups, self.tau = k, groups, top_groups, tau

    def __call__(self, x: torch.Tensor, trace=None):
        """x [n, d] bf16 -> (logits [n, classes] float32, exit index [n] int32:
        the number of blocks a row went through).  trace, a list, receives each
        block's (row ids, routing)."""
        n, dev = x.shape[0], x.device
        logits = torch.empty((n, self.head.n), dtype=torch.float32, device=dev)
        exits = torch.zeros(n, dtype=torch.int32, device=dev)
        rows = torch.arange(n, dtype=torch.int32, device=dev)
        h, y, before = x, None, None
        for i in range(len(self.blocks) + 1):
            last = i == len(self.blocks)
            pre = self.last_weight if last else self.blocks[i].pre_weight
            h, u = ex.norm(h, y, post="none" if y is None else "rms", post_weight=None if y is None else before.post_weight,
                           channel_scale=None if y is None else before.scale, pre="rms", pre_weight=pre)
            z = ex.linear(u, self.head, out_dtype=torch.float32)
            leaves = torch.ones(len(rows), dtype=torch.uint8, device=dev) if last else \
                (torch.softmax(z, 1).amax(1) >= self.tau).to(torch.uint8)
            (gone, gone_rows), (stay, stay_rows) = partition(leaves, rows)
            logits[gone_rows.long()] = z[gone.long()]
            exits[gone_rows.long()] = i
            if last or len(stay) == 0:
                break
            h, u, rows = gather(h, stay), gather(u, stay), stay_rows
            before = self.blocks[i]
            routing = ex.route(ex.linear(u, before.router, out_dtype=torch.float32), self.k, score="sigmoid", bias=before.balance,
                               groups=self.groups, top_groups=self.top_groups)
            if trace is not None:
                trace.append((rows, routing))
            y = ex.experts(u, routing, before.up, before.down, act="silu")
        return logits, exits


def partition(flags: torch.Tensor, rows: torch.Tensor):
    """dycl_op_compact: (positions, ids) of the rows with a set flag, and of the others."""
    n, dev = len(flags), flags.device
    lists = [torch.empty(n, dtype=torch.int32, device=dev) for _ in range(4)]
    counts = torch.empty(2, dtype=torch.int32, device=dev)
    nbytes = _lib.lib.dycl_op_compact_workspace(n)
    ws = torch.empty(max(nbytes, 8), dtype=torch.uint8, device=dev)
    _lib.check(_lib.lib.dycl_op_compact(flags.data_ptr(), rows.data_ptr(), n, *[t.data_ptr() for t in lists], counts.data_ptr(),
                                        ws.data_ptr(), nbytes, torch.cuda.current_stream(dev).cuda_stream))
    a, b = counts.tolist()
    return (lists[0][:a], lists[1][:a]), (lists[2][:b], lists[3][:b])


def gather(t: torch.Tensor, positions: torch.Tensor) -> torch.Tensor:
    """dycl_op_move_rows: the rows of t at `positions` (row bytes a multiple of 16).  It takes packed, 16-byte aligned rows;
    others, which the operators read where they are, are packed first."""
    if not t.is_contiguous() or t.data_ptr() % 16:
        t = t.clone(memory_format=torch.contiguous_format)
    out = torch.empty((len(positions), t.shape[1]), dtype=t.dtype, device=t.device)
    _lib.check(_lib.lib.dycl_op_move_rows(out.data_ptr(), None, t.data_ptr(), positions.data_ptr(), t.shape[1] * t.element_size(),
                                          len(positions), torch.cuda.current_stream(t.device).cuda_stream))
    return out


def weights(blocks: int, d: int, f: int, experts: int, classes: int, seed: int = 0, device="cuda"):
    """Random weights of a stack, unpacked: a list of dicts and the head's."""
    g = torch.Generator(device=device).manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=g, device=device)  # noqa: E731
    layer = lambda *s: (normal(*s) / math.sqrt(s[-1])).bfloat16()  # noqa: E731
    made = [{"pre_weight": 1 + 0.1 * normal(d), "post_weight": 1 + 0.1 * normal(d), "scale": 0.5 + 0.1 * normal(d),
             "router": layer(experts, d), "balance": 0.02 * normal(experts), "up": layer(experts, f, d), "gate": layer(experts, f, d),
             "down": layer(experts, d, f)} for _ in range(blocks)]
    return made, {"weight": 1 + 0.1 * normal(d), "head": (4 * layer(classes, d).float()).bfloat16()}


def build(made, head, k=2, groups=4, top_groups=2, tau=0.9) -> Stack:
    blocks = [Block(b["pre_weight"], b["post_weight"], b["scale"], ex.pack(b["router"]), b["balance"], ex.pack(b["up"], b["gate"]),
                    ex.pack(b["down"])) for b in made]
    return Stack(blocks, head["weight"], ex.pack(head["head"]), k, groups, top_groups, tau)


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, default in (("rows", 4096), ("blocks", 4), ("d", 1024), ("f", 512), ("experts", 32), ("classes", 100)):
        p.add_argument(f"--{name}", type=int, default=default)
    p.add_argument("--tau", type=float, default=0.9)
    a = p.parse_args()
    stack = build(*weights(a.blocks, a.d, a.f, a.experts, a.classes), tau=a.tau)
    x = torch.randn((a.rows, a.d), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).bfloat16()
    stack(x)
    torch.cuda.synchronize()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    logits, exits = stack(x)
    end.record()
    torch.cuda.synchronize()
    print(f"{a.rows} rows, {a.blocks} blocks of {a.experts} experts: {begin.elapsed_time(end):.3f} ms; rows that left before each block:",
          torch.bincount(exits, minlength=a.blocks + 1).tolist(), "finite:", bool(torch.isfinite(logits).all()))


if __name__ == "__main__":
    main()

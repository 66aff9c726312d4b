"""One transformer block's MoE half that drops nothing, put together from the library's entry points: norm, routing, rows sorted
by expert, the experts' products on them, rows brought back with their weights, and the join with the residual stream and
the next block's norm in one pass; and its backward, for the same routing.

    h = N(x) w_pre;  gate = softmax(cos(pooled h, w_emb));  y = sum over a token's k best experts of gate W_down (SiLU(W_gate h) (W_up h))
    x_out = x + N(y) w_post;  h_next = N(x_out) w_next

A capacity-bounded layer keeps [E][capacity] buffers and drops what they cannot hold (etr_moe_forward); here every chosen
pair has a row, T * k of them in all.  The class owns its buffers, so that a step allocates nothing and can be captured into a graph.

    python -m paper_2406_00023_amd.dropless_block          # one step of 4096 tokens, timed
"""
from __future__ import annotations

from dataclasses import dataclass

import torch

from . import binding as B
from . import inputs as I


@dataclass
class BlockShape:
    T: int
    d: int
    E: int
    D: int
    k: int
    H: int
    dtype: torch.dtype = torch.bfloat16
    gate_norm: int = 0


class DroplessBlock:
    WEIGHTS = ("w_pre", "w_post", "w_next", "w_gate", "w_up", "w_down")

    def __init__(self, s: BlockShape, device="cuda"):
        self.s = s
        T, d, E, k, H, dt = s.T, s.d, s.E, s.k, s.H, s.dtype
        R = T * k
        self.layer = B.EtrConfig(T, d, E, s.D, k, T, H, I.DT_F32 if dt == torch.float32 else I.DT_BF16, I.MODE_TCR, I.COS_FULL,
                                 s.gate_norm)                  # capacity T: token choice keeps every pair
        self.norm = B.make_norm_config(T, d, dt)
        self.sort = B.make_sort_config(T, k, E, d, dt, gate_norm=s.gate_norm)
        self.up = B.make_linear_config(R, d, H, E, dt, act=B.ACT_SWIGLU)
        self.down = B.make_linear_config(R, H, d, E, dt)

        def rows(n, width):
            return torch.zeros(n, width, dtype=dt, device=device)

        def i32(*n):
            return torch.zeros(*n, dtype=torch.int32, device=device)

        def f32(*n):
            return torch.zeros(*n, dtype=torch.float32, device=device)

        self.h, self.y, self.x_out, self.h_next = (rows(T, d) for _ in range(4))
        self.hs, self.ys, self.dhs, self.dys = (rows(R, d) for _ in range(4))
        self.a, self.pre, self.pre_up, self.da = (rows(R, H) for _ in range(4))
        self.dx, self.dy, self.dh = (rows(T, d) for _ in range(3))
        self.score, self.gate, self.dgate = f32(T, E), f32(T, E), f32(T, E)
        self.topk, self.slot_of, self.slot_token, self.counts = i32(T, k), i32(T, E), i32(E, T), i32(E)
        self.offsets, self.row_of, self.pair_of = i32(E + 1), i32(T, k), i32(R)
        self.grads = {"w_pre": f32(d), "w_post": f32(d), "w_next": f32(d)}
        self.grads.update({n: torch.zeros(E, *sh, dtype=dt, device=device) for n, sh in (("w_gate", (H, d)), ("w_up", (H, d)), ("w_down", (d, H)))})
        # the stages follow each other on one stream: they share one workspace
        self.ws = B.alloc_workspace(max(B.etr_select_workspace_bytes(self.layer), B.etr_sort_workspace_bytes(self.sort),
                                        B.etr_norm_workspace_bytes(self.norm), B.etr_linear_workspace_bytes(self.up),
                                        B.etr_linear_workspace_bytes(self.down)), device)

    def forward(self, x, w_emb, w):
        """x [T][d], w_emb [E][d/D] fp32, w: the tensors of WEIGHTS; returns (x_out, h_next)."""
        B.etr_block_norm(self.norm, x, w_pre=w["w_pre"], h=self.h)
        B.etr_route(self.layer, self.h, w_emb, self.score, self.gate)
        B.etr_select(self.layer, self.score, self.topk, self.slot_of, self.slot_token, self.counts, self.ws)
        B.etr_sort_tokens(self.sort, self.topk, None, self.offsets, self.row_of, self.pair_of, self.ws)
        B.etr_sort_rows(self.sort, self.h, self.row_of, self.hs)
        B.etr_expert_linear(self.up, self.hs, self.offsets, w["w_gate"], self.a, w_up=w["w_up"], pre=self.pre, pre_up=self.pre_up)
        B.etr_expert_linear(self.down, self.a, self.offsets, w["w_down"], self.ys)
        B.etr_unsort_rows(self.sort, self.ys, self.gate, self.topk, self.row_of, self.y)
        B.etr_block_norm(self.norm, x, self.y, None, w["w_post"], w["w_next"], self.x_out, self.h_next)
        return self.x_out, self.h_next

    def backward(self, x, w_emb, w, dx_out, dh_next):
        """Gradients of the last forward call: returns dx; those of the tensors of WEIGHTS are in `grads`.  The experts' embeddings w_emb are constants
        of the method and get none."""
        g = self.grads
        B.etr_block_norm_backward(self.norm, self.x_out, self.y, None, w["w_post"], w["w_next"], dx_out, dh_next, self.dx, self.dy, None,
                                  g["w_post"], g["w_next"], self.ws)
        B.etr_unsort_rows_backward(self.sort, self.dy, self.ys, self.gate, self.topk, self.row_of, self.dys, self.dgate)
        B.etr_expert_linear_backward(self.down, self.a, self.offsets, w["w_down"], self.dys, self.ws, dx=self.da, dw=g["w_down"])
        B.etr_expert_linear_backward(self.up, self.hs, self.offsets, w["w_gate"], self.da, self.ws, w_up=w["w_up"], pre=self.pre,
                                     pre_up=self.pre_up, dx=self.dhs, dw=g["w_gate"], dw_up=g["w_up"])
        B.etr_sort_rows_backward(self.sort, self.dhs, self.row_of, self.dh)
        B.etr_route_backward(self.layer, self.h, w_emb, self.score, self.gate, self.dgate, self.dh, self.dh)
        B.etr_block_norm_backward(self.norm, x, None, None, None, w["w_pre"], self.dx, self.dh, self.dx, dw_pre=g["w_pre"], ws=self.ws)
        return self.dx


def random_weights(s: BlockShape, seed: int = 1, device="cuda"):
    """Embeddings with orthonormal rows and weights of the block, from a seed."""
    gen = torch.Generator().manual_seed(seed)

    def normal(*n, std=1.0):
        return torch.randn(*n, generator=gen) * std

    w_emb = torch.linalg.qr(normal(s.d // s.D, s.E))[0].t().contiguous().to(device)
    w = {n: (1 + normal(s.d, std=0.1)).to(device) for n in ("w_pre", "w_post", "w_next")}
    for n, shape, std in (("w_gate", (s.E, s.H, s.d), s.d ** -0.5), ("w_up", (s.E, s.H, s.d), s.d ** -0.5), ("w_down", (s.E, s.d, s.H), s.H ** -0.5)):
        w[n] = normal(*shape, std=std).to(s.dtype).to(device)
    return w_emb, w


def main():
    s = BlockShape(T=4096, d=1024, E=16, D=16, k=2, H=2816)
    block = DroplessBlock(s)
    w_emb, w = random_weights(s)
    x, dx_out, dh = (torch.randn(s.T, s.d, device="cuda").to(s.dtype) for _ in range(3))
    events = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
    for step in range(12):
        if step == 2:
            events[0].record()
        block.forward(x, w_emb, w)
        block.backward(x, w_emb, w, dx_out, dh)
    events[1].record()
    torch.cuda.synchronize()
    rows = (block.offsets[1:] - block.offsets[:-1]).tolist()
    print(f"forward and backward of {s.T} tokens, {s.E} experts of {min(rows)} to {max(rows)} rows: {events[0].elapsed_time(events[1]) / 10:.3f} ms")


if __name__ == "__main__":
    main()

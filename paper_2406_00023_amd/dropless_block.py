"""One transformer block's MoE half that drops nothing, put together from the library's entry points: norm, routing, rows sorted
by expert, the experts' products on them, rows brought back with their weights, and the join with the residual stream and
the next block's norm in one pass; and its backward, for the same routing.

    h = N(x) w_pre;  gate = softmax(cos(pooled h, w_emb));  y = sum over a token's k best experts of gate W_down (SiLU(W_gate h) (W_up h))
    x_out = x + N(y) w_post;  h_next = N(x_out) w_next

A capacity-bounded layer keeps [E][capacity] buffers and drops what they cannot hold (etr_moe_forward); here every chosen
pair has a row, T * k of them in all.  The class owns its buffers, so that a step allocates nothing and can be captured into a graph.

PackedBlock is the same block with the experts in 8 bits: tokens are packed as they are sorted, the experts' products take packed operands, and
what a step keeps for its backward (the sorted tokens, the pre-activations, the activation) is kept packed, half of what bf16 takes.

    python -m paper_2406_00023_amd.dropless_block          # one step of 4096 tokens, timed, with and without packing
"""
from __future__ import annotations

import weakref
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
        self.ys, self.dhs, self.dys = (rows(R, d) for _ in range(3))
        self.da = rows(R, H)
        self.dx, self.dy, self.dh = (rows(T, d) for _ in range(3))
        self.score, self.gate, self.dgate = f32(T, E), f32(T, E), f32(T, E)
        self.topk, self.slot_of, self.slot_token, self.counts = i32(T, k), i32(T, E), i32(E, T), i32(E)
        self.offsets, self.row_of, self.pair_of = i32(E + 1), i32(T, k), i32(R)
        self.grads = {"w_pre": f32(d), "w_post": f32(d), "w_next": f32(d)}
        self.grads.update({n: torch.zeros(E, *sh, dtype=dt, device=device) for n, sh in (("w_gate", (H, d)), ("w_up", (H, d)), ("w_down", (d, H)))})
        # the stages follow each other on one stream: they share one workspace
        self.ws = B.alloc_workspace(max(B.etr_select_workspace_bytes(self.layer), B.etr_sort_workspace_bytes(self.sort),
                                        B.etr_norm_workspace_bytes(self.norm), self._prepare_experts(device)), device)

    def _prepare_experts(self, device):
        """Buffers of the experts' stages; returns the bytes of scratch that they take."""
        s, R = self.s, self.s.T * self.s.k
        self.hs = torch.zeros(R, s.d, dtype=s.dtype, device=device)
        self.a, self.pre, self.pre_up = (torch.zeros(R, s.H, dtype=s.dtype, device=device) for _ in range(3))
        return max(B.etr_linear_workspace_bytes(self.up), B.etr_linear_workspace_bytes(self.down))

    def _experts(self, w):
        """From the normed tokens h to the experts' rows ys."""
        B.etr_sort_rows(self.sort, self.h, self.row_of, self.hs)
        B.etr_expert_linear(self.up, self.hs, self.offsets, w["w_gate"], self.a, w_up=w["w_up"], pre=self.pre, pre_up=self.pre_up)
        B.etr_expert_linear(self.down, self.a, self.offsets, w["w_down"], self.ys)

    def _experts_backward(self, w):
        """From the gradient dys of the experts' rows to dhs, that of the sorted tokens, and the weights' gradients."""
        g = self.grads
        B.etr_expert_linear_backward(self.down, self.a, self.offsets, w["w_down"], self.dys, self.ws, dx=self.da, dw=g["w_down"])
        B.etr_expert_linear_backward(self.up, self.hs, self.offsets, w["w_gate"], self.da, self.ws, w_up=w["w_up"], pre=self.pre,
                                     pre_up=self.pre_up, dx=self.dhs, dw=g["w_gate"], dw_up=g["w_up"])

    def forward(self, x, w_emb, w):
        """x [T][d], w_emb [E][d/D] fp32, w: the tensors of WEIGHTS; returns (x_out, h_next)."""
        B.etr_block_norm(self.norm, x, w_pre=w["w_pre"], h=self.h)
        B.etr_route(self.layer, self.h, w_emb, self.score, self.gate)
        B.etr_select(self.layer, self.score, self.topk, self.slot_of, self.slot_token, self.counts, self.ws)
        B.etr_sort_tokens(self.sort, self.topk, None, self.offsets, self.row_of, self.pair_of, self.ws)
        self._experts(w)
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
        self._experts_backward(w)
        B.etr_sort_rows_backward(self.sort, self.dhs, self.row_of, self.dh)
        B.etr_route_backward(self.layer, self.h, w_emb, self.score, self.gate, self.dgate, self.dh, self.dh)
        B.etr_block_norm_backward(self.norm, x, None, None, None, w["w_pre"], self.dx, self.dh, self.dx, dw_pre=g["w_pre"], ws=self.ws)
        return self.dx


EXPERT_WEIGHTS = ("w_gate", "w_up", "w_down")


class _Source:
    """Which tensor was packed: the memory that it looks at (not kept alive), which part of it, and how often torch has changed that in place."""

    def __init__(self, t: torch.Tensor):
        self.memory, self.rest = weakref.ref(t.untyped_storage()), self._rest(t)

    @staticmethod
    def _rest(t):
        return t.storage_offset(), t.shape, t.dtype, None if t.is_inference() else t._version

    def __call__(self, t: torch.Tensor) -> bool:
        """Whether t is that tensor, unchanged."""
        return self.memory() is t.untyped_storage() and self.rest == self._rest(t)


class PackedBlock(DroplessBlock):
    """The block with the experts in 8 bits.  Its products take the weights as pack_weights last packed them, forward and backward, so that it has to
    follow every change of the experts' weights.  forward refuses experts' weights that are not what was packed: other tensors, or the same ones after an
    operation of torch in place.  What torch does not count it cannot see (a replayed graph, `.data`, inference tensors, writes through an address).
    A caller who keeps the packed weights only leaves the experts' out of w.

    exact_sums: the product whose results are packed (pre-activations and activation) sums in fp32 also in a bf16 block, at half the rate of the 8-bit
    matrix pipe.  Without it some 1 in 600 to 1200 of these values, next to a tie, is packed a step of e4m3 away from the nearest."""

    def __init__(self, s: BlockShape, device="cuda", exact_sums: bool = False):
        self.exact_sums = exact_sums
        super().__init__(s, device)

    def _prepare_experts(self, device):
        s, R, E, d, H, dt = self.s, self.s.T * self.s.k, self.s.E, self.s.d, self.s.H, self.s.dtype
        dp, Hp = -(-d // 128) * 128, -(-H // 128) * 128

        def rows(n, width, E=1):
            return B.alloc_packed_rows(B.make_pack_config(n, width, dt, E=E), device)

        def columns(width):
            return B.alloc_packed_columns(B.make_pack_config(R, width, dt, E=E, sorted=1), device)

        # kept for the backward: the sorted tokens, both pre-activations, the activation
        self.hs8, self.a8, self.pre8, self.pre_up8 = rows(R, d), rows(R, H), rows(R, H), rows(R, H)
        # gradients along rows (for the next ones down) and along columns (for the weights'), and what was kept along columns
        self.dys8, self.dab8 = rows(R, d), rows(R, 2 * Hp)
        self.dyst8, self.dabt8, self.hst8, self.at8 = columns(d), columns(2 * H), columns(d), columns(H)
        self.w8 = {"w_gate": rows(H, d, E), "w_up": rows(H, d, E), "w_down": rows(d, H, E), "up_t": rows(d, 2 * Hp, E), "down_t": rows(H, d, E)}
        self.rows_up, self.rows_down = B.make_pack_config(H, d, dt, E=E), B.make_pack_config(d, H, dt, E=E)
        self.sorted_h, self.sorted_a = B.make_pack_config(R, d, dt, E=E, sorted=1), B.make_pack_config(R, H, dt, E=E, sorted=1)
        self.dx_up, self.dx_down = B.make_linear_config(R, 2 * Hp, d, E, dt), B.make_linear_config(R, dp, H, E, dt)
        self.up_packing = B.make_linear_config(R, d, H, E, torch.float32 if self.exact_sums else dt, act=B.ACT_SWIGLU)
        self.packed = None                                     # the weights that are packed, by name; they only say what forward refuses
        return max(B.etr_packed_act_workspace_bytes(self.up), B.etr_packed_act_workspace_bytes(self.down))

    def pack_weights(self, w):
        """The experts' weights along rows, for the forward products, and along columns, for their input's gradients."""
        self.packed = None                                     # (until all of them are)
        q = self.w8
        for n, cfg in (("w_gate", self.rows_up), ("w_up", self.rows_up), ("w_down", self.rows_down)):
            B.etr_pack_rows(cfg, w[n], q[n])
        B.etr_pack_columns_pair(self.rows_up, w["w_gate"], w["w_up"], q["up_t"])
        B.etr_pack_columns(self.rows_down, w["w_down"], None, q["down_t"])
        self.packed = {n: _Source(w[n]) for n in EXPERT_WEIGHTS}

    def __getstate__(self):
        """A copy holds the packed weights, and does not know whose they are."""
        return {**self.__dict__, "packed": self.packed and dict.fromkeys(self.packed)}

    def forward(self, x, w_emb, w):
        if self.packed is None:
            raise RuntimeError("PackedBlock.forward before pack_weights: the experts' weights are not packed yet")
        for n in EXPERT_WEIGHTS:
            if n in w and not (self.packed[n] and self.packed[n](w[n])):
                raise RuntimeError(f"PackedBlock.forward: {n} is not what pack_weights has packed, or has changed since; pack it again")
        return super().forward(x, w_emb, w)

    def _experts(self, w):
        q = self.w8
        B.etr_pack_sorted_rows(self.sort, self.h, self.row_of, self.hs8)
        B.etr_packed_linear(self.up_packing, self.hs8, self.offsets, q["w_gate"], w_up8=q["w_up"], y8=self.a8, pre8=self.pre8, pre_up8=self.pre_up8)
        B.etr_packed_linear(self.down, self.a8, self.offsets, q["w_down"], y=self.ys)

    def _experts_backward(self, w):
        g, q = self.grads, self.w8
        B.etr_packed_act_backward(self.down, self.dys, self.offsets, d8=self.dys8, dt8=self.dyst8)
        B.etr_packed_linear(self.dx_down, self.dys8, self.offsets, q["down_t"], y=self.da)
        B.etr_repack_columns(self.sorted_a, self.a8, self.offsets, self.at8)
        B.etr_packed_weight_gradient(self.down, self.dyst8, self.at8, self.offsets, g["w_down"])
        B.etr_packed_act_backward(self.up, self.da, self.offsets, pre8=self.pre8, pre_up8=self.pre_up8, d8=self.dab8, dt8=self.dabt8)
        B.etr_packed_linear(self.dx_up, self.dab8, self.offsets, q["up_t"], y=self.dhs)
        B.etr_repack_columns(self.sorted_h, self.hs8, self.offsets, self.hst8)
        B.etr_packed_weight_gradient(self.up, self.dabt8, self.hst8, self.offsets, g["w_gate"], dw_up=g["w_up"])


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
    w_emb, w = random_weights(s)
    x, dx_out, dh = (torch.randn(s.T, s.d, device="cuda").to(s.dtype) for _ in range(3))
    for kind in (DroplessBlock, PackedBlock):
        block = kind(s)
        events = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        for step in range(12):
            if step == 2:
                events[0].record()
            if kind is PackedBlock:
                block.pack_weights(w)                          # as after an optimizer's step
            block.forward(x, w_emb, w)
            block.backward(x, w_emb, w, dx_out, dh)
        events[1].record()
        torch.cuda.synchronize()
        rows = (block.offsets[1:] - block.offsets[:-1]).tolist()
        print(f"{kind.__name__}: forward and backward of {s.T} tokens, {s.E} experts of {min(rows)} to {max(rows)} rows: "
              f"{events[0].elapsed_time(events[1]) / 10:.3f} ms")


if __name__ == "__main__":
    main()

"""The operators around the layer put together against the fused layer (etr_moe_forward, etr_moe_backward) on the same routing: a layer that
drops nothing, and one whose capacity drops pairs, which the sorted rows leave out by its slot table."""
import pytest
import torch

from paper_2406_00023_amd import binding as B
from paper_2406_00023_amd import inputs as I

pytestmark = pytest.mark.gpu

# relative 2-norms.  fp32: sums of up to 328 terms in different orders, several one behind the other.  bf16: the stages' roundings, half a
# step (2^-8) at most each and about six along a path on either side, which add up in squares
TOL = {I.DT_F32: 2e-5, I.DT_BF16: 2e-2}
SHAPES = [dict(T=333, d=256, E=8, D=8, k=2, H=136, dtype=I.DT_F32), dict(T=700, d=512, E=4, D=16, k=3, H=328, dtype=I.DT_BF16)]


def _off(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm())


@pytest.mark.parametrize("gate_norm", [0, 1])
@pytest.mark.parametrize("cos", [I.COS_FULL, I.COS_POOLED])
@pytest.mark.parametrize("mode,share", [(I.MODE_TCR, 1.0), (I.MODE_BIDIR, 0.15)])
@pytest.mark.parametrize("sizes", SHAPES)
def test_forward_and_gradients(sizes, mode, share, cos, gate_norm):
    T, d, E, k, H = (sizes[n] for n in ("T", "d", "E", "k", "H"))
    shape = I.EtrShape("chain", 1, capacity=max(1, int(share * T)), mode=mode, recipe="iso", **sizes)
    dt, C = shape.torch_dtype, shape.capacity
    t, dout = I.make_inputs(shape, "cuda"), I.make_upstream_gradient(shape, "cuda")
    cfg = B.make_config(shape, cos=cos, gate_norm=gate_norm)
    new = lambda *n, ty=dt: torch.full(n, 7, dtype=ty, device="cuda")
    f32, i32 = torch.float32, torch.int32
    # the layer
    score, gate, out = new(T, E, ty=f32), new(T, E, ty=f32), new(T, d)
    topk, slot_of, slot_token, counts = new(T, k, ty=i32), new(T, E, ty=i32), new(E, C, ty=i32), new(E, ty=i32)
    B.etr_moe_forward(cfg, t["x"], t["w_emb"], t["w_gate"], t["w_up"], t["w_down"], out, B.alloc_workspace(B.etr_workspace_bytes(cfg)), score=score,
                      gate=gate, topk_expert=topk, slot_of=slot_of, slot_token=slot_token, counts=counts)
    want = dict(dx=new(T, d), dw_gate=new(E, H, d), dw_up=new(E, H, d), dw_down=new(E, d, H), dgate=new(T, E, ty=f32), dscore=new(T, E, ty=f32))
    B.etr_moe_backward(cfg, t["x"], t["w_emb"], t["w_gate"], t["w_up"], t["w_down"], score, gate, slot_of, slot_token, counts, dout, want["dx"],
                       want["dw_gate"], want["dw_up"], want["dw_down"], B.alloc_workspace(B.etr_backward_workspace_bytes(cfg)), dgate=want["dgate"],
                       dscore=want["dscore"])
    # the chain
    R = T * k
    sort = B.make_sort_config(T, k, E, d, dt, gate_norm=gate_norm)
    up, down = B.make_linear_config(R, d, H, E, dt, act=B.ACT_SWIGLU), B.make_linear_config(R, H, d, E, dt)
    ws = B.alloc_workspace(max(B.etr_sort_workspace_bytes(sort), B.etr_linear_workspace_bytes(up), B.etr_linear_workspace_bytes(down)))
    offsets, row_of, pair_of = new(E + 1, ty=i32), new(T, k, ty=i32), new(R, ty=i32)
    B.etr_sort_tokens(sort, topk, slot_of, offsets, row_of, pair_of, ws)
    xs, ys, dys, dxs, a, pre, pre_up, da, y = new(R, d), new(R, d), new(R, d), new(R, d), new(R, H), new(R, H), new(R, H), new(R, H), new(T, d)
    got = dict(dx=new(T, d), dw_gate=new(E, H, d), dw_up=new(E, H, d), dw_down=new(E, d, H), dgate=new(T, E, ty=f32))
    B.etr_sort_rows(sort, t["x"], row_of, xs)
    B.etr_expert_linear(up, xs, offsets, t["w_gate"], a, w_up=t["w_up"], pre=pre, pre_up=pre_up)
    B.etr_expert_linear(down, a, offsets, t["w_down"], ys)
    B.etr_unsort_rows(sort, ys, gate, topk, row_of, y)
    B.etr_unsort_rows_backward(sort, dout, ys, gate, topk, row_of, dys, got["dgate"])
    B.etr_expert_linear_backward(down, a, offsets, t["w_down"], dys, ws, dx=da, dw=got["dw_down"])
    B.etr_expert_linear_backward(up, xs, offsets, t["w_gate"], da, ws, w_up=t["w_up"], pre=pre, pre_up=pre_up, dx=dxs, dw=got["dw_gate"], dw_up=got["dw_up"])
    B.etr_sort_rows_backward(sort, dxs, row_of, got["dx"])
    experts = got["dx"].clone()
    B.etr_route_backward(cfg, t["x"], t["w_emb"], score, gate, got["dgate"], got["dx"], got["dx"])
    torch.cuda.synchronize()
    kept = int(offsets[-1])
    assert kept == int(counts.sum()) and (kept == R if mode == I.MODE_TCR else 0 < kept < R)
    tol = TOL[sizes["dtype"]]
    assert _off(y, out) <= tol
    for n, v in got.items():
        assert _off(v, want[n]) <= tol, n
    dscore = gate.double() * (want["dgate"].double() - (want["dgate"].double() * gate.double()).sum(1, keepdim=True))
    assert _off(want["dscore"], dscore) <= 2e-5
    if dt != f32:                                              # (bf16's rounding of the layer's dx is as large as the term)
        return
    # the router's term by itself: what the layer's dx has beside the experts' part
    term, size = want["dx"].double() - experts.double(), float(want["dx"].double().norm())
    alone = new(T, d)
    B.etr_route_backward(cfg, t["x"], t["w_emb"], score, gate, want["dgate"], None, alone)
    torch.cuda.synchronize()
    assert float(term.norm()) > 0.01 * size
    assert float((alone.double() - term).norm()) <= 2 * tol * size

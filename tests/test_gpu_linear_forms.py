"""Every form of the experts' products, element by element against the definition in 64 bits, and the same bits on a second call whose
workspace and outputs hold something else."""
import pytest
import torch

import linear_forms as F
import test_gpu_expert_linear as L
from operator_refs import DT, U32, activation, assert_within, half_step, randn
from paper_2406_00023_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("product,dtype,act,form,rows,E,K,N", F.listed(F.FORWARD))
def test_forward_of_each_form(product, dtype, act, form, rows, E, K, N):
    assert F.plan(product, dtype, act, rows, E, K, N) == form
    counts, spare = F.counts(rows, E)
    L.test_forward(counts, spare, K, N, act, True, True, True, dtype)


@pytest.mark.parametrize("product,dtype,act,form,rows,E,K,N", F.listed(F.INPUT, F.WEIGHT, F.JOINT))
def test_backward_of_each_form(product, dtype, act, form, rows, E, K, N):
    assert F.plan(product, dtype, act, rows, E, K, N) == form
    print(f"linear backward, product {product} {dtype} {act} form {form}: rows {rows} of {E}, K {K} N {N}", flush=True)
    dt, glu = DT[dtype], act == "swiglu"
    counts, spare = F.counts(rows, E)
    used = rows - spare
    s = L._inputs(counts, spare, K, N, dt, act, False, False, seed=21)
    pre, pre_up, dy = (randn(i, rows, N, dtype=dt) for i in (41, 42, 43))
    for v in (pre, pre_up, dy):
        v[used:] = float("nan")
    g, off = L._cuda(s), L._offsets(counts).cuda()
    up = [v.cuda() for v in (dy, pre, pre_up)]
    cfg = B.make_linear_config(rows, K, N, E, dt, act=F.ACT[act])
    got = []
    for fill, byte in ((7.0, 255), (-3.0, 85)):
        out = {}
        if product != F.WEIGHT:
            out["dx"] = torch.full((rows, K), fill, dtype=dt, device="cuda")
        if product != F.INPUT:
            out.update({n: torch.full((E, N, K), fill, dtype=dt, device="cuda") for n in (("dw", "dw_up") if glu else ("dw",))})
        ws = torch.full((B.etr_linear_workspace_bytes(cfg),), byte, dtype=torch.uint8, device="cuda")
        B.etr_expert_linear_backward(cfg, g["x"] if product != F.INPUT else None, off, g["w"] if product != F.WEIGHT else None, up[0], ws,
                                     w_up=g["w_up"] if product != F.WEIGHT else None, pre=up[1] if glu else None, pre_up=up[2] if glu else None, **out)
        torch.cuda.synchronize()
        if "dx" in out:
            assert bool((out["dx"][used:] == fill).all())
        got.append(out)
    for n, v in got[0].items():
        assert torch.equal(v[:used] if n == "dx" else v, got[1][n][:used] if n == "dx" else got[1][n]), n
    hs, at = half_step(dt), 0
    mid = (hs if dtype == "bf16" else 0.0) + 2.0 ** -20        # the middle's own rounding and its exponentials
    for e, n in enumerate(counts):
        part = slice(at, at + n)
        at += n
        d = dy[part].double()
        grads, offs = [d], [torch.zeros_like(d)]
        if glu:
            a, b = pre[part].double(), pre_up[part].double()
            sig = 1 / (1 + torch.exp(-a))
            grads = [d * b * sig * (1 + a * (1 - sig)), d * activation("silu", a)]
            # terms up to |dy| (1 + |a|) |up|, which may cancel
            offs = [mid * v.abs() + 2.0 ** -20 * m for v, m in zip(grads, (d.abs() * (1 + a.abs()) * b.abs(), d.abs() * (1 + a.abs())))]
        if product != F.WEIGHT:
            want, err = torch.zeros(n, K, dtype=torch.float64), torch.zeros(n, K, dtype=torch.float64)
            for v, o, w in zip(grads, offs, (s["w"], s["w_up"])):
                want += v @ w[e].double()
                err += (o + len(grads) * (N + 4) * U32 * v.abs()) @ w[e].double().abs()
            assert_within(got[0]["dx"][part], want, hs * want.abs() + (1 + hs) * err, ("dx", e))
        if product != F.INPUT:
            x = s["x"][part].double()
            for v, o, name in zip(grads, offs, ("dw", "dw_up")):
                want = v.t().contiguous() @ x
                assert_within(got[0][name][e], want, hs * want.abs() + (1 + hs) * ((o + (n + 4) * U32 * v.abs()).t() @ x.abs()), (name, e))

"""The experts' products on sorted rows (etr_expert_linear and its backward) against their definitions in 64 bits."""
import pytest
import torch

from operator_refs import DT, U32, activation, assert_within, half_step, randn
from paper_2406_00023_amd import binding as B

pytestmark = pytest.mark.gpu
ACT = {"none": B.ACT_NONE, "silu": B.ACT_SILU, "gelu": B.ACT_GELU, "swiglu": B.ACT_SWIGLU}


def _offsets(counts):
    return torch.tensor([0] + list(torch.tensor(counts).cumsum(0)), dtype=torch.int32)


# (rows of each expert, rows that belong to nobody, K, N): single rows and empty experts; few rows on ragged widths and on whole tiles;
# short tiles; one dense product; a contraction of one piece; rows for the large tiles of either type, ragged by a row or a piece
CASES = [((1,), 0, 8, 8), ((1, 0, 3), 2, 136, 72), ((0, 0), 5, 64, 64), ((5, 33, 0, 17), 0, 520, 264), ((32, 32), 0, 256, 256), ((100, 1, 65), 9, 136, 200),
         ((70, 0, 129, 64), 3, 512, 384), ((300,), 0, 1032, 264), ((257, 0, 511, 1, 256, 300, 270, 520), 4, 200, 2056),
         ((2049, 300), 1, 72, 3592)]


def _inputs(counts, spare, K, N, dt, act, bias, residual, seed=1):
    E, R = len(counts), sum(counts) + spare
    glu = act == "swiglu"
    s = dict(x=randn(seed, R, K, dtype=dt), w=randn(seed + 1, E, N, K, dtype=dt, std=K ** -0.5), w_up=None, bias=None, bias_up=None, residual=None)
    if glu:
        s["w_up"] = randn(seed + 2, E, N, K, dtype=dt, std=K ** -0.5)
    if bias:
        s["bias"] = randn(seed + 3, E, N, std=0.3)
        s["bias_up"] = randn(seed + 4, E, N, std=0.3) if glu else None
    if residual:
        s["residual"] = randn(seed + 5, R, N, dtype=dt)
    s["x"][sum(counts):] = float("nan")                        # rows that belong to nobody are never read
    return s


def _cuda(s):
    return {n: None if v is None else v.cuda() for n, v in s.items()}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act,bias,residual,keep", [("none", False, False, False), ("none", True, True, True), ("silu", True, False, True),
                                                    ("gelu", False, True, False), ("swiglu", False, False, False), ("swiglu", True, True, True)])
@pytest.mark.parametrize("counts,spare,K,N", CASES)
def test_forward(counts, spare, K, N, act, bias, residual, keep, dtype):
    dt = DT[dtype]
    print(f"linear forward {counts} spare {spare} K {K} N {N} {act} {dtype}", flush=True)
    E, used = len(counts), sum(counts)
    R = used + spare
    s = _inputs(counts, spare, K, N, dt, act, bias, residual)
    g = _cuda(s)
    cfg = B.make_linear_config(R, K, N, E, dt, act=ACT[act])
    new = lambda: torch.full((R, N), 7.0, dtype=dt, device="cuda")
    y, pre, pre_up = new(), new() if keep else None, new() if keep and act == "swiglu" else None
    B.etr_expert_linear(cfg, g["x"], _offsets(counts).cuda(), g["w"], y, w_up=g["w_up"], bias=g["bias"], bias_up=g["bias_up"],
                        residual=g["residual"], pre=pre, pre_up=pre_up)
    torch.cuda.synchronize()
    assert bool((y[used:] == 7.0).all())
    hs, at = half_step(dt), 0
    for e, n in enumerate(counts):
        rows = slice(at, at + n)
        at += n
        if n == 0:
            continue
        x = s["x"][rows].double()
        a = x @ s["w"][e].double().t()
        mag = x.abs() @ s["w"][e].double().abs().t()
        b = ub = None
        if bias:
            a, mag = a + s["bias"][e].double(), mag + s["bias"][e].double().abs()
        ea = (K + 4) * U32 * mag                                # fp32 sum of K products and a bias
        if act == "swiglu":
            b = x @ s["w_up"][e].double().t()
            ub = x.abs() @ s["w_up"][e].double().abs().t()
            if bias:
                b, ub = b + s["bias_up"][e].double(), ub + s["bias_up"][e].double().abs()
            ub = (K + 4) * U32 * ub
        if keep:
            assert_within(pre[rows], a, hs * a.abs() + ea, "pre")
            if b is not None:
                assert_within(pre_up[rows], b, hs * b.abs() + ub, "pre_up")
        want = activation(act, a, b)
        # |act'| <= 1.13; exponential, reciprocal and the fit of the distribution function: 2^-20 of the larger of value and argument
        err = 1.13 * ea * (1 if b is None else b.abs()) + (0 if b is None else (a.abs() + 1) * ub) + (0 if act == "none" else 2.0 ** -20 * (want.abs() + a.abs() * (1 if b is None else b.abs())))
        if residual:
            r = s["residual"][rows].double()
            want, err = want + r, err + U32 * (want.abs() + r.abs())
        assert_within(y[rows], want, hs * want.abs() + (1 + hs) * err, "y")


# few rows against a long contraction, which many waves share: k-tiles that do not divide by their number, a last row tile of one row,
# column tiles of a piece
LONG = [((1,), 0, 1544, 72), ((17,), 3, 4104, 200), ((3, 0, 16, 33), 1, 1096, 152), ((130,), 0, 2048, 40), ((0, 1), 0, 8192, 8)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act,bias,residual,keep", [("none", False, False, False), ("silu", True, True, True), ("gelu", False, True, False),
                                                    ("swiglu", True, True, True)])
@pytest.mark.parametrize("counts,spare,K,N", LONG)
def test_forward_of_few_rows(counts, spare, K, N, act, bias, residual, keep, dtype):
    test_forward(counts, spare, K, N, act, bias, residual, keep, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "silu", "gelu", "swiglu"])
@pytest.mark.parametrize("counts,spare,K,N", CASES)
def test_backward(counts, spare, K, N, act, dtype):
    dt = DT[dtype]
    print(f"linear backward {counts} spare {spare} K {K} N {N} {act} {dtype}", flush=True)
    E, used, glu = len(counts), sum(counts), act == "swiglu"
    R = used + spare
    s = _inputs(counts, spare, K, N, dt, act, False, False, seed=11)
    pre, pre_up = (randn(i, R, N, dtype=dt) for i in (31, 32))
    dy = randn(33, R, N, dtype=dt)
    for v in (pre, pre_up, dy):
        v[used:] = float("nan")
    g = _cuda(s)
    cfg = B.make_linear_config(R, K, N, E, dt, act=ACT[act])
    new = lambda *n, t=dt: torch.full(n, 7.0, dtype=t, device="cuda")
    dx, dw, dw_up, dbias, dbias_up = new(R, K), new(E, N, K), new(E, N, K), new(E, N, t=torch.float32), new(E, N, t=torch.float32)
    ws = torch.full((B.etr_linear_workspace_bytes(cfg),), 255, dtype=torch.uint8, device="cuda")
    B.etr_expert_linear_backward(cfg, g["x"], _offsets(counts).cuda(), g["w"], dy.cuda(), ws, w_up=g["w_up"], pre=None if act == "none" else pre.cuda(),
                                 pre_up=pre_up.cuda() if glu else None, dx=dx, dw=dw, dw_up=dw_up if glu else None, dbias=dbias,
                                 dbias_up=dbias_up if glu else None)
    torch.cuda.synchronize()
    assert bool((dx[used:] == 7.0).all())
    hs, at = half_step(dt), 0
    mid = 0.0 if act == "none" else (hs if dtype == "bf16" else 0.0) + 2.0 ** -20      # the middle's own rounding and its exponentials
    for e, n in enumerate(counts):
        rows = slice(at, at + n)
        at += n
        x, d = s["x"][rows].double(), dy[rows].double()
        leaf = [pre[rows].double().requires_grad_(True)] + ([pre_up[rows].double().requires_grad_(True)] if glu else [])
        grads = [d] if act == "none" else list(torch.autograd.grad(activation(act, *leaf), leaf, d)) if n else [torch.zeros(0, N, dtype=torch.float64)] * len(leaf)
        # a derivative is made of terms up to |dy| (1 + |a|) (|up|), which may cancel
        terms = [d.abs() * (1 + leaf[0].detach().abs()) * (leaf[1].detach().abs() if glu else 1)] + ([d.abs() * (1 + leaf[0].detach().abs())] if glu else [])
        off = [mid * g_.abs() + (0.0 if act == "none" else 2.0 ** -20) * m for g_, m in zip(grads, terms)]
        dx_want, dx_err = torch.zeros(n, K, dtype=torch.float64), torch.zeros(n, K, dtype=torch.float64)
        for i, (grad, o, w, got_w, got_b) in enumerate(zip(grads, off, (s["w"], s["w_up"]), (dw, dw_up), (dbias, dbias_up))):
            wt = w[e].double()
            dx_want += grad @ wt
            dx_err += (o + len(grads) * (N + 4) * U32 * grad.abs()) @ wt.abs()
            want = grad.t().contiguous() @ x
            assert_within(got_w[e], want, hs * want.abs() + (1 + hs) * ((o + (n + 4) * U32 * grad.abs()).t() @ x.abs()), ("dw", i, e))
            exact_off = (o - (hs * grad.abs() if dtype == "bf16" and act != "none" else 0)).clamp_min(0)   # summed before the rounding
            assert_within(got_b[e], grad.sum(0), (exact_off + (n + 4) * U32 * grad.abs()).sum(0), ("dbias", i, e))
        assert_within(dx[rows], dx_want, hs * dx_want.abs() + (1 + hs) * dx_err, ("dx", e))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "gelu", "swiglu"])
@pytest.mark.parametrize("counts,spare,N,K", LONG)
def test_backward_of_few_rows(counts, spare, K, N, act, dtype):
    test_backward(counts, spare, K, N, act, dtype)


def test_dense_without_offsets_and_in_place_residual():
    R, K, N = 300, 264, 136
    s = _inputs((R,), 0, K, N, torch.bfloat16, "gelu", True, True)
    g = _cuda(s)
    cfg = B.make_linear_config(R, K, N, 1, torch.bfloat16, act=B.ACT_GELU)
    a, b = torch.empty(R, N, dtype=torch.bfloat16, device="cuda"), g["residual"].clone()
    B.etr_expert_linear(cfg, g["x"], _offsets((R,)).cuda(), g["w"], a, bias=g["bias"], residual=g["residual"])
    B.etr_expert_linear(cfg, g["x"], None, g["w"], b, bias=g["bias"], residual=b)
    torch.cuda.synchronize()
    assert torch.equal(a, b)


def test_parts_of_the_backward_alone():
    """Each output by itself is what it is beside the others."""
    counts, K, N = (40, 0, 90), 136, 200
    s = _cuda(_inputs(counts, 0, K, N, torch.bfloat16, "silu", False, False, seed=3))
    R, E = sum(counts), len(counts)
    cfg = B.make_linear_config(R, K, N, E, torch.bfloat16, act=B.ACT_SILU)
    pre, dy, off = randn(5, R, N, dtype=torch.bfloat16).cuda(), randn(6, R, N, dtype=torch.bfloat16).cuda(), _offsets(counts).cuda()
    ws = B.alloc_workspace(B.etr_linear_workspace_bytes(cfg))
    out = lambda: dict(dx=torch.empty(R, K, dtype=torch.bfloat16, device="cuda"), dw=torch.empty(E, N, K, dtype=torch.bfloat16, device="cuda"),
                       dbias=torch.empty(E, N, device="cuda"))
    full = out()
    B.etr_expert_linear_backward(cfg, s["x"], off, s["w"], dy, ws, pre=pre, **full)
    for n, v in out().items():
        B.etr_expert_linear_backward(cfg, s["x"] if n == "dw" else None, off, s["w"] if n == "dx" else None, dy, ws, pre=pre, **{n: v})
        torch.cuda.synchronize()
        assert torch.equal(v, full[n]), n


def test_offsets_past_the_rows_are_clamped():
    R, K, N = 40, 64, 64
    s = _cuda(_inputs((R,), 0, K, N, torch.float32, "none", False, False))
    w = torch.cat([s["w"], s["w"] * 2, s["w"] * 3])
    cfg = B.make_linear_config(R, K, N, 3, torch.float32)
    y, z = (torch.full((R, N), 7.0, device="cuda") for _ in range(2))
    B.etr_expert_linear(cfg, s["x"], torch.tensor([0, 10, 1000, 900], dtype=torch.int32, device="cuda"), w, y)
    B.etr_expert_linear(cfg, s["x"], torch.tensor([0, 10, R, R], dtype=torch.int32, device="cuda"), w, z)
    torch.cuda.synchronize()
    assert torch.equal(y, z)


def test_gradients_against_differences():
    counts, K, N = (5, 0, 7), 72, 40
    for act in ACT:
        glu = act == "swiglu"
        s = _inputs(counts, 0, K, N, torch.float32, act, True, False, seed=41)
        R, E = sum(counts), len(counts)
        g, off = _cuda(s), _offsets(counts)
        cfg = B.make_linear_config(R, K, N, E, torch.float32, act=ACT[act])
        up = randn(51, R, N)
        y, pre, pre_up = (torch.empty(R, N, device="cuda") for _ in range(3))
        B.etr_expert_linear(cfg, g["x"], off.cuda(), g["w"], y, w_up=g["w_up"], bias=g["bias"], bias_up=g["bias_up"], pre=pre, pre_up=pre_up if glu else None)
        out = dict(x=torch.empty(R, K, device="cuda"), w=torch.empty(E, N, K, device="cuda"), bias=torch.empty(E, N, device="cuda"))
        if glu:
            out.update(w_up=torch.empty(E, N, K, device="cuda"), bias_up=torch.empty(E, N, device="cuda"))
        B.etr_expert_linear_backward(cfg, g["x"], off.cuda(), g["w"], up.cuda(), B.alloc_workspace(B.etr_linear_workspace_bytes(cfg)), w_up=g["w_up"],
                                     pre=pre, pre_up=pre_up if glu else None, dx=out["x"], dw=out["w"], dw_up=out.get("w_up"), dbias=out["bias"],
                                     dbias_up=out.get("bias_up"))
        torch.cuda.synchronize()

        def loss(q):
            total = 0.0
            for e in range(E):
                r = slice(int(off[e]), int(off[e + 1]))
                a = q["x"][r] @ q["w"][e].t() + q["bias"][e]
                b = q["x"][r] @ q["w_up"][e].t() + q["bias_up"][e] if glu else None
                total += float((activation(act, a, b) * up[r].double()).sum())
            return total

        at = {n: s[n].double() for n in ("x", "w", "bias", "w_up", "bias_up") if s[n] is not None}
        for n, grad in out.items():
            v, step = randn(60, *at[n].shape).double(), 1e-5
            diff = (loss({**at, n: at[n] + step * v}) - loss({**at, n: at[n] - step * v})) / (2 * step)
            prod = grad.cpu().double() * v
            assert abs(float(prod.sum()) - diff) <= 2e-5 * float(prod.abs().sum()) + 1e-5 * max(1.0, abs(diff)), (act, n)

"""The join of a block with the residual stream and the norm in front of the next one (etr_block_norm and its backward)
against their definitions in 64 bits."""
import pytest
import torch

from operator_refs import DT, U32, assert_within, half_step, join, randn, rms
from paper_2406_00023_amd import binding as B

pytestmark = pytest.mark.gpu
EPS, RS, BS = 1e-5, 0.9, 0.6
# roundings of a row's sum of squares (up to 64 terms one after the other in a thread, then a tree) and of what is made of it
SUM, ROW = 80 * U32, 120 * U32


def _inputs(T, d, dt, block, gate, post, pre, seed=1):
    s = dict(x=randn(seed, T, d, dtype=dt, std=2.0), y=None, gate=None, w_post=None, w_pre=None)
    if block:
        s["y"] = randn(seed + 1, T, d, dtype=dt, std=0.7)
        s["gate"] = torch.sigmoid(randn(seed + 2, T)) if gate else None
        s["w_post"] = 1 + randn(seed + 3, d, std=0.1) if post else None
    if pre:
        s["w_pre"] = 1 + randn(seed + 4, d, std=0.1)
    return s


def _cuda(s):
    return {n: None if v is None else v.cuda() for n, v in s.items()}


def _d(v):
    return None if v is None else v.double()


SHAPES = [(1, 8), (3, 520), (5, 512), (2, 2048), (2500, 1080), (3, 8192), (2, 16384)]
PARTS = [(True, True, True, True), (True, False, False, True), (True, True, False, False), (True, False, True, False), (False, False, False, True)]


@pytest.mark.parametrize("parts", PARTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,d", SHAPES)
def test_forward(T, d, dtype, parts):
    block, gate, post, pre = parts
    dt = DT[dtype]
    s = _inputs(T, d, dt, block, gate, post, pre)
    g = _cuda(s)
    cfg = B.make_norm_config(T, d, dt, eps=EPS, residual_scale=RS, block_scale=BS)
    x_out = torch.full((T, d), 7.0, dtype=dt, device="cuda") if block else None
    h = torch.full((T, d), 7.0, dtype=dt, device="cuda") if pre else None
    B.etr_block_norm(cfg, g["x"], g["y"], g["gate"], g["w_post"], g["w_pre"], x_out, h)
    torch.cuda.synchronize()
    stream = s["x"]
    if block:
        want = join(*(_d(s[n]) for n in ("x", "y", "gate", "w_post")), EPS, RS, BS)
        parts_abs = (RS * s["x"].double()).abs() + (want - RS * s["x"].double()).abs()
        assert_within(x_out, want, half_step(dt) * want.abs() + ROW * parts_abs, "x_out")
        stream = x_out.cpu()
    if pre:                                            # from the stream as it was stored
        want = rms(stream.double(), EPS) * s["w_pre"].double()
        assert_within(h, want, (half_step(dt) + ROW) * want.abs() + 1e-38, "h")


@pytest.mark.parametrize("parts", PARTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,d", SHAPES + [(5000, 264)])
def test_backward(T, d, dtype, parts):
    block, gate, post, pre = parts
    dt = DT[dtype]
    s = _inputs(T, d, dt, block, gate, post, pre, seed=11)
    stream, dxo, dh = randn(21, T, d, dtype=dt, std=2.0), randn(22, T, d, dtype=dt), randn(23, T, d, dtype=dt)
    if T == 3:
        dxo = None                                     # nothing comes along the stream
        if not pre:
            pytest.skip("no gradient at all")
    g = _cuda(s)
    cfg = B.make_norm_config(T, d, dt, eps=EPS, residual_scale=RS, block_scale=BS)
    new = lambda *n, t=torch.float32: torch.full(n, 7.0, dtype=t, device="cuda")
    dx, dy = new(T, d, t=dt), new(T, d, t=dt) if block else None
    dgate, dwp, dwn = new(T) if gate else None, new(d) if post else None, new(d) if pre else None
    ws = B.alloc_workspace(B.etr_norm_workspace_bytes(cfg))
    B.etr_block_norm_backward(cfg, stream.cuda() if pre else None, g["y"], g["gate"], g["w_post"], g["w_pre"],
                              None if dxo is None else dxo.cuda(), dh.cuda() if pre else None, dx, dy, dgate, dwp, dwn, ws)
    torch.cuda.synchronize()
    hs = half_step(dt)
    # r, and the sum of the magnitudes it is made of
    r = torch.zeros(T, d, dtype=torch.float64) if dxo is None else dxo.double()
    mag = r.abs()
    if pre:
        v, u = stream.double(), dh.double() * s["w_pre"].double()
        inv = 1 / (v.square().mean(1, keepdim=True) + EPS).sqrt()
        r = r + inv * (u - v * inv ** 2 * (u * v).mean(1, keepdim=True))
        mag = mag + inv * (u.abs() + v.abs() * inv ** 2 * (u * v).abs().mean(1, keepdim=True))
        terms = dh.double() * v * inv
        assert_within(dwn, terms.sum(0), (SUM + ROW + 40 * U32) * terms.abs().sum(0), "dw_pre")
    scale = RS if block else 1.0
    assert_within(dx, scale * r, hs * scale * r.abs() + ROW * mag, "dx")
    if not block:
        return
    y = s["y"].double()
    inv = 1 / (y.square().mean(1, keepdim=True) + EPS).sqrt() if post else torch.ones(T, 1, dtype=torch.float64)
    wp = s["w_post"].double() if post else torch.ones(d, dtype=torch.float64)
    w = BS * (s["gate"].double()[:, None] if gate else 1.0) * torch.ones(T, 1, dtype=torch.float64)
    p, u = y * inv * wp, w * r * wp
    mag_u = w * mag * wp.abs()
    if gate:
        assert_within(dgate, BS * (r * p).sum(1), 3 * ROW * BS * (mag * p.abs()).sum(1), "dgate")
    if post:
        assert_within(dwp, (w * r * y * inv).sum(0), (SUM + 2 * ROW + 40 * U32) * (w * mag * (y * inv).abs()).sum(0), "dw_post")
        dy_want = inv * (u - y * inv ** 2 * (u * y).mean(1, keepdim=True))
        mag_y = inv * (mag_u + y.abs() * inv ** 2 * (mag_u * y.abs()).mean(1, keepdim=True))
    else:
        dy_want, mag_y = u, mag_u
    assert_within(dy, dy_want, hs * dy_want.abs() + 3 * ROW * mag_y, "dy")


def test_gradients_against_differences():
    """<gradient, direction> against the central difference of the 64-bit loss along that direction, for every input."""
    T, d = 6, 264
    s = _inputs(T, d, torch.float32, True, True, True, True, seed=31)
    up, uh = randn(41, T, d), randn(42, T, d)
    cfg = B.make_norm_config(T, d, torch.float32, eps=EPS, residual_scale=RS, block_scale=BS)
    g = _cuda(s)
    x_out, h = torch.empty(T, d, device="cuda"), torch.empty(T, d, device="cuda")
    B.etr_block_norm(cfg, g["x"], g["y"], g["gate"], g["w_post"], g["w_pre"], x_out, h)
    out = dict(x=torch.empty(T, d), y=torch.empty(T, d), gate=torch.empty(T), w_post=torch.empty(d), w_pre=torch.empty(d))
    out = _cuda(out)
    B.etr_block_norm_backward(cfg, x_out, g["y"], g["gate"], g["w_post"], g["w_pre"], up.cuda(), uh.cuda(), out["x"], out["y"],
                              out["gate"], out["w_post"], out["w_pre"], B.alloc_workspace(B.etr_norm_workspace_bytes(cfg)))
    torch.cuda.synchronize()

    def loss(q):
        xo = join(q["x"], q["y"], q["gate"], q["w_post"], EPS, RS, BS)
        return float((xo * up.double()).sum() + (rms(xo, EPS) * q["w_pre"] * uh.double()).sum())

    at = {n: v.double() for n, v in s.items()}
    for n in out:
        v = randn(50, *at[n].shape).double()
        step = 1e-5
        diff = (loss({**at, n: at[n] + step * v}) - loss({**at, n: at[n] - step * v})) / (2 * step)
        got = float((out[n].cpu().double() * v).sum())
        # fp32 gradients (2e-5 of the magnitudes that are added) and the difference's own error (step^2 and 2^-53 loss / step)
        size = float((out[n].cpu().double() * v).abs().sum())
        assert abs(got - diff) <= 2e-5 * size + 1e-5 * max(1.0, abs(diff)), n


def test_in_place_zero_rows_and_non_finite_rows():
    T, d = 9, 1032
    s = _inputs(T, d, torch.bfloat16, True, True, True, True, seed=61)
    s["x"][2] = 0
    s["y"][2] = 0                                       # nothing to norm: 0 / sqrt(eps)
    s["y"][5, 7] = float("inf")
    s["x"][6, 3] = float("nan")
    g = _cuda(s)
    cfg = B.make_norm_config(T, d, torch.bfloat16, eps=EPS)
    a, ha, hb = (torch.empty(T, d, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    B.etr_block_norm(cfg, g["x"], g["y"], g["gate"], g["w_post"], g["w_pre"], a, ha)
    b = g["x"].clone()
    B.etr_block_norm(cfg, b, g["y"], g["gate"], g["w_post"], g["w_pre"], b, hb)        # x_out is x
    torch.cuda.synchronize()
    ok = torch.tensor([t for t in range(T) if t not in (5, 6)], device="cuda")
    assert torch.equal(a[ok], b[ok]) and torch.equal(ha[ok], hb[ok])
    assert bool((a[2] == 0).all()) and bool((ha[2] == 0).all())
    assert bool(torch.isfinite(a[ok]).all()) and bool(torch.isfinite(ha[ok]).all())    # the rows beside them are theirs alone
    assert bool(torch.isnan(a[6, 3])) and bool(torch.isnan(ha[6]).any())


def test_same_results_twice_and_from_an_unused_workspace():
    T, d = 4099, 520
    s = _cuda(_inputs(T, d, torch.float32, True, True, True, True, seed=71))
    up, uh = randn(72, T, d).cuda(), randn(73, T, d).cuda()
    cfg = B.make_norm_config(T, d, torch.float32, eps=EPS)
    n = B.etr_norm_workspace_bytes(cfg)
    got = []
    for fill in (0, 255):
        ws = torch.full((n,), fill, dtype=torch.uint8, device="cuda")
        o = [torch.empty(T, d, device="cuda") for _ in range(2)] + [torch.empty(T, device="cuda")] + [torch.empty(d, device="cuda") for _ in range(2)]
        B.etr_block_norm_backward(cfg, s["x"], s["y"], s["gate"], s["w_post"], s["w_pre"], up, uh, *o, ws)
        torch.cuda.synchronize()
        got.append(o)
    assert all(torch.equal(a, b) for a, b in zip(*got))

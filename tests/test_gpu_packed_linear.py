"""Products of packed operands against the definition in 64 bits, on the values that the operands stand for.

Bounds.  fp32 results: a sum of n terms in 32 bits is off by n half steps of the sum of the terms' magnitudes at most; the activations
by 40 half steps (four operations behind an exponential and a reciprocal, each a few), and a result by a half step.  bf16 results: half a step of bf16
for the result, and what the matrix pipe cuts off: 2^-13 of the largest product of a group of 16, for each product (one in sixteen times the sum over the groups is what
a group's 16 products can lose).  Packed results: half a step of e4m3 (2^-4), half of its smallest step (2^-10) of the block's power, and the
error of what was packed."""
import pytest
import torch

import operator_refs as O
import packed_refs as R
from paper_2406_00023_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTS = {"none": 0, "silu": 1, "gelu": 2, "swiglu": 3}
SLOPE = 1.2                                                    # |act'| of SiLU and GELU is 1.13 at most


def operand(seed, *shape, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return R.pack((torch.randn(*shape, generator=g) * std).double())


def gpu(packed):
    return tuple(t.cuda() for t in packed)


def sum_error(x, w, wide):
    """Bound of a product's error: [rows][N]."""
    K = x.shape[1]
    magnitude = x.abs() @ w.abs().t()
    if wide:
        return (K + 2) * O.U32 * magnitude
    pad = -K % 16
    p = torch.nn.functional.pad(x, (0, pad)).abs().unflatten(1, (-1, 16)).amax(2) @ torch.nn.functional.pad(w, (0, pad)).abs().unflatten(1, (-1, 16)).amax(2).t()
    return 16 * 2.0 ** -13 * p + (K + 2) * O.U32 * magnitude


def check_packed(q, s, want, err, what):
    """What is packed is within a half step of what should be, and its powers are the right ones for values that far off."""
    rows, N = want.shape
    power = R.unlayout(s, R.blocks(N))
    got = R.values(q, s, N)
    unit = torch.exp2(power.double() - 127).repeat_interleave(128, 1)[:, :N]
    O.assert_within(got, want, 2.0 ** -4 * (want.abs() + err) + 2.0 ** -10 * unit + err, what)
    pad = R.blocks(N) * 128 - N
    top = torch.nn.functional.pad(want.abs(), (0, pad)).unflatten(1, (-1, 128)).amax(2)
    slack = torch.nn.functional.pad(err, (0, pad)).unflatten(1, (-1, 128)).amax(2)
    unit = torch.exp2(power.double() - 127)
    assert bool((top - slack <= 448 * unit).all()) and bool(((top + slack > 224 * unit) | (power == 0)).all()), what
    if pad:
        assert not q[:, N:].any(), what
    if R.blocks(N) % 4:
        assert bool((s[-1, :, R.blocks(N) % 4:] == 127).all()), what


def case(counts, K, N, dtype, act, bias=False, residual=False, keep=False, y=True, extra=2, seed=0):
    E, used = len(counts), sum(counts)
    rows = used + extra
    offsets = [sum(counts[:e]) for e in range(E + 1)]
    glu, wide = act == "swiglu", dtype == "f32"
    x8, w8 = operand(seed + 1, rows, K), operand(seed + 2, E, N, K, std=K ** -0.5)
    up8 = operand(seed + 3, E, N, K, std=K ** -0.5) if glu else None
    b = O.randn(seed + 4, E, N, std=0.3) if bias else None
    bu = O.randn(seed + 5, E, N, std=0.3) if bias and glu else None
    res = O.randn(seed + 6, rows, N, dtype=DT[dtype]) if residual else None
    cfg = B.make_linear_config(rows, K, N, E, DT[dtype], act=ACTS[act])
    out_cfg = B.make_pack_config(rows, N, DT[dtype])

    def buffers():
        return (torch.full((rows, R.blocks(N) * 128), 0xA5, dtype=torch.uint8, device="cuda"),
                torch.full((R.blocks(R.blocks(N) * 32), rows, 4), 0xA5, dtype=torch.uint8, device="cuda"))

    out = torch.full((rows, N), 7.0, dtype=DT[dtype], device="cuda") if y else None
    y8 = buffers() if keep else None
    assert y8 is None or (y8[0].numel() == B.etr_packed_rows_bytes(out_cfg) and y8[1].numel() == B.etr_packed_rows_scale_bytes(out_cfg))
    pre8 = buffers() if keep else None
    pre_up8 = buffers() if keep and glu else None
    cuda = lambda t: None if t is None else t.cuda()
    B.etr_packed_linear(cfg, gpu(x8), torch.tensor(offsets, dtype=torch.int32, device="cuda"), gpu(w8), y=out, w_up8=gpu(up8) if glu else None, bias=cuda(b),
                        bias_up=cuda(bu), residual=cuda(res), y8=y8, pre8=pre8, pre_up8=pre_up8)
    torch.cuda.synchronize()
    xv, wv = R.values(*x8, K), R.values(*w8, K)
    uv = R.values(*up8, K) if glu else None
    a, ea, u, eu = (torch.zeros(rows, N, dtype=torch.float64) for _ in range(4))
    for e in range(E):
        sl = slice(offsets[e], offsets[e + 1])
        a[sl], ea[sl] = xv[sl] @ wv[e].t(), sum_error(xv[sl], wv[e], wide)
        if glu:
            u[sl], eu[sl] = xv[sl] @ uv[e].t(), sum_error(xv[sl], uv[e], wide)
        if bias:
            a[sl] += b[e].double()
            ea[sl] += 2 * O.U32 * a[sl].abs()
            if glu:
                u[sl] += bu[e].double()
                eu[sl] += 2 * O.U32 * u[sl].abs()
    want = O.activation(act, a, u if glu else None)
    if glu:
        err = SLOPE * ea * (u.abs() + eu) + (a.abs() + ea) * eu + 40 * O.U32 * want.abs()
    else:
        err = ea if act == "none" else SLOPE * ea + 40 * O.U32 * want.abs()
    # (bf16: the activations' exponential without its lower part: 208 half steps of fp32 at most)
    if not wide:
        err = err + 256 * O.U32 * want.abs()
    if residual:
        want = want + res.double()
        err = err + 2 * O.U32 * want.abs()
    live = slice(0, used)
    what = (counts, K, N, dtype, act)
    if y:
        O.assert_within(out[live], want[live], err[live] + O.half_step(DT[dtype]) * (want[live].abs() + err[live]), what)
        if used and not wide:                                  # (what is cut off is far below that bound: 2^-14 of the result's size)
            off = (out[live].cpu().double() - want[live])
            assert float(off.norm()) <= (O.half_step(DT[dtype]) + 2.0 ** -12) * float(want[live].norm()), what
        assert bool((out[used:] == 7.0).all()), what
    for buf, w, er in ((y8, want, err), (pre8, a, ea), (pre_up8, u, eu)):
        if buf is not None:
            q, s = buf[0].cpu(), buf[1].cpu()
            check_packed(q[live], s[:, live], w[live], er[live], what)
            assert bool((q[used:] == 0xA5).all()) and bool((s[:, used:] == 0xA5).all()), what


# counts: few rows, a tile in part, several tiles, experts without rows and with one
FEW, MIDDLE, MANY = [3, 0, 1, 16, 17], [130, 1, 64, 40], [700, 513]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts", [[1], FEW, MIDDLE, MANY], ids=["one", "few", "middle", "many"])
@pytest.mark.parametrize("K,N", [(8, 8), (128, 128), (136, 24), (520, 264), (1000, 520), (2056, 136)])
def test_product(counts, K, N, dtype):
    case(counts, K, N, dtype, "none", seed=K + N)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts", [FEW, MIDDLE, MANY], ids=["few", "middle", "many"])
@pytest.mark.parametrize("act", ["silu", "gelu", "swiglu", "none"])
@pytest.mark.parametrize("K,N", [(264, 136), (648, 520)])
def test_everything_in_the_epilogue(counts, K, N, act, dtype):
    case(counts, K, N, dtype, act, bias=True, residual=True, keep=True, seed=K)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["none", "swiglu"])
@pytest.mark.parametrize("counts", [FEW, MIDDLE, MANY], ids=["few", "middle", "many"])
def test_packed_results_alone(counts, act, dtype):
    case(counts, 384, 640, dtype, act, keep=True, y=False, extra=0)


def test_no_rows_at_all():
    case([0, 0, 0], 136, 136, "bf16", "swiglu", keep=True, extra=5)


@pytest.mark.parametrize("counts", [[40], [900]])
def test_dense(counts):
    """One expert, no table."""
    rows, K, N = counts[0], 264, 392
    x8, w8 = operand(1, rows, K), operand(2, 1, N, K, std=K ** -0.5)
    y = torch.zeros(rows, N, device="cuda")
    B.etr_packed_linear(B.make_linear_config(rows, K, N, 1, torch.float32), gpu(x8), None, gpu(w8), y=y)
    xv, wv = R.values(*x8, K), R.values(*w8, K)[0]
    O.assert_within(y, xv @ wv.t(), sum_error(xv, wv, True) + O.U32 * (xv @ wv.t()).abs(), counts)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [5, 100, 1100])
def test_powers_far_apart_and_no_numbers(rows, dtype):
    """Blocks whose powers lie far apart; a NaN is in the results of its row, or of its column, and nowhere else."""
    K, N = 520, 136
    g = torch.Generator().manual_seed(rows)
    x = torch.randn(rows, K, generator=g).double() * torch.exp2(torch.randint(-30, 30, (rows, 5), generator=g).double()).repeat_interleave(128, 1)[:, :K]
    w = torch.randn(1, N, K, generator=g).double() * torch.exp2(torch.randint(-30, 30, (1, N, 5), generator=g).double()).repeat_interleave(128, 2)[:, :, :K]
    x[1, 7] = float("nan")
    w[0, 9, 500] = float("inf")
    x8, w8 = R.pack(x), R.pack(w)
    y = torch.zeros(rows, N, dtype=DT[dtype], device="cuda")
    B.etr_packed_linear(B.make_linear_config(rows, K, N, 1, DT[dtype]), gpu(x8), None, gpu(w8), y=y)
    y = y.cpu()
    bad = torch.zeros(rows, N, dtype=torch.bool)
    bad[1], bad[:, 9] = True, True
    assert torch.equal(torch.isnan(y), bad)
    xv, wv = R.values(*x8, K).nan_to_num(nan=0.0), R.values(*w8, K)[0].nan_to_num(nan=0.0)
    want = xv @ wv.t()
    err = sum_error(xv, wv, dtype == "f32") + O.half_step(DT[dtype]) * want.abs()
    off = (y.double() - want).abs() - 1.01 * err
    assert bool((off[~bad] <= 0).all())

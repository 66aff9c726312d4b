"""Packed operators at the limits that the header names: 64 experts, what is no number inside packed results and gradients, operands and results of the
gradients past 4 GiB, offsets inside a tile past 2^31."""
import pytest
import torch

import operator_refs as O
import packed_forms as F
import packed_refs as R
from paper_2406_00023_amd import binding as B
from test_gpu_packed_backward import act_case, derivative, weights_case
from test_gpu_packed_linear import ACTS, DT, SLOPE, case, check_packed, gpu, operand, sum_error

pytestmark = pytest.mark.gpu

# 64 experts, one to a lane of the kernels' tables: the first and the last without rows, only the last with rows, one row each, many rows
EXPERTS = {"ends_empty": [0] + [(7 * e) % 23 for e in range(62)] + [0], "last_alone": [0] * 63 + [300], "one_each": [1] * 64,
           "many": [(131 * e) % 260 for e in range(64)]}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act,keep", [("none", False), ("swiglu", False), ("gelu", True), ("swiglu", True)])
@pytest.mark.parametrize("counts", EXPERTS.values(), ids=EXPERTS)
def test_products_of_64_experts(counts, act, keep, dtype):
    case(counts, 136, 264, dtype, act, bias=True, keep=keep, seed=3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["none", "swiglu"])
@pytest.mark.parametrize("counts", EXPERTS.values(), ids=EXPERTS)
def test_element_wise_part_of_64_experts(counts, act, dtype):
    act_case(counts, 264, dtype, act, seed=4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("glu", [False, True])
@pytest.mark.parametrize("counts", EXPERTS.values(), ids=EXPERTS)
def test_weights_gradient_of_64_experts(counts, glu, dtype):
    weights_case(counts, 136, 264, glu, dtype)


# ---- no numbers

def _no_numbers(q, s, bad, want, err, what):
    """Packed NaN where `bad`; everything else as if what is bad were not there."""
    N = want.shape[1]
    assert torch.equal((q[:, :N] & 0x7F) == 0x7F, bad), what
    kept = q.clone()
    kept[:, :N][bad] = 0
    check_packed(kept, s, want.masked_fill(bad, 0.0), err.masked_fill(bad, 0.0), what)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["none", "silu", "gelu", "swiglu"])
@pytest.mark.parametrize("rows", [5, 100, 1100])
def test_packed_results_that_are_no_numbers(rows, act, dtype):
    """A NaN in a row of x, an infinity in a weight's: NaN in the results of that row and that column, of the pre-activations too, and no part in
    any block's power."""
    K, N, glu = 264, 392, act == "swiglu"
    g = torch.Generator().manual_seed(rows)
    x, w, u = (torch.randn(*n, K, generator=g).double() for n in ((rows,), (1, N), (1, N)))
    x[1, 7], w[0, 9, 200], u[0, 150, 3] = float("nan"), float("inf"), float("nan")
    x8, w8, u8 = R.pack(x), R.pack(w), R.pack(u)
    out = B.make_pack_config(rows, N, DT[dtype])
    y8, pre8, up8 = B.alloc_packed_rows(out), B.alloc_packed_rows(out), B.alloc_packed_rows(out) if glu else None
    B.etr_packed_linear(B.make_linear_config(rows, K, N, 1, DT[dtype], act=ACTS[act]), gpu(x8), None, gpu(w8), w_up8=gpu(u8) if glu else None, y8=y8, pre8=pre8,
                        pre_up8=up8)
    xv, wv, uv = (R.values(*v, K).nan_to_num(nan=0.0).reshape(-1, K) for v in (x8, w8, u8))
    a, ea, up, eu = xv @ wv.t(), sum_error(xv, wv, dtype == "f32"), xv @ uv.t(), sum_error(xv, uv, dtype == "f32")
    bad_a, bad_u = (torch.zeros(rows, N, dtype=torch.bool) for _ in range(2))
    bad_a[1], bad_a[:, 9], bad_u[1], bad_u[:, 150] = True, True, True, True
    want = O.activation(act, a, up if glu else None)
    # (as in the products' tests: 40 half steps for the activations, 256 where the exponential goes without its lower part)
    some = (40 if dtype == "f32" else 296) * O.U32 * want.abs()
    err = SLOPE * ea * (up.abs() + eu) + (a.abs() + ea) * eu + some if glu else ea if act == "none" else SLOPE * ea + some
    for p8, bad, v, e in ((y8, bad_a | bad_u if glu else bad_a, want, err), (pre8, bad_a, a, ea), (up8, bad_u, up, eu)):
        if p8 is not None:
            _no_numbers(p8[0].cpu().reshape(rows, -1), p8[1].cpu().reshape(-1, rows, 4), bad, v, e, (rows, act, dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["none", "silu", "gelu", "swiglu"])
@pytest.mark.parametrize("counts", [[40, 0, 57], [300, 129], [2000, 700]], ids=str)
def test_gradients_that_are_no_numbers(counts, act, dtype):
    """NaN and infinities in dy, NaN in the packed pre-activations: NaN in the gradients of these elements along both directions, no part in any block's power,
    and no number in the biases' gradients of these columns alone."""
    rows, E, N, glu, n = sum(counts), len(counts), 264, act == "swiglu", 2 if act == "swiglu" else 1
    offsets = [sum(counts[:e]) for e in range(E + 1)]
    dy, pre8, up8 = O.randn(1, rows, N, dtype=DT[dtype], std=0.02), operand(2, rows, N, std=2.0), operand(3, rows, N)
    dy[3, 5], dy[rows - 1, 6], dy[20, 7] = float("nan"), float("inf"), float("-inf")
    pre8[0][4, 100], pre8[0][rows - 2, 101], up8[0][6, 200] = 0x7F, 0xFF, 0x7F
    cfg, Np = B.make_linear_config(rows, 64, N, E, DT[dtype], act=ACTS[act]), R.blocks(N) * 128
    d8 = B.alloc_packed_rows(B.make_pack_config(rows, n * Np, DT[dtype]))
    dt8 = B.alloc_packed_columns(B.make_pack_config(rows, n * N, DT[dtype], E=E, sorted=1))
    sums = [torch.full((E, N), 9.0, device="cuda") for _ in range(n)]
    B.etr_packed_act_backward(cfg, dy.cuda(), torch.tensor(offsets, dtype=torch.int32, device="cuda"), B.alloc_workspace(B.etr_packed_act_workspace_bytes(cfg)),
                              pre8=gpu(pre8) if act != "none" else None, pre_up8=gpu(up8) if glu else None, d8=d8, dt8=dt8, dbias=sums[0],
                              dbias_up=sums[1] if glu else None)
    a, u = R.values(*pre8, N), R.values(*up8, N)
    if act == "none":
        want = [dy.double()]
    else:
        want = derivative(act, dy.double(), a, u if glu else None)
    # (as in the element-wise part's own tests: 40 half steps of the terms)
    scale = dy.double().abs() * (1 + (u.abs() if glu else 0) + (a.abs() if act != "none" else 0))
    q, s = d8[0].cpu().reshape(rows, -1), d8[1].cpu().reshape(-1, rows, 4)
    flat = R.unlayout(s, n * R.blocks(N))
    tq, ts, at, at_s = dt8[0].cpu(), dt8[1].cpu(), 0, 0
    columns = []
    for e in range(E):
        b = R.blocks(counts[e])
        columns.append((tq[at: at + n * N * b * 128].reshape(n * N, b * 128), ts[at_s: at_s + n * N * 4 * -(-b // 4)].reshape(-1, n * N, 4)))
        at, at_s = at + n * N * b * 128, at_s + n * N * 4 * -(-b // 4)
    for h in range(n):
        bad, what = ~torch.isfinite(want[h]), (counts, act, dtype, h)
        assert 3 <= int(bad.sum()) <= 6
        w = want[h].nan_to_num(nan=0.0, posinf=0.0, neginf=0.0)
        err = torch.zeros_like(w) if act == "none" else (40 * O.U32 * scale).nan_to_num(nan=0.0, posinf=0.0)
        part = slice(h * R.blocks(N), (h + 1) * R.blocks(N))
        _no_numbers(q[:, h * Np: (h + 1) * Np], R.layout(flat[:, part]), bad, w, err, what)
        for e in range(E):
            sl = slice(offsets[e], offsets[e + 1])
            if counts[e]:
                cq, cs = columns[e]
                _no_numbers(cq[h * N: (h + 1) * N], cs[:, h * N: (h + 1) * N], bad[sl].t(), w[sl].t(), err[sl].t(), what)
            got, fine = sums[h][e].cpu(), ~bad[sl].any(0)
            assert torch.equal(torch.isfinite(got), fine), what
            bound = (counts[e] + 2) * O.U32 * w[sl].abs().sum(0) + err[sl].sum(0)
            O.assert_within(got[fine], w[sl].sum(0)[fine], bound[fine], what)


# ---- past 32 bits

def test_element_wise_part_past_4_gib():
    """The last rows and the first of gradients of 4.5e9 values, along both directions, and the sums over the last rows."""
    rows, N, used, dt = 2_200_000, 2048, 297, torch.bfloat16
    again = rows // 512 + 1
    dy = O.randn(1, 512, N, dtype=dt, std=0.02).cuda().repeat(again, 1)[:rows].contiguous()
    q, s = operand(2, 512, N, std=2.0)
    pre8 = (q.cuda().repeat(again, 1)[:rows].contiguous(), s.cuda().repeat(1, again, 1)[:, :rows].contiguous())
    assert pre8[0].numel() > 2 ** 32
    first = rows - used - 3
    offsets = torch.tensor([0, first, rows - 3], dtype=torch.int32, device="cuda")
    cfg = B.make_linear_config(rows, 64, N, 2, dt, act=B.ACT_SILU)
    d8 = tuple(t.fill_(0xA5) for t in B.alloc_packed_rows(B.make_pack_config(rows, N, dt)))
    dt8 = B.alloc_packed_columns(B.make_pack_config(rows, N, dt, E=2, sorted=1))
    dbias = torch.zeros(2, N, device="cuda")
    B.etr_packed_act_backward(cfg, dy, offsets, B.alloc_workspace(B.etr_packed_act_workspace_bytes(cfg)), pre8=pre8, d8=d8, dt8=dt8, dbias=dbias)
    d8 = (d8[0].reshape(rows, N), d8[1].reshape(-1, rows, 4))
    for sl in (slice(0, 64), slice(first - 64, first), slice(first, rows - 3)):
        a = R.values(pre8[0][sl].cpu(), pre8[1][:, sl].cpu(), N)
        want, err = derivative("silu", dy[sl].cpu().double(), a, None)[0], 40 * O.U32 * dy[sl].cpu().double().abs() * (1 + a.abs())
        check_packed(d8[0][sl].cpu(), d8[1][:, sl].cpu(), want, err, sl)
    assert bool((d8[0][-3:] == 0xA5).all()) and bool((d8[1][:, -3:] == 0xA5).all())
    # (want, err: of the last expert's rows)
    O.assert_within(dbias[1], want.sum(0), (used + 2) * O.U32 * want.abs().sum(0) + err.sum(0), "sums")
    at, at_s, b = N * 128 * R.blocks(first), N * 4 * R.blocks(R.blocks(first) * 32), R.blocks(used)
    assert at > 2 ** 32
    columns = dt8[0][at: at + N * b * 128].cpu().reshape(N, -1), dt8[1][at_s: at_s + N * 4].cpu().reshape(1, N, 4)
    check_packed(*columns, want.t(), err.t(), "along columns")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weights_gradient_of_the_most_rows(dtype):
    """2^24 rows, of one expert of 64: 32-bit offsets inside a tile of 256 rows end at 0xFF000070.  Operands of zeros but for 200 places of the
    contraction, its two ends and both sides of a k-tile's border among them."""
    rows, E, e, K, N = 1 << 24, 64, 62, 512, 512
    assert F.plan(F.WEIGHT, "none", rows, E, K, N, dtype) == "256"
    offsets = torch.tensor([0] * (e + 1) + [rows] * (E - e), dtype=torch.int32, device="cuda")
    g = torch.Generator().manual_seed(1)
    at = torch.cat([torch.tensor([0, 1, 127, 128, rows - 129, rows - 128, rows - 1]), torch.randint(2, rows - 130, (193,), generator=g)]).unique()
    t8, values = [], []
    for width in (N, K):
        q = torch.randint(0, 256, (width, len(at)), generator=g, dtype=torch.uint8)
        q[(q & 0x7F) == 0x7F] = 0x30                           # (no NaN)
        s = torch.randint(122, 133, (rows // 512, width, 4), generator=g, dtype=torch.uint8)
        block = at // 128
        values.append(R.decode(q) * torch.exp2(s[block // 4, :, block % 4].t().double() - 127))
        whole = torch.zeros(width, rows, dtype=torch.uint8, device="cuda")
        whole[:, at.cuda()] = q.cuda()
        t8.append((whole, s.cuda()))
    cfg = B.make_pack_config(rows, N, DT[dtype], E=E, sorted=1)
    assert t8[0][0].numel() <= B.etr_packed_columns_bytes(cfg) and t8[0][1].numel() <= B.etr_packed_columns_scale_bytes(cfg)
    dw = torch.full((E, N, K), 5.0, dtype=DT[dtype], device="cuda")
    B.etr_packed_weight_gradient(B.make_linear_config(rows, K, N, E, DT[dtype]), t8[0], t8[1], offsets, dw)
    da, xt = values
    want, size = da @ xt.t(), da.abs() @ xt.abs().t()
    # bf16: a product loses 2^-13 of the largest of its group, which is one of those that are summed, 16 to a group at most
    bound = (len(at) + 2) * O.U32 * size + O.half_step(DT[dtype]) * 1.01 * want.abs() + (16 * 2.0 ** -13 * size if dtype == "bf16" else 0)
    O.assert_within(dw[e], want, bound, dtype)
    dw[e] = 0
    assert not bool(dw.any())                                  # the other experts have no rows


def test_first_and_last_rows_of_a_product_past_4_gib():
    """Every element of rows at both ends by its own bound, each with the weights of its own expert."""
    rows, K, N, dt = 2_200_000, 2048, 264, torch.bfloat16
    q, s = operand(1, 512, K)
    again = rows // 512 + 1
    x8 = (q.cuda().repeat(again, 1)[:rows].contiguous(), s.cuda().repeat(1, again, 1)[:, :rows].contiguous())
    w8 = operand(2, 2, N, K, std=K ** -0.5)
    first = rows - 300
    offsets = torch.tensor([0, first, rows], dtype=torch.int32, device="cuda")
    y = torch.zeros(rows, N, dtype=dt, device="cuda")
    B.etr_packed_linear(B.make_linear_config(rows, K, N, 2, dt), x8, offsets, gpu(w8), y=y)
    wv = R.values(*w8, K)
    for sl, w in ((slice(0, 64), wv[0]), (slice(first - 64, first), wv[0]), (slice(first, rows), wv[1])):
        xv = R.values(x8[0][sl].cpu(), x8[1][:, sl].cpu(), K)
        want = xv @ w.t()
        O.assert_within(y[sl], want, sum_error(xv, w, False) + O.half_step(dt) * 1.01 * want.abs(), sl)

"""Calls that the packed operators allow at their edges: powers at both ends of their range, some of the results only, one expert without a table, two calls
at once on streams of their own."""
import pytest
import torch

import operator_refs as O
import packed_refs as R
from paper_2406_00023_amd import binding as B
from test_gpu_packed_backward import act_case
from test_gpu_packed_linear import ACTS, DT, gpu, operand, sum_error

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("small", ["x", "w"])
@pytest.mark.parametrize("rows", [5, 100, 1100])
def test_powers_at_the_ends(rows, small, dtype):
    """One operand with powers from the smallest on, 2^-127, the other with large ones: results of ordinary size.  What fp32 results add to the bound
    of a sum: values below 2^-126 are rounded to a multiple of 2^-133 on their way through bf16."""
    K, N = 648, 264
    g = torch.Generator().manual_seed(rows)

    def matrix(n, low, high):
        power = torch.randint(low, high, (n, R.blocks(K)), generator=g).double()
        return torch.randn(n, K, generator=g).double() * torch.exp2(power).repeat_interleave(128, 1)[:, :K]

    low, high = (-130, -100), (95, 118)
    x8, w8 = R.pack(matrix(rows, *(low if small == "x" else high))), R.pack(matrix(N, *(high if small == "x" else low))[None])
    assert int((x8 if small == "x" else w8)[1][..., 0].min()) == 0
    y = torch.zeros(rows, N, dtype=DT[dtype], device="cuda")
    B.etr_packed_linear(B.make_linear_config(rows, K, N, 1, DT[dtype]), gpu(x8), None, gpu(w8), y=y)
    xv, wv = R.values(*x8, K), R.values(*w8, K)[0]
    want = xv @ wv.t()
    err = sum_error(xv, wv, dtype == "f32")
    if dtype == "f32":
        other = wv.abs().sum(1)[None, :] if small == "x" else xv.abs().sum(1)[:, None]
        err = err + 2.0 ** -134 * other
    O.assert_within(y, want, err + O.half_step(DT[dtype]) * (want.abs() + err), (rows, small, dtype))


@pytest.mark.parametrize("act", ["silu", "swiglu"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [12, 400, 2600])
def test_some_of_the_results(rows, dtype, act):
    """Whatever else is asked for, a packed product's results are the same."""
    K, N, E, glu = 264, 520, 2, act == "swiglu"
    x8, w8, up8 = gpu(operand(1, rows, K)), gpu(operand(2, E, N, K, std=K ** -0.5)), gpu(operand(3, E, N, K, std=K ** -0.5)) if glu else None
    offsets = torch.tensor([0, rows // 3, rows], dtype=torch.int32, device="cuda")
    res = O.randn(4, rows, N, dtype=DT[dtype]).cuda()
    bias = [O.randn(5 + i, E, N).cuda() for i in range(2)]
    cfg, out = B.make_linear_config(rows, K, N, E, DT[dtype], act=ACTS[act]), B.make_pack_config(rows, N, DT[dtype])

    def call(y, y8, pre):
        got = {"y": torch.zeros_like(res) if y else None, "y8": B.alloc_packed_rows(out) if y8 else None, "pre8": B.alloc_packed_rows(out) if pre else None,
               "pre_up8": B.alloc_packed_rows(out) if pre and glu else None}
        B.etr_packed_linear(cfg, x8, offsets, w8, w_up8=up8, bias=bias[0], bias_up=bias[1] if glu else None, residual=res, **got)
        return {n: v if isinstance(v, tuple) else (v,) for n, v in got.items() if v is not None}

    whole = call(True, True, True)
    for asked in ((True, False, True), (False, True, True), (False, True, False), (True, True, False)):
        for n, v in call(*asked).items():
            assert all(torch.equal(a, b) for a, b in zip(v, whole[n])), (asked, n)


@pytest.mark.parametrize("rows", [40, 700])
def test_one_expert_without_a_table(rows):
    K, N, dt = 264, 136, torch.bfloat16
    table = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    x, dy, pre8 = O.randn(1, rows, K, dtype=dt).cuda(), O.randn(2, rows, N, dtype=dt).cuda(), gpu(operand(3, rows, N))
    cfg, cx = B.make_linear_config(rows, K, N, 1, dt, act=B.ACT_GELU), B.make_pack_config(rows, K, dt, sorted=1)
    runs = []
    for offsets in (None, table):
        xt8, again8, dt8 = B.alloc_packed_columns(cx), B.alloc_packed_columns(cx), B.alloc_packed_columns(B.make_pack_config(rows, N, dt, sorted=1))
        x8, d8 = B.alloc_packed_rows(cx), B.alloc_packed_rows(B.make_pack_config(rows, N, dt))
        B.etr_pack_columns(cx, x, offsets, xt8)
        B.etr_pack_rows(cx, x, x8)
        B.etr_repack_columns(cx, x8, offsets, again8)
        dbias, dw = torch.zeros(1, N, device="cuda"), torch.zeros(1, N, K, dtype=dt, device="cuda")
        ws = B.alloc_workspace(B.etr_packed_act_workspace_bytes(cfg))
        B.etr_packed_act_backward(cfg, dy, offsets, ws, pre8=pre8, d8=d8, dt8=dt8, dbias=dbias)
        B.etr_packed_weight_gradient(cfg, dt8, xt8, offsets, dw)
        runs.append([*xt8, *again8, *d8, *dt8, dbias, dw])
    assert all(torch.equal(a, b) for a, b in zip(*runs))
    assert float(runs[0][-1].float().abs().max()) > 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["none", "silu", "gelu", "swiglu"])
@pytest.mark.parametrize("counts,N,bias", [([1000, 0, 700, 1], 1160, True), ([128, 1, 129], 264, False), ([40, 0, 88], 136, True)])
def test_few_tiles_and_many_of_the_element_wise_part(counts, N, bias, act, dtype):
    """A tile's directions and halves go to workgroups of their own as long as half of a chip of 256 CUs is idle otherwise."""
    act_case(counts, N, dtype, act, seed=N, bias=bias)


@pytest.mark.parametrize("act", ["none", "swiglu"])
@pytest.mark.parametrize("rows,N", [(300, 264), (2100, 1160)])
def test_some_of_the_gradients(rows, N, act):
    """Each result of the element-wise part by itself is what it is beside the others."""
    E, dt, n = 3, torch.bfloat16, 2 if act == "swiglu" else 1
    offsets = torch.tensor([0, rows // 2, rows // 2, rows - 5], dtype=torch.int32, device="cuda")
    dy, pre = O.randn(1, rows, N, dtype=dt).cuda(), [gpu(operand(2 + i, rows, N)) if act == "swiglu" else None for i in range(2)]
    cfg = B.make_linear_config(rows, 64, N, E, dt, act=ACTS[act])
    ws = B.alloc_workspace(B.etr_packed_act_workspace_bytes(cfg))

    def call(along_rows, along_columns, sums):
        got = {"d8": B.alloc_packed_rows(B.make_pack_config(rows, n * R.blocks(N) * 128, dt)) if along_rows else None,
               "dt8": B.alloc_packed_columns(B.make_pack_config(rows, n * N, dt, E=E, sorted=1)) if along_columns else None}
        for i, name in enumerate(("dbias", "dbias_up")[:n]):
            got[name] = torch.full((E, N), 3.0, device="cuda") if sums else None
        B.etr_packed_act_backward(cfg, dy, offsets, ws, pre8=pre[0], pre_up8=pre[1], **got)
        return {k: v if isinstance(v, tuple) else (v,) for k, v in got.items() if v is not None}

    whole = call(True, True, True)
    for asked in ((True, False, False), (False, True, False), (False, False, True), (True, True, False), (False, True, True), (True, False, True)):
        for k, v in call(*asked).items():
            assert all(torch.equal(a, b) for a, b in zip(v, whole[k])), (asked, k)


def test_two_calls_at_once():
    """Nothing is shared between calls: on two streams they give what they give one after the other."""
    rows, E, K, N, dt = 2600, 4, 520, 1032, torch.bfloat16
    offsets = [torch.tensor([0, *(rows * e // E + shift for e in range(1, E)), rows], dtype=torch.int32, device="cuda") for shift in (0, 300)]
    cfg, out = B.make_linear_config(rows, K, N, E, dt, act=B.ACT_SILU), B.make_pack_config(rows, N, dt)
    cx, cn = B.make_pack_config(rows, K, dt, E=E, sorted=1), B.make_pack_config(rows, N, dt, E=E, sorted=1)

    def operands(i):
        return dict(x8=gpu(operand(10 * i + 1, rows, K)), w8=gpu(operand(10 * i + 2, E, N, K, std=K ** -0.5)), dy=O.randn(10 * i + 3, rows, N, dtype=dt).cuda())

    def results():
        return dict(y=torch.zeros(rows, N, dtype=dt, device="cuda"), pre8=B.alloc_packed_rows(out), dt8=B.alloc_packed_columns(cn), xt8=B.alloc_packed_columns(cx),
                    dbias=torch.zeros(E, N, device="cuda"), dw=torch.zeros(E, N, K, dtype=dt, device="cuda"), ws=B.alloc_workspace(B.etr_packed_act_workspace_bytes(cfg)))

    def call(i, o, r):
        B.etr_packed_linear(cfg, o["x8"], offsets[i], o["w8"], y=r["y"], pre8=r["pre8"])
        B.etr_packed_act_backward(cfg, o["dy"], offsets[i], r["ws"], pre8=r["pre8"], dt8=r["dt8"], dbias=r["dbias"])
        B.etr_repack_columns(cx, o["x8"], offsets[i], r["xt8"])
        B.etr_packed_weight_gradient(cfg, r["dt8"], r["xt8"], offsets[i], r["dw"])

    given, apart, together = [operands(i) for i in range(2)], [results() for _ in range(2)], [results() for _ in range(2)]
    for i in range(2):
        call(i, given[i], apart[i])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                call(i, given[i], together[i])
    torch.cuda.synchronize()
    for a, b in zip(apart, together):
        for n in ("y", "dbias", "dw"):
            assert torch.equal(a[n], b[n]), n
        for n in ("pre8", "dt8", "xt8"):
            assert all(torch.equal(p, q) for p, q in zip(a[n], b[n])), n

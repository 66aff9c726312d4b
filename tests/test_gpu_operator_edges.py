"""Values and tables at the edges of what the operators around the layer are given."""
import pytest
import torch

from operator_refs import DT, U32, assert_within, half_step, pair_weights, randn, unsort
from paper_2406_00023_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_weights_whose_sum_has_no_reciprocal(dtype):
    """Gates below the smallest normal number: their ratios are ordinary numbers, the inverse of their sum is not."""
    T, k, E, d = 40, 3, 6, 64
    dt = DT[dtype]
    topk = torch.rand(T, E, generator=torch.Generator().manual_seed(1)).argsort(1)[:, :k].to(torch.int32).contiguous()
    gate = torch.softmax(randn(2, T, E), 1)
    gate[::2] *= 2.0 ** -131                               # every other token; the others as they are
    gate[5] = 0                                            # nothing to divide by: no weights
    ys, dout = randn(3, T * k, d, dtype=dt), randn(4, T, d, dtype=dt, std=1e-4)
    cfg = B.make_sort_config(T, k, E, d, dt, gate_norm=1)
    offsets, row_of, pair_of = (torch.empty(n, dtype=torch.int32, device="cuda") for n in ((E + 1,), (T, k), (T * k,)))
    tk, g = topk.cuda(), gate.cuda()
    B.etr_sort_tokens(cfg, tk, None, offsets, row_of, pair_of, B.alloc_workspace(B.etr_sort_workspace_bytes(cfg)))
    out, dys, dgate = torch.empty(T, d, dtype=dt, device="cuda"), torch.empty(T * k, d, dtype=dt, device="cuda"), torch.empty(T, E, device="cuda")
    B.etr_unsort_rows(cfg, ys.cuda(), g, tk, row_of, out)
    B.etr_unsort_rows_backward(cfg, dout.cuda(), ys.cuda(), g, tk, row_of, dys, dgate)
    torch.cuda.synchronize()
    rows, hs, sums = row_of.cpu(), half_step(dt), (k + 8) * U32
    g64 = gate.double().requires_grad_(True)
    w = pair_weights(g64, topk, rows, 1)
    wd = w.detach()
    assert bool((wd[:5].sum(1) - 1).abs().max() < 1e-12) and bool((wd[5] == 0).all())
    want, mag = unsort(ys.double(), wd, rows), unsort(ys.double().abs(), wd, rows)
    assert_within(out, want, hs * want.abs() + sums * mag, "out")
    at = pair_of.cpu().long()
    want = wd.reshape(-1)[at][:, None] * dout.double()[at // k]
    assert_within(dys, want, (hs + sums) * want.abs() + 1e-38, "dys")
    dw = dout.double()[:, None, :] * ys.double()[rows.long()]
    want = torch.autograd.grad(w, g64, dw.sum(2))[0]
    s = torch.gather(gate.double(), 1, topk.long()).sum(1, keepdim=True)
    scale = torch.where(s > 0, 2 / torch.where(s > 0, s, 1.0), 0.0)
    assert float(want.abs().max()) < torch.finfo(torch.float32).max / 4      # (the definition fits fp32)
    assert_within(dgate, want, (100 + 3 * k) * U32 * scale * dw.abs().sum((1, 2))[:, None] + 1e-30, "dgate")


class Guarded:
    """Tensors between guards of their own, which say whether anything was written beside them."""
    ROOM, BYTE = 4096, 85

    def __init__(self):
        self.all = []

    def new(self, *shape, dtype=torch.float32):
        n = torch.empty(0, dtype=dtype).element_size()
        for v in shape:
            n *= v
        held = torch.full((n + 2 * self.ROOM,), self.BYTE, dtype=torch.uint8, device="cuda")
        self.all.append((held, n))
        return held[self.ROOM:self.ROOM + n].view(dtype).view(shape)

    def untouched(self):
        return all(bool((h[:self.ROOM] == self.BYTE).all()) and bool((h[self.ROOM + n:] == self.BYTE).all()) for h, n in self.all)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate_norm", [0, 1])
def test_rows_of_experts_that_do_not_exist(gate_norm, dtype):
    """Rows that exist under experts outside [0, E): no weight, no gradient, and nothing read beside the gates."""
    T, k, E, d = 52, 4, 5, 72
    dt, gen = DT[dtype], torch.Generator().manual_seed(11)
    row_of = torch.randperm(T * k, generator=gen).to(torch.int32).reshape(T, k)
    topk = torch.rand(T, E, generator=gen).argsort(1)[:, :k].to(torch.int32).contiguous()
    real = torch.ones(T, k, dtype=torch.bool)
    for place, e in ((1, E), (2, -1), (3, 63), (1, 64), (2, 2 ** 31 - 1), (3, -2 ** 31), (0, E + 3)):
        pick = torch.rand(T, generator=gen) < 0.2
        topk[pick, place] = e
        real[pick, place] = False
    topk[7], real[7] = E, False                                # a token with none that exists
    ys, dout, gate = randn(12, T * k, d, dtype=dt), randn(13, T, d, dtype=dt), torch.softmax(randn(14, T, E), 1)
    large = torch.full((3 * T, E), 1e30, device="cuda")         # what a read beside the gates would find
    large[T:2 * T] = gate.cuda()
    cfg, guard = B.make_sort_config(T, k, E, d, dt, gate_norm=gate_norm), Guarded()
    out, dys, dgate = guard.new(T, d, dtype=dt), guard.new(T * k, d, dtype=dt), guard.new(T, E)
    g, tk, ro = large[T:2 * T], topk.cuda(), row_of.cuda()
    B.etr_unsort_rows(cfg, ys.cuda(), g, tk, ro, out)
    B.etr_unsort_rows_backward(cfg, dout.cuda(), ys.cuda(), g, tk, ro, dys, dgate)
    torch.cuda.synchronize()
    assert guard.untouched()
    used = torch.where(real, row_of, -1)
    g64 = gate.double().requires_grad_(True)
    w = pair_weights(g64, topk, used, gate_norm)
    wd, hs, sums = w.detach(), half_step(dt), (k + 8) * U32
    want, mag = unsort(ys.double(), wd, used), unsort(ys.double().abs(), wd, used)
    assert_within(out, want, hs * want.abs() + sums * mag, "out")
    want = torch.zeros(T * k, d, dtype=torch.float64)
    want[row_of.reshape(-1).long()] = (wd[:, :, None] * dout.double()[:, None, :]).reshape(T * k, d)
    assert_within(dys, want, (hs + sums) * want.abs() + 1e-38, "dys")
    dw = torch.where(real[:, :, None], dout.double()[:, None, :] * ys.double()[row_of.long()], 0.0)
    want = torch.autograd.grad(w, g64, dw.sum(2))[0]
    s = torch.where(real, torch.gather(gate.double(), 1, topk.long().clamp(0, E - 1)), 0.0).sum(1, keepdim=True)
    scale = torch.where(s > 0, 2 / torch.where(s > 0, s, 1.0), 0.0) if gate_norm else 1.0
    assert_within(dgate, want, (100 + 3 * k) * U32 * scale * dw.abs().sum((1, 2))[:, None] + 1e-30, "dgate")
    assert bool((dgate[7] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d,N", [(600, 64, 72), (30, 200, 136), (3000, 264, 520)])
def test_offsets_that_make_no_sense_write_nothing_beside_the_outputs(rows, d, N, dtype):
    """Offsets that fall, overlap or lie far outside: values that make no sense, in the outputs alone."""
    E, dt, guard = 4, DT[dtype], Guarded()
    new = lambda *shape, t=dt: guard.new(*shape, dtype=t)
    cfg = B.make_linear_config(rows, d, N, E, dt, act=B.ACT_SWIGLU)
    x, dy = randn(1, rows, d, dtype=dt).cuda(), randn(2, rows, N, dtype=dt).cuda()
    w, w_up = (randn(i, E, N, d, dtype=dt).cuda() for i in (3, 4))
    bias, bias_up = (randn(i, E, N).cuda() for i in (5, 6))
    y, pre, pre_up, dx, dw, dw_up = new(rows, N), new(rows, N), new(rows, N), new(rows, d), new(E, N, d), new(E, N, d)
    dbias, dbias_up = new(E, N, t=torch.float32), new(E, N, t=torch.float32)
    ws = new(B.etr_linear_workspace_bytes(cfg), t=torch.uint8)
    R = rows
    for off in ([0, R, 0, R, 0], [R, 5, 400, 3, R], [-9, 2 ** 30, -2 ** 31, 2 ** 31 - 1, 0], [7, 7, 7, 7, 7], [R, R, R, R, R]):
        print(f"offsets {off}: {rows} x {d} x {N} {dtype}", flush=True)
        off = torch.tensor(off, dtype=torch.int32, device="cuda")
        B.etr_expert_linear(cfg, x, off, w, y, w_up=w_up, bias=bias, bias_up=bias_up, residual=dy, pre=pre, pre_up=pre_up)
        B.etr_expert_linear_backward(cfg, x, off, w, dy, ws, w_up=w_up, pre=pre, pre_up=pre_up, dx=dx, dw=dw, dw_up=dw_up, dbias=dbias, dbias_up=dbias_up)
        torch.cuda.synchronize()
        assert guard.untouched()
    for v in (dw, dw_up, dbias, dbias_up):                     # no expert had rows in the last table
        assert bool((v == 0).all())

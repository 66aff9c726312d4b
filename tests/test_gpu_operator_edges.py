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

"""Arrays past 4 GiB and odd tables: the operators around the layer keep 64-bit offsets, and tables that make no sense give values
that make none, within the arrays."""
import pytest
import torch

from paper_2406_00023_amd import binding as B

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _fill(n, d, seed):
    """Values that depend on the row and repeat along it, exact in bf16."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-8, 9, (n, d), generator=g, device="cuda", dtype=torch.int8).to(BF)


def test_sorted_rows_past_4_gib():
    T, k, E, d = 70001, 8, 16, 4096                            # 4.6 GB of rows
    g = torch.Generator(device="cuda").manual_seed(1)
    topk = torch.rand(T, E, generator=g, device="cuda").argsort(1)[:, :k].to(torch.int32).contiguous()
    x = _fill(T, d, 2)
    gate = torch.full((T, E), 0.125, device="cuda")
    cfg = B.make_sort_config(T, k, E, d, BF)
    off, row_of, pair_of = (torch.empty(n, dtype=torch.int32, device="cuda") for n in ((E + 1,), (T, k), (T * k,)))
    B.etr_sort_tokens(cfg, topk, None, off, row_of, pair_of, B.alloc_workspace(B.etr_sort_workspace_bytes(cfg)))
    xs, out = torch.empty(T * k, d, dtype=BF, device="cuda"), torch.empty(T, d, dtype=BF, device="cuda")
    B.etr_sort_rows(cfg, x, row_of, xs)
    B.etr_unsort_rows(cfg, xs, gate, topk, row_of, out)       # eight copies at an eighth each
    torch.cuda.synchronize()
    assert torch.equal(out, x)
    at = torch.tensor([0, 1, 262143, 262144, 262145, 524288, T * k - 1], device="cuda")          # on both sides of 2 and 4 GiB
    assert torch.equal(xs[at], x[(pair_of[at] // k).long()])
    dys, dgate = torch.empty_like(xs), torch.empty(T, E, device="cuda")
    B.etr_unsort_rows_backward(cfg, x, xs, gate, topk, row_of, dys, dgate)
    B.etr_sort_rows_backward(cfg, dys, row_of, out)
    torch.cuda.synchronize()
    assert torch.equal(out, x)
    rows = [0, 35000, T - 1]
    for t in rows:                                             # whole numbers below 2^24: exact in any order
        want = torch.zeros(E, dtype=torch.float64)
        want[topk[t].long().cpu()] = float(x[t].double().square().sum())
        assert torch.equal(dgate[t].cpu().double(), want)


def test_products_of_rows_past_4_gib():
    R, K, N, E = 530003, 4096, 64, 3                           # 4.3 GB of x and of dx
    x = _fill(R, K, 3)
    w = _fill(E * N, K, 4).reshape(E, N, K)
    off = torch.tensor([0, 1000, 262144, R], dtype=torch.int32, device="cuda")
    cfg = B.make_linear_config(R, K, N, E, BF)
    y = torch.empty(R, N, dtype=BF, device="cuda")
    B.etr_expert_linear(cfg, x, off, w, y)
    at = torch.tensor([0, 999, 1000, 262143, 262144, 524287, 524288, R - 1], device="cuda")
    e = torch.bucketize(at, off[1:-1].long(), right=True)
    want = (x[at].double()[:, None, :] * w[e].double()).sum(2)                # exact sums, rounded once
    torch.cuda.synchronize()
    assert torch.equal(y[at], want.to(BF))
    dy = _fill(R, N, 5)
    dx, dw, ws = torch.empty_like(x), torch.empty_like(w), B.alloc_workspace(B.etr_linear_workspace_bytes(cfg))
    B.etr_expert_linear_backward(cfg, x, off, w, dy, ws, dx=dx, dw=dw)
    torch.cuda.synchronize()
    want = (dy[at].double()[:, :, None] * w[e].double()).sum(1)
    assert torch.equal(dx[at], want.to(BF))
    want = dy[:1000].double().t().contiguous() @ x[:1000].double()            # whole numbers below 2^24
    assert torch.equal(dw[0], want.to(BF))


def test_norm_past_4_gib():
    T, d = 530003, 4096
    x = _fill(T, d, 6)
    cfg = B.make_norm_config(T, d, BF)
    h, w = torch.empty_like(x), torch.ones(d, device="cuda")
    B.etr_block_norm(cfg, x, w_pre=w, h=h)
    torch.cuda.synchronize()
    at = torch.tensor([0, 262143, 262144, 524287, 524288, T - 1], device="cuda")
    v = x[at].double()
    want = v / (v.square().mean(1, keepdim=True) + 1e-5).sqrt()
    assert float(((h[at].double() - want).abs() / want.abs().clamp_min(1e-9)).max()) <= 2.0 ** -8 + 2.0 ** -17


def test_tables_that_make_no_sense_stay_within_the_arrays():
    T, k, E, d, N = 300, 2, 4, 64, 72
    sort = B.make_sort_config(T, k, E, d, torch.float32)
    g = torch.Generator().manual_seed(7)
    wild = torch.randint(-2 ** 31, 2 ** 31 - 1, (T, k), generator=g).to(torch.int32)
    x, guard = torch.randn(T, d, device="cuda"), 4096
    room = torch.full((guard + T * k * d + guard,), 7.0, device="cuda")       # rows between two guards
    xs = room[guard:guard + T * k * d].view(T * k, d)
    gate = torch.rand(T, E, device="cuda")
    out, dgate = torch.empty(T, d, device="cuda"), torch.empty(T, E, device="cuda")
    for row_of in (wild, torch.full((T, k), T * k, dtype=torch.int32), torch.full((T, k), -5, dtype=torch.int32)):
        row_of = row_of.cuda()
        B.etr_sort_rows(sort, x, row_of, xs)
        B.etr_unsort_rows(sort, xs, gate, wild.cuda(), row_of, out)
        B.etr_unsort_rows_backward(sort, x, xs, gate, wild.cuda(), row_of, xs, dgate)
        B.etr_sort_rows_backward(sort, xs, row_of, out)
    torch.cuda.synchronize()
    assert bool((room[:guard] == 7).all()) and bool((room[-guard:] == 7).all())
    # offsets that fall, overlap or lie far outside
    R = T * k
    lin = B.make_linear_config(R, d, N, E, torch.float32, act=B.ACT_SILU)
    w, xr, dy = torch.randn(E, N, d, device="cuda"), torch.randn(R, d, device="cuda"), torch.randn(R, N, device="cuda")
    room = torch.full((guard + R * N + guard,), 7.0, device="cuda")
    y, pre = room[guard:guard + R * N].view(R, N), torch.empty(R, N, device="cuda")
    dx, dw, dbias = torch.empty(R, d, device="cuda"), torch.empty(E, N, d, device="cuda"), torch.empty(E, N, device="cuda")
    n = B.etr_linear_workspace_bytes(lin)
    ws = torch.full((n + guard,), 7, dtype=torch.uint8, device="cuda")
    for off in ([0, R, 0, R, 0], [R, 5, 400, 3, R], [-9, 2 ** 30, -2 ** 31, 2 ** 31 - 1, 0]):
        off = torch.tensor(off, dtype=torch.int32, device="cuda")
        B.etr_expert_linear(lin, xr, off, w, y, pre=pre)
        B.etr_expert_linear_backward(lin, xr, off, w, dy, ws[:n], pre=pre, dx=dx, dw=dw, dbias=dbias)
    torch.cuda.synchronize()
    assert bool((room[:guard] == 7).all()) and bool((room[-guard:] == 7).all()) and bool((ws[n:] == 7).all())

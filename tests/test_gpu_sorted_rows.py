"""Rows sorted by expert and back: tables against a sort in Python, rows bit by bit, weighted sums and gradients against
their definitions in 64 bits."""
import pytest
import torch

from operator_refs import DT, U32, assert_within, half_step, pair_weights, randn, sort_tables, unsort
from paper_2406_00023_amd import binding as B

pytestmark = pytest.mark.gpu


def _tables(cfg, topk, slot_of=None, fill=-77):
    T, k, E = cfg.T, cfg.k, cfg.E
    offsets, row_of, pair_of = (torch.full(n, fill, dtype=torch.int32, device="cuda") for n in ((E + 1,), (T, k), (T * k,)))
    ws = torch.full((max(16, B.etr_sort_workspace_bytes(cfg)),), 255, dtype=torch.uint8, device="cuda")
    B.etr_sort_tokens(cfg, topk.cuda(), None if slot_of is None else slot_of.cuda(), offsets, row_of, pair_of, ws)
    torch.cuda.synchronize()
    return offsets, row_of, pair_of


def _topk(seed, T, k, E, kind="random"):
    g = torch.Generator().manual_seed(seed)
    if kind == "one":                                          # everybody wants the last expert first
        top = torch.stack([(torch.arange(k) * (E - 1) + E - 1) % max(E, 1)] * T)
    else:
        top = torch.rand(T, E, generator=g).argsort(1)[:, :k].clone()
    if kind == "holes":
        top[torch.rand(T, k, generator=g) < 0.3] = -1
        top[torch.rand(T, k, generator=g) < 0.1] = E           # no expert either
        top[T // 2] = -1                                       # a token that goes nowhere
    if kind == "none":
        top[:] = -1
    if kind == "twice" and k > 1:
        top[:, 1] = top[:, 0]
    return top.to(torch.int32).contiguous()


# one pair; one wave; one workgroup's limit on both sides; several workgroups, a ragged last one; as many as there are
@pytest.mark.parametrize("T,k,E,kind", [(1, 1, 1, "random"), (1, 4, 8, "random"), (37, 3, 12, "holes"), (64, 1, 64, "random"), (2048, 2, 16, "random"),
                                        (2049, 2, 16, "holes"), (4097, 1, 5, "one"), (5000, 8, 64, "random"), (9001, 3, 33, "holes"),
                                        (300, 2, 6, "twice"), (700, 64, 64, "random"), (513, 2, 4, "none"), (6000, 1, 1, "random")])
def test_tables(T, k, E, kind):
    topk = _topk(T + k, T, k, E, kind)
    cfg = B.make_sort_config(T, k, E, 8, torch.float32)
    got = _tables(cfg, topk)
    for name, a, b in zip(("offsets", "row_of", "pair_of"), got, sort_tables(topk, E)):
        assert torch.equal(a.cpu(), b), name


def test_tables_of_a_million_pairs():
    """More pairs than 256 workgroups of the least share hold, against torch's stable sort."""
    T, k, E = 300007, 4, 48
    g = torch.Generator().manual_seed(5)
    topk = torch.randint(-1, E, (T, k), generator=g, dtype=torch.int32)
    cfg = B.make_sort_config(T, k, E, 8, torch.float32)
    offsets, row_of, pair_of = (v.cpu() for v in _tables(cfg, topk))
    key = torch.where(topk < 0, E, topk).reshape(-1)
    order = torch.sort(key, stable=True)[1]
    n = int((topk >= 0).sum())
    assert torch.equal(pair_of[:n], order[:n].to(torch.int32)) and bool((pair_of[n:] == -1).all())
    want = torch.full((T * k,), -1, dtype=torch.int32)
    want[order[:n]] = torch.arange(n, dtype=torch.int32)
    assert torch.equal(row_of.reshape(-1), want)
    assert offsets.tolist() == [int((topk.reshape(-1)[topk.reshape(-1) >= 0] < e).sum()) for e in range(E + 1)]


def test_tables_of_a_selection_under_a_capacity():
    """slot_of from etr_select: what it has dropped is not in use."""
    T, E, k, C = 777, 8, 2, 150
    from paper_2406_00023_amd import inputs as I
    shape = I.EtrShape("bounded", 1, T=T, d=64, E=E, D=8, k=k, capacity=C, H=8, dtype=I.DT_F32, mode=I.MODE_BIDIR, recipe="iso")
    lay = B.make_config(shape)
    score = randn(3, T, E).tanh().cuda()
    topk, slot_of = (torch.empty(T, n, dtype=torch.int32, device="cuda") for n in (k, E))
    slot_token, counts = torch.empty(E, C, dtype=torch.int32, device="cuda"), torch.empty(E, dtype=torch.int32, device="cuda")
    B.etr_select(lay, score, topk, slot_of, slot_token, counts, B.alloc_workspace(B.etr_select_workspace_bytes(lay)))
    cfg = B.make_sort_config(T, k, E, 64, torch.float32)
    got = _tables(cfg, topk, slot_of)
    for a, b in zip(got, sort_tables(topk.cpu(), E, slot_of.cpu())):
        assert torch.equal(a.cpu(), b)
    assert torch.equal(got[0][1:] - got[0][:-1], counts)
    # rows of one expert in the order of its slots
    offsets, pair_of = got[0].cpu(), got[2].cpu()
    for e in range(E):
        assert torch.equal(pair_of[offsets[e]:offsets[e + 1]] // k, slot_token[e, :int(counts[e])].cpu())


ROWS = [(1, 1, 1, 8, "random"), (3, 2, 4, 520, "random"), (40, 3, 12, 1080, "holes"), (2100, 2, 16, 512, "holes"), (2100, 2, 8, 2048, "random"),
        (5, 8, 16, 4096, "random"), (2500, 1, 4, 4104, "holes"), (6, 2, 6, 8200, "twice"), (3, 3, 4, 16384, "random"), (30, 2, 4, 264, "none"),
        (4, 2, 4, 32768, "random")]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,k,E,d,kind", ROWS)
def test_rows_and_gradients(T, k, E, d, kind, dtype):
    dt = DT[dtype]
    topk = _topk(T + d, T, k, E, kind)
    hs = half_step(dt)
    x, ys, dout, dxs = randn(1, T, d, dtype=dt), randn(2, T * k, d, dtype=dt), randn(3, T, d, dtype=dt), randn(4, T * k, d, dtype=dt)
    gate = torch.softmax(randn(5, T, E), 1)
    for gate_norm in (0, 1):
        cfg = B.make_sort_config(T, k, E, d, dt, gate_norm=gate_norm)
        offsets, row_of, pair_of = _tables(cfg, topk)
        n = int(offsets[-1])
        rows = row_of.cpu()
        ysg = ys.clone()
        ysg[n:] = float("nan")                                 # rows that nobody has: never read
        ysg, gg, tk = ysg.cuda(), gate.cuda(), topk.cuda()
        xs, dys = (torch.full((T * k, d), 7.0, dtype=dt, device="cuda") for _ in range(2))
        out, dx = (torch.full((T, d), 7.0, dtype=dt, device="cuda") for _ in range(2))
        dgate = torch.full((T, E), 7.0, device="cuda")
        B.etr_sort_rows(cfg, x.cuda(), row_of, xs)
        B.etr_unsort_rows(cfg, ysg, gg, tk, row_of, out)
        B.etr_unsort_rows_backward(cfg, dout.cuda(), ysg, gg, tk, row_of, dys, dgate)
        B.etr_sort_rows_backward(cfg, dxs.cuda(), row_of, dx)
        torch.cuda.synchronize()
        used = pair_of.cpu()[:n].long()
        assert torch.equal(xs.cpu()[:n], x[used // k]) and bool((xs[n:] == 7.0).all()) and bool((dys[n:] == 7.0).all())
        g64 = gate.double().requires_grad_(True)
        w = pair_weights(g64, topk, rows, gate_norm)
        wd, y64 = w.detach(), ys.double()
        want = unsort(y64, wd, rows)
        mag = unsort(y64.abs(), wd.abs(), rows)
        sums = (k + 8) * U32                                   # k products and sums, and the weights' own roundings
        assert_within(out, want, hs * want.abs() + sums * mag, "out")
        ones = torch.ones_like(wd)
        want = unsort(dxs.double(), ones, rows)
        assert_within(dx, want, hs * want.abs() + k * U32 * unsort(dxs.double().abs(), ones, rows), "dx")
        wr, up = wd.reshape(-1)[used][:, None], dout.double()[used // k]
        assert_within(dys[:n], wr * up, (hs + sums) * (wr * up).abs() + 1e-38, "dys")
        # weights' gradients: 64 products a lane at most, then a tree
        taken, on = y64[rows.long().clamp(min=0)], (rows >= 0)
        dw = torch.where(on, (dout.double()[:, None, :] * taken).sum(2), torch.zeros_like(wd))
        dw_mag = torch.where(on, (dout.double()[:, None, :] * taken).abs().sum(2), torch.zeros_like(wd))
        want = torch.autograd.grad(w, g64, dw)[0] if bool(on.any()) else torch.zeros(T, E, dtype=torch.float64)
        scale = 1.0
        if gate_norm:
            s = (torch.gather(gate.double(), 1, topk.long().clamp(0, E - 1)) * on).sum(1)
            scale = torch.where(s > 0, 1 / torch.where(s > 0, s, 1.0), 0.0)[:, None] * 2
        assert_within(dgate, want, (100 + 3 * k) * U32 * scale * dw_mag.sum(1, keepdim=True) + 1e-30, "dgate")


def test_gradients_against_differences():
    T, k, E, d = 12, 3, 6, 264
    topk = _topk(9, T, k, E, "holes")
    x, ys, up, gate = randn(1, T, d), randn(2, T * k, d), randn(3, T, d), torch.softmax(randn(4, T, E), 1)
    for gate_norm in (0, 1):
        cfg = B.make_sort_config(T, k, E, d, torch.float32, gate_norm=gate_norm)
        offsets, row_of, _ = _tables(cfg, topk)
        rows, n = row_of.cpu(), int(offsets[-1])
        dys, dgate, dx = torch.zeros(T * k, d, device="cuda"), torch.zeros(T, E, device="cuda"), torch.zeros(T, d, device="cuda")
        B.etr_unsort_rows_backward(cfg, up.cuda(), ys.cuda(), gate.cuda(), topk.cuda(), row_of, dys, dgate)
        dxs = randn(6, T * k, d)
        B.etr_sort_rows_backward(cfg, dxs.cuda(), row_of, dx)
        torch.cuda.synchronize()

        def loss(ysv, gv):
            return float((unsort(ysv, pair_weights(gv, topk, rows, gate_norm), rows) * up.double()).sum())

        step = 1e-5
        for which, grad, at in (("ys", dys, ys.double()), ("gate", dgate, gate.double())):
            v = randn(8, *at.shape).double()
            args = (lambda q: (q, gate.double())) if which == "ys" else (lambda q: (ys.double(), q))
            diff = (loss(*args(at + step * v)) - loss(*args(at - step * v))) / (2 * step)
            prod = grad.cpu().double() * v
            assert abs(float(prod.sum()) - diff) <= 2e-5 * float(prod.abs().sum()) + 1e-5 * max(1.0, abs(diff)), which
        # the rows are taken linearly: <xs, dxs> = <x, dx>
        pairs = torch.where(rows.reshape(-1) >= 0)[0]
        lhs = float((x.double()[pairs // k] * dxs.double()[rows.reshape(-1)[pairs].long()]).sum())
        prod = x.double() * dx.cpu().double()
        assert abs(float(prod.sum()) - lhs) <= 1e-5 * float(prod.abs().sum())

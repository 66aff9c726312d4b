"""Packing kernels against the 64-bit definitions, byte for byte (powers of two make the division exact, so that there is one right answer)."""
import pytest
import torch

import packed_refs as R
from paper_2406_00023_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
GUARD = 256


def guarded(nbytes):
    """A buffer of `nbytes` between guards, all of it 0xA5."""
    whole = torch.full((nbytes + 2 * GUARD,), 0xA5, dtype=torch.uint8, device="cuda")
    return whole, whole[GUARD: GUARD + nbytes]


def intact(whole):
    return bool((whole[:GUARD] == 0xA5).all()) and bool((whole[-GUARD:] == 0xA5).all())


def matrix(seed, rows, K, dtype):
    """Blocks of unlike size, with the values where rounding and powers can go wrong."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, K, generator=g) * torch.exp2(torch.randint(-12, 12, (rows, R.blocks(K)), generator=g).float()).repeat_interleave(128, 1)[:, :K]
    x = x.to(DT[dtype])
    for r in range(0, rows, 3):                                # the largest of a block on the border between two powers, and next to it
        c = (r * 37) % K
        border = torch.tensor(448.0 * 2.0 ** (r % 7 - 3)).to(DT[dtype])
        x[r, c] = border if r % 2 else torch.nextafter(border.float(), torch.tensor(1e30)).to(DT[dtype])
    if rows > 4:
        x[4, :] = 0
        x[2, K // 2:] = 0
    return x


def same_codes(got, want):
    nan = (want & 127) == 127
    return torch.equal(got[~nan], want[~nan]) and bool(((got[nan] & 127) == 127).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("E,rows,K", [(1, 1, 8), (1, 3, 128), (2, 5, 136), (1, 7, 504), (3, 2, 512), (1, 9, 520), (2, 4, 2056), (1, 130, 1080), (1, 2, 8200)])
def test_rows(E, rows, K, dtype):
    x = matrix(rows * K, E * rows, K, dtype).reshape(E, rows, K)
    cfg = B.make_pack_config(rows, K, DT[dtype], E=E)
    (wq, q), (ws, s) = guarded(B.etr_packed_rows_bytes(cfg)), guarded(B.etr_packed_rows_scale_bytes(cfg))
    B.etr_pack_rows(cfg, x.cuda(), (q, s))
    want_q, want_s = R.pack(x.double())
    assert torch.equal(s.cpu().reshape(want_s.shape), want_s) and torch.equal(q.cpu().reshape(want_q.shape), want_q)
    assert intact(wq) and intact(ws)
    whole, y = guarded(x.numel() * x.element_size())
    B.etr_unpack_rows(cfg, (q, s), y.view(DT[dtype]))
    assert torch.equal(y.view(DT[dtype]).cpu().double().reshape(x.shape), R.values(want_q, want_s, K)) and intact(whole)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_that_are_no_numbers(dtype):
    t = DT[dtype]
    big, tiny = torch.finfo(t).max, 2.0 ** -133 if dtype == "bf16" else 2.0 ** -149
    x = torch.randn(12, 256, generator=torch.Generator().manual_seed(3))
    x[0, 3], x[1, 5], x[2, 7] = float("inf"), float("-inf"), float("nan")
    x[3, :] = float("nan")
    x[4, 0], x[4, 200] = big, -big
    x[5, :] = tiny
    x[6, :] = -0.0
    x[7, 0] = 2.0 ** -126
    x[7, 1:] = 0
    x[8, :128] = float("inf")
    x[9, 0] = 1e30
    x = x.to(t)
    cfg = B.make_pack_config(12, 256, t)
    out = B.alloc_packed_rows(cfg)
    B.etr_pack_rows(cfg, x.cuda(), out)
    q, s = out[0].cpu().reshape(12, 256), out[1].cpu().reshape(1, 12, 4)
    want_q, want_s = R.pack(x.double())
    assert torch.equal(s, want_s) and same_codes(q, want_q)
    # the same along columns, whose blocks are other ones
    cfg = B.make_pack_config(12, 256, t)
    out = B.alloc_packed_columns(cfg)
    B.etr_pack_columns(cfg, x.cuda(), None, out)
    want_q, want_s = R.pack(x.double().t().contiguous())
    assert torch.equal(out[1].cpu().reshape(want_s.shape), want_s) and same_codes(out[0].cpu().reshape(want_q.shape), want_q)
    # and what is no number is one in what the matrix stands for
    y = torch.zeros(12, 256, dtype=t, device="cuda")
    rows = B.alloc_packed_rows(cfg)
    B.etr_pack_rows(cfg, x.cuda(), rows)
    B.etr_unpack_rows(cfg, rows, y)
    assert torch.equal(torch.isnan(y.cpu()), ~torch.isfinite(x))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_unpack_of_every_code_and_power(dtype):
    q = torch.arange(256, dtype=torch.int32).to(torch.uint8).repeat(255, 1).reshape(255, 256)
    s = torch.full((1, 255, 4), 127, dtype=torch.uint8)
    s[0, :, 0] = s[0, :, 1] = torch.arange(255, dtype=torch.int32).to(torch.uint8)
    y = torch.zeros(255, 256, dtype=DT[dtype], device="cuda")
    B.etr_unpack_rows(B.make_pack_config(255, 256, DT[dtype]), (q.cuda(), s.cuda()), y)
    want = R.values(q, s, 256).float().to(DT[dtype])
    assert torch.equal(y.cpu().nan_to_num(nan=0.5), want.nan_to_num(nan=0.5)) and torch.equal(torch.isnan(y.cpu()), torch.isnan(want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,k,E,d", [(1, 1, 1, 8), (33, 2, 16, 2048), (130, 3, 5, 1080), (9, 8, 64, 520)])
def test_sorted_rows(T, k, E, d, dtype):
    g = torch.Generator().manual_seed(T)
    x = matrix(T, T, d, dtype)
    row_of = torch.randperm(T * k, generator=g).to(torch.int32).reshape(T, k)
    row_of[torch.rand(T, k, generator=g) < 0.2] = -1
    n = T * k
    cfg, out_cfg = B.make_sort_config(T, k, E, d, DT[dtype]), B.make_pack_config(n, d, DT[dtype])
    (wq, q), (ws, s) = guarded(B.etr_packed_rows_bytes(out_cfg)), guarded(B.etr_packed_rows_scale_bytes(out_cfg))
    B.etr_pack_sorted_rows(cfg, x.cuda(), row_of.cuda(), (q, s))
    code, power = R.pack_blocks(x.double())
    want_q = torch.full((n, code.shape[1]), 0xA5, dtype=torch.uint8)
    want_s = torch.full((R.blocks(power.shape[1] * 32), n, 4), 0xA5, dtype=torch.uint8)
    token = R.layout(power)
    for t in range(T):
        for j in range(k):
            if row_of[t, j] >= 0:
                want_q[row_of[t, j]], want_s[:, row_of[t, j]] = code[t], token[:, t]
    assert torch.equal(q.cpu().reshape(want_q.shape), want_q) and torch.equal(s.cpu().reshape(want_s.shape), want_s)
    assert intact(wq) and intact(ws)


COUNTS = [[1], [128], [129, 0, 127], [0, 0, 5], [600, 1, 0, 513, 128], [0]]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts", COUNTS)
@pytest.mark.parametrize("K", [8, 136, 520])
def test_columns_of_sorted_rows(counts, K, dtype):
    E, used = len(counts), sum(counts)
    rows = max(used + 3, 1)                                    # and rows that belong to nobody
    offsets = [sum(counts[:e]) for e in range(E + 1)]
    x = matrix(K + rows, rows, K, dtype)
    x[used:] = float("nan")
    want_q, want_s = R.pack_columns(x.double(), offsets)
    cfg = B.make_pack_config(rows, K, DT[dtype], E=E, sorted=1)
    dev = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    (wq, q), (ws, s) = guarded(B.etr_packed_columns_bytes(cfg)), guarded(B.etr_packed_columns_scale_bytes(cfg))
    assert q.numel() >= want_q.numel() and s.numel() >= want_s.numel()
    B.etr_pack_columns(cfg, x.cuda(), dev, (q, s))
    assert torch.equal(q[: want_q.numel()].cpu(), want_q) and torch.equal(s[: want_s.numel()].cpu(), want_s)
    assert bool((q[want_q.numel():] == 0xA5).all()) and bool((s[want_s.numel():] == 0xA5).all()) and intact(wq) and intact(ws)
    # the same from rows that are packed already
    packed = B.alloc_packed_rows(cfg)
    B.etr_pack_rows(cfg, x.cuda(), packed)
    want_q, want_s = R.pack_columns(R.values(*R.pack(x.double()), K), offsets)
    (wq, q), (ws, s) = guarded(B.etr_packed_columns_bytes(cfg)), guarded(B.etr_packed_columns_scale_bytes(cfg))
    B.etr_repack_columns(cfg, packed, dev, (q, s))
    assert torch.equal(q[: want_q.numel()].cpu(), want_q) and torch.equal(s[: want_s.numel()].cpu(), want_s)
    assert bool((q[want_q.numel():] == 0xA5).all()) and bool((s[want_s.numel():] == 0xA5).all()) and intact(wq) and intact(ws)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("E,rows,K", [(1, 1, 8), (2, 130, 136), (3, 520, 264), (1, 1048, 40)])
def test_columns_of_stacks(E, rows, K, dtype):
    x, up = (matrix(rows + K + i, E * rows, K, dtype).reshape(E, rows, K) for i in (0, 1))
    cfg = B.make_pack_config(rows, K, DT[dtype], E=E)
    (wq, q), (ws, s) = guarded(B.etr_packed_columns_bytes(cfg)), guarded(B.etr_packed_columns_scale_bytes(cfg))
    B.etr_pack_columns(cfg, x.cuda(), None, (q, s))
    want_q, want_s = R.pack(x.double().transpose(1, 2).contiguous())
    assert torch.equal(q.cpu().reshape(want_q.shape), want_q) and torch.equal(s.cpu().reshape(want_s.shape), want_s) and intact(wq) and intact(ws)
    packed = B.alloc_packed_rows(cfg)
    B.etr_pack_rows(cfg, x.cuda(), packed)
    B.etr_repack_columns(cfg, packed, None, (q, s))
    again_q, again_s = R.pack(R.values(*R.pack(x.double()), K).transpose(1, 2).contiguous())
    assert torch.equal(q.cpu().reshape(want_q.shape), again_q) and torch.equal(s.cpu().reshape(want_s.shape), again_s)
    # two stacks beside each other
    half = R.blocks(rows) * 128
    pair = B.make_pack_config(K, 2 * half, DT[dtype], E=E)
    (wq, q), (ws, s) = guarded(B.etr_packed_rows_bytes(pair)), guarded(B.etr_packed_rows_scale_bytes(pair))
    B.etr_pack_columns_pair(cfg, x.cuda(), up.cuda(), (q, s))
    both = torch.cat([torch.nn.functional.pad(v.double().transpose(1, 2), (0, half - rows)) for v in (x, up)], 2)
    want_q, want_s = R.pack(both)
    assert torch.equal(q.cpu().reshape(want_q.shape), want_q) and torch.equal(s.cpu().reshape(want_s.shape), want_s) and intact(wq) and intact(ws)


@pytest.mark.parametrize("offsets", [[0, 300, 100, 300], [300, 0, 300, 0], [-5, 7, 1000, 2], [0, 0, 0, 0]])
def test_offsets_that_do_not_ascend_stay_in_bounds(offsets):
    rows, K = 300, 136
    x = matrix(1, rows, K, "bf16").cuda()
    cfg = B.make_pack_config(rows, K, torch.bfloat16, E=3, sorted=1)
    (wq, q), (ws, s) = guarded(B.etr_packed_columns_bytes(cfg)), guarded(B.etr_packed_columns_scale_bytes(cfg))
    B.etr_pack_columns(cfg, x, torch.tensor(offsets, dtype=torch.int32, device="cuda"), (q, s))
    torch.cuda.synchronize()
    assert intact(wq) and intact(ws)

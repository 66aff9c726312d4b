"""Packed operators as programs use them: again and again on the same buffers, in place, on another stream, in a graph, with tables that make no sense, past
4 GiB, and put together as a block."""
import pytest
import torch

import operator_refs as O
import packed_refs as R
from paper_2406_00023_amd import binding as B
from paper_2406_00023_amd.dropless_block import BlockShape, DroplessBlock, PackedBlock, random_weights
from test_gpu_dropless_block import _off, _outputs, _reference
from test_gpu_pack import guarded, intact
from test_gpu_packed_linear import gpu, operand, sum_error

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,E,K,N", [(12, 4, 264, 136), (400, 4, 264, 520), (2600, 2, 520, 1032)])
def test_the_same_bits_every_time_and_in_place(rows, E, K, N):
    x8, w8, up8 = gpu(operand(1, rows, K)), gpu(operand(2, E, N, K, std=K ** -0.5)), gpu(operand(3, E, N, K, std=K ** -0.5))
    offsets = torch.tensor([rows * e // E for e in range(E + 1)], dtype=torch.int32, device="cuda")
    res = O.randn(4, rows, N, dtype=torch.bfloat16).cuda()
    cfg = B.make_linear_config(rows, K, N, E, torch.bfloat16, act=B.ACT_SWIGLU)
    first = None
    for _ in range(3):
        y, y8, pre8, up = res.clone(), *(B.alloc_packed_rows(B.make_pack_config(rows, N, torch.bfloat16)) for _ in range(3))
        B.etr_packed_linear(cfg, x8, offsets, w8, y=y, w_up8=up8, residual=y, y8=y8, pre8=pre8, pre_up8=up)        # y is the residual
        apart, other8 = torch.zeros_like(res), B.alloc_packed_rows(B.make_pack_config(rows, N, torch.bfloat16))
        B.etr_packed_linear(cfg, x8, offsets, w8, y=apart, w_up8=up8, residual=res, y8=other8)      # (without packed results the sums may go in another order)
        got = [y, *y8, *pre8, *up]
        assert torch.equal(y, apart) and torch.equal(y8[0], other8[0])
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(got, first))
    # and the sums of the biases' gradients, whose parts are joined by another kernel
    dy = O.randn(5, rows, N, dtype=torch.bfloat16).cuda()
    ws = B.alloc_workspace(B.etr_packed_act_workspace_bytes(cfg))
    first = None
    for _ in range(3):
        ws.fill_(0x7F)
        out = [torch.full((E, N), 3.0, device="cuda") for _ in range(2)]
        B.etr_packed_act_backward(cfg, dy, offsets, ws, pre8=pre8, pre_up8=up, dbias=out[0], dbias_up=out[1])
        first = first or out
        assert all(torch.equal(a, b) for a, b in zip(out, first))


@pytest.mark.parametrize("offsets", [[0, 300, 100, 300], [300, 0, 300, 0], [-5, 7, 1000, 2], [0, 0, 0, 0], [2 ** 31 - 1, -2 ** 31, 5, 9]])
@pytest.mark.parametrize("act", [B.ACT_NONE, B.ACT_SWIGLU])
def test_tables_that_make_no_sense_stay_in_bounds(offsets, act):
    rows, E, K, N = 300, 3, 136, 264
    glu, n, dt = act == B.ACT_SWIGLU, 2 if act == B.ACT_SWIGLU else 1, torch.bfloat16
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    x8, w8, up8, pre8 = gpu(operand(1, rows, K)), gpu(operand(2, E, N, K)), gpu(operand(3, E, N, K)), gpu(operand(4, rows, N))
    cfg, Np = B.make_linear_config(rows, K, N, E, dt, act=act), R.blocks(N) * 128
    wholes = []

    def room(nbytes):
        whole, inner = guarded(nbytes)
        wholes.append(whole)
        return inner

    def packed(c, columns=False):
        a, b = (B.etr_packed_columns_bytes, B.etr_packed_columns_scale_bytes) if columns else (B.etr_packed_rows_bytes, B.etr_packed_rows_scale_bytes)
        return room(a(c)), room(b(c))

    out = B.make_pack_config(rows, N, dt)
    y8, p8, pu8 = packed(out), packed(out), packed(out) if glu else None
    y = room(rows * N * 2).view(dt)
    B.etr_packed_linear(cfg, x8, off, w8, y=y, w_up8=up8 if glu else None, y8=y8, pre8=p8, pre_up8=pu8)
    d8 = packed(B.make_pack_config(rows, n * Np, dt))
    dt8, xt8 = packed(B.make_pack_config(rows, n * N, dt, E=E, sorted=1), True), packed(B.make_pack_config(rows, K, dt, E=E, sorted=1), True)
    dbias = [room(E * N * 4).view(torch.float32) for _ in range(n)]
    ws = room(B.etr_packed_act_workspace_bytes(cfg))
    dy = O.randn(5, rows, N, dtype=dt).cuda()
    B.etr_packed_act_backward(cfg, dy, off, ws, pre8=None if act == B.ACT_NONE else pre8, pre_up8=pre8 if glu else None, d8=d8, dt8=dt8, dbias=dbias[0],
                              dbias_up=dbias[1] if glu else None)
    B.etr_repack_columns(B.make_pack_config(rows, K, dt, E=E, sorted=1), x8, off, xt8)
    dw = [room(E * N * K * 2).view(dt) for _ in range(n)]
    B.etr_packed_weight_gradient(cfg, dt8, xt8, off, dw[0], dw_up=dw[1] if glu else None)
    torch.cuda.synchronize()
    assert all(intact(w) for w in wholes)


def test_past_4_gib():
    """Rows, and offsets in bytes, that 32 bits do not hold: packing, the product and its results, looked at where they end."""
    rows, K, N = 2_200_000, 2048, 1032
    x = torch.randn(512, K, device="cuda").to(torch.bfloat16).repeat(rows // 512 + 1, 1)[:rows].contiguous()
    cfg = B.make_pack_config(rows, K, torch.bfloat16)
    x8 = B.alloc_packed_rows(cfg)
    assert x8[0].numel() > 2 ** 32
    B.etr_pack_rows(cfg, x, x8)
    want_q, want_s = R.pack(x[-300:].cpu().double())
    assert torch.equal(x8[0].reshape(rows, K)[-300:].cpu(), want_q) and torch.equal(x8[1].reshape(4, rows, 4)[:, -300:].cpu(), want_s)
    back = torch.zeros_like(x)
    B.etr_unpack_rows(cfg, x8, back)
    assert torch.equal(back[-300:].cpu().double(), R.values(want_q, want_s, K))
    del back
    w8 = operand(2, 2, N, K, std=K ** -0.5)
    offsets = torch.tensor([0, rows - 300, rows - 3], dtype=torch.int32, device="cuda")
    y = torch.full((rows, N), 7.0, dtype=torch.bfloat16, device="cuda")
    y8 = B.alloc_packed_rows(B.make_pack_config(rows, N, torch.bfloat16))
    B.etr_packed_linear(B.make_linear_config(rows, K, N, 2, torch.bfloat16), x8, offsets, gpu(w8), y=y, y8=y8)
    xv, wv = R.values(want_q, want_s, K), R.values(*w8, K)
    want = xv[:297] @ wv[1].t()
    bound = sum_error(xv[:297], wv[1], False) + O.half_step(torch.bfloat16) * 1.01 * want.abs()
    O.assert_within(y[-300:-3], want, bound, "last rows")
    assert bool((y[-3:] == 7.0).all())
    O.assert_within(y[:64], R.values(*R.pack(x[:64].cpu().double()), K) @ wv[0].t(), 1.2 * bound[:64].max().expand(64, N), "first rows")
    q, s = y8[0].reshape(rows, -1)[-300:-3].cpu(), y8[1].reshape(3, rows, 4)[:, -300:-3].cpu()
    unit = torch.exp2(R.unlayout(s, 9).double() - 127).repeat_interleave(128, 1)[:, :N]
    O.assert_within(R.values(q, s, N), want, 2.0 ** -4 * (want.abs() + bound) + 2.0 ** -10 * unit + bound, "last packed rows")
    # along columns, one expert with nearly all rows
    xt = B.alloc_packed_columns(B.make_pack_config(rows, K, torch.bfloat16, E=2, sorted=1))
    B.etr_repack_columns(B.make_pack_config(rows, K, torch.bfloat16, E=2, sorted=1), x8, offsets, xt)
    blocks = R.blocks(rows - 300)
    tq, ts = R.pack(xv[:297].t().contiguous())
    at, at_s = K * blocks * 128, K * 4 * -(-blocks // 4)
    assert torch.equal(xt[0][at: at + tq.numel()].cpu(), tq.reshape(-1)) and torch.equal(xt[1][at_s: at_s + ts.numel()].cpu(), ts.reshape(-1))


def test_more_rows_than_waves():
    """The row kernels walk what is over 2^22 rows."""
    rows, K = (1 << 22) + 1001, 8
    x = torch.randn(rows, K, device="cuda")
    cfg = B.make_pack_config(rows, K, torch.float32)
    x8 = B.alloc_packed_rows(cfg)
    B.etr_pack_rows(cfg, x, x8)
    back = torch.zeros_like(x)
    B.etr_unpack_rows(cfg, x8, back)
    for part in (slice(0, 500), slice((1 << 22) - 250, (1 << 22) + 250), slice(rows - 500, rows)):
        want_q, want_s = R.pack(x[part].cpu().double())
        assert torch.equal(x8[0].reshape(rows, 128)[part].cpu(), want_q) and torch.equal(x8[1].reshape(1, rows, 4)[:, part].cpu(), want_s)
        assert torch.equal(back[part].cpu().double(), R.values(want_q, want_s, K))


# relative 2-norms.  A rounding to e4m3 is off by 2^-4 at most; roundings along a path add up in squares.  Outputs: tokens, weights, activation, weights
# again: sqrt(4) 2^-4.  Gradients: those that they multiply (the outputs' share of the activations included), two gradients, two weights: sqrt(9) 2^-4
TOL_OUT, TOL_GRAD = 2 * 2.0 ** -4, 3 * 2.0 ** -4


@pytest.mark.parametrize("shape", [BlockShape(1, 256, 8, 8, 2, 128, torch.bfloat16), BlockShape(37, 136, 4, 8, 2, 72, torch.float32),
                                   BlockShape(700, 512, 16, 16, 2, 704, torch.bfloat16), BlockShape(2000, 512, 4, 16, 2, 1408, torch.bfloat16, gate_norm=1)])
def test_block_against_64_bits(shape):
    block = PackedBlock(shape)
    w_emb, w = random_weights(shape)
    block.pack_weights(w)
    g = torch.Generator().manual_seed(3)
    x, dx_out, dh = (torch.randn(shape.T, shape.d, generator=g).to(shape.dtype).cuda() for _ in range(3))
    block.forward(x, w_emb, w)
    block.backward(x, w_emb, w, dx_out, dh)
    torch.cuda.synchronize()
    x_out, h_next, grads = _reference(block, x, w_emb, w, dx_out, dh)
    assert _off(block.x_out, x_out) <= TOL_OUT and _off(block.h_next, h_next) <= TOL_OUT
    assert _off(block.dx, grads.pop("x")) <= TOL_GRAD
    for n, want in grads.items():
        assert _off(block.grads[n], want) <= TOL_GRAD, n
    # the routing does not see the experts: the same tables as without packing
    plain = DroplessBlock(shape)
    plain.forward(x, w_emb, w)
    assert torch.equal(plain.row_of, block.row_of) and torch.equal(plain.offsets, block.offsets)


@pytest.mark.parametrize("shape", [BlockShape(300, 256, 8, 8, 3, 136, torch.float32), BlockShape(2000, 512, 4, 16, 2, 1408, torch.bfloat16)])
def test_graph_replays_match_eager_steps_on_another_stream(shape):
    captured, eager = PackedBlock(shape), PackedBlock(shape)
    w_emb, w = random_weights(shape)
    x, dx_out, dh = (torch.randn(shape.T, shape.d, device="cuda").to(shape.dtype) for _ in range(3))

    def step(block):
        block.pack_weights(w)
        block.forward(x, w_emb, w)
        block.backward(x, w_emb, w, dx_out, dh)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(captured)                                         # outside the capture first: kernel attributes are set here
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(captured)
    x0 = x.clone()
    for rep in range(3):
        x.copy_(torch.roll(x0, shifts=7 * rep + 1, dims=0))
        dh.mul_(-0.5)
        w["w_gate"].mul_(1.25)                                 # weights change between the steps, and are packed in them
        for v in _outputs(captured).values():
            v.fill_(3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        step(eager)
        torch.cuda.synchronize()
        for n, v in _outputs(captured).items():
            assert torch.equal(v, _outputs(eager)[n]), (rep, n)

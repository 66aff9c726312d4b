"""Every stage of the packed block by itself, against 64 bits on the packed operands that the block holds: each product has the operand that it should
have, element by element."""
import pytest
import torch

import operator_refs as O
import packed_refs as R
from paper_2406_00023_amd.dropless_block import BlockShape, PackedBlock, random_weights
from test_gpu_packed_backward import derivative
from test_gpu_packed_linear import check_packed, sum_error

pytestmark = pytest.mark.gpu

SHAPES = [BlockShape(40, 264, 4, 8, 2, 136, torch.bfloat16), BlockShape(37, 136, 4, 8, 2, 72, torch.float32), BlockShape(900, 512, 4, 16, 2, 392, torch.bfloat16)]


def split(packed, rows):
    """Codes [rows][Kp] and scales [groups][rows][4] of one packed matrix, on the CPU."""
    return packed[0].cpu().reshape(rows, -1), packed[1].cpu().reshape(-1, rows, 4)


def stack(packed, E, rows):
    return packed[0].cpu().reshape(E, rows, -1), packed[1].cpu().reshape(E, -1, rows, 4)


@pytest.mark.parametrize("shape", SHAPES)
def test_stages(shape):
    block, dt = PackedBlock(shape), shape.dtype
    w_emb, w = random_weights(shape)
    g = torch.Generator().manual_seed(7)
    x, dx_out, dh = (torch.randn(shape.T, shape.d, generator=g).to(dt).cuda() for _ in range(3))
    block.pack_weights(w)
    block.forward(x, w_emb, w)
    block.backward(x, w_emb, w, dx_out, dh)
    E, d, H, rows, wide = shape.E, shape.d, shape.H, shape.T * shape.k, dt == torch.float32
    ends = block.offsets.tolist()
    assert ends[E] == rows
    Hp, parts = R.blocks(H) * 128, [slice(a, b) for a, b in zip(ends[:-1], ends[1:])]
    cpu = {n: v.cpu().double() for n, v in w.items()}

    def product(got, a, b, what):
        for e, sl in enumerate(parts):
            want = a[sl] @ b[e].t()
            O.assert_within(got[sl], want, sum_error(a[sl], b[e], wide) + O.half_step(dt) * 1.01 * want.abs(), (what, e))

    def contraction(got, a, b, what):
        for e in range(E):
            if ends[e + 1] > ends[e]:
                want = a[e] @ b[e].t()
                O.assert_within(got[e], want, sum_error(a[e], b[e], wide) + O.half_step(dt) * 1.01 * want.abs(), (what, e))

    # the weights, along rows and along columns: the bytes of the definition
    for n, at, v in (("w_gate", H, cpu["w_gate"]), ("w_up", H, cpu["w_up"]), ("w_down", d, cpu["w_down"]), ("down_t", H, cpu["w_down"].transpose(1, 2)),
                     ("up_t", d, torch.cat([torch.nn.functional.pad(cpu[m].transpose(1, 2), (0, Hp - H)) for m in ("w_gate", "w_up")], 2))):
        assert all(torch.equal(p, q) for p, q in zip(stack(block.w8[n], E, at), R.pack(v))), n
    weights = {n: R.values(*stack(block.w8[n], E, at), K) for n, at, K in (("w_gate", H, d), ("w_up", H, d), ("w_down", d, H), ("down_t", H, d), ("up_t", d, 2 * Hp))}
    # the tokens, by expert
    sorted_h = torch.zeros(rows, d, dtype=torch.float64)
    sorted_h[block.row_of.cpu().long().reshape(-1)] = block.h.cpu().double().repeat_interleave(shape.k, 0)
    assert all(torch.equal(p, q) for p, q in zip(split(block.hs8, rows), R.pack(sorted_h)))
    hs, a8 = R.values(*split(block.hs8, rows), d), R.values(*split(block.a8, rows), H)
    pre = []
    for n, m in (("pre8", "w_gate"), ("pre_up8", "w_up")):
        want = torch.cat([hs[sl] @ weights[m][e].t() for e, sl in enumerate(parts)])
        err = torch.cat([sum_error(hs[sl], weights[m][e], wide) for e, sl in enumerate(parts)])
        check_packed(*split(getattr(block, n), rows), want, err, n)
        pre.append(R.values(*split(getattr(block, n), rows), H))
    product(block.ys, a8, weights["w_down"], "ys")
    # backward of the down product
    dys = block.dys.cpu().double()
    assert all(torch.equal(p, q) for p, q in zip(split(block.dys8, rows), R.pack(dys)))
    product(block.da, R.values(*split(block.dys8, rows), d), weights["down_t"], "da")
    for n, v, width in (("dyst8", dys, d), ("at8", a8, H), ("hst8", hs, d)):
        q, s = R.pack_columns(v, ends)
        got = getattr(block, n)
        assert torch.equal(got[0].cpu()[: q.numel()], q) and torch.equal(got[1].cpu()[: s.numel()], s), n

    def columns(n, width):
        return R.column_parts(getattr(block, n)[0].cpu(), getattr(block, n)[1].cpu(), width, ends)

    contraction(block.grads["w_down"], columns("dyst8", d), columns("at8", H), "w_down")
    # the element-wise part between the products, by the bound of its own tests
    da = block.da.cpu().double()
    want = derivative("swiglu", da, *pre)
    err = 40 * O.U32 * da.abs() * (1 + pre[0].abs() + pre[1].abs())
    q, s = split(block.dab8, rows)
    flat = R.unlayout(s, 2 * Hp // 128)
    for h in range(2):
        check_packed(q[:, h * Hp: (h + 1) * Hp], R.layout(flat[:, h * Hp // 128: (h + 1) * Hp // 128]), want[h], err, ("dab8", h))
    # backward of the gate and up products
    product(block.dhs, R.values(q, s, 2 * Hp), weights["up_t"], "dhs")
    both, tokens = columns("dabt8", 2 * H), columns("hst8", d)
    contraction(block.grads["w_gate"], [v[:H] for v in both], tokens, "w_gate")
    contraction(block.grads["w_up"], [v[H:] for v in both], tokens, "w_up")

"""The packed block's choice of sums, and its outputs after its weights have changed."""
import pytest
import torch

import packed_refs as R
from paper_2406_00023_amd import binding as B
from paper_2406_00023_amd.dropless_block import BlockShape, PackedBlock, random_weights
from test_gpu_dropless_block import _outputs
from test_gpu_packed_linear import check_packed, sum_error

pytestmark = pytest.mark.gpu

SHAPES = [BlockShape(40, 264, 4, 8, 2, 136, torch.bfloat16), BlockShape(1500, 512, 4, 16, 2, 704, torch.bfloat16)]


def inputs(shape):
    g = torch.Generator().manual_seed(5)
    return [torch.randn(shape.T, shape.d, generator=g).to(shape.dtype).cuda() for _ in range(3)]


@pytest.mark.parametrize("exact", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_sums_of_what_is_kept(shape, exact):
    """The kept pre-activations against 64 bits: element by element by the bound of the sums that were asked for, and the 2-norm of their distance from what is
    nearest.  Steps of e4m3 are 2^-3 of a value at most; an error e crosses a tie with a probability of 2 e / step and is a step then, so that the square of
    that norm is sum(2 e step) <= 2^-2 sum(e |v|) <= 2^-2 r |v|^2, with r the sums' error in norm: off <= sqrt(r) / 2.  fp32: K + 2 roundings of
    partial sums, which in random data are no larger than the results, r = (K + 2) 2^-24.  8-bit matrix pipe: 2^-13 of the largest of 16 products for each, 16 of them
    to a result's size of sqrt(16) of that largest at least, r = 2^-11."""
    block = PackedBlock(shape, exact_sums=exact)
    w_emb, w = random_weights(shape)
    block.pack_weights(w)
    x = inputs(shape)[0]
    block.forward(x, w_emb, w)
    rows, E, d, H = shape.T * shape.k, shape.E, shape.d, shape.H
    ends = block.offsets.tolist()
    xv = R.values(block.hs8[0].cpu().reshape(rows, -1), block.hs8[1].cpu().reshape(-1, rows, 4), d)
    for name, weight in (("pre8", "w_gate"), ("pre_up8", "w_up")):
        q, s = (t.cpu() for t in getattr(block, name))
        q, s = q.reshape(rows, -1), s.reshape(-1, rows, 4)
        wq, ws = (t.cpu() for t in block.w8[weight])
        wv = R.values(wq.reshape(E, H, -1), ws.reshape(E, -1, H, 4), d)
        want = torch.cat([xv[a:b] @ wv[e].t() for e, (a, b) in enumerate(zip(ends[:-1], ends[1:]))])
        err = torch.cat([sum_error(xv[a:b], wv[e], exact) for e, (a, b) in enumerate(zip(ends[:-1], ends[1:]))])
        check_packed(q, s, want, err, (shape, exact, name))
        nearest = R.values(*R.pack(want), H)
        off = float((R.values(q, s, H) - nearest).norm() / nearest.norm())
        r = (d + 2) * 2.0 ** -24 if exact else 2.0 ** -11
        assert off <= 0.5 * r ** 0.5, (off, exact)
    # the same bits as the product by itself, with the type of results that says how exact its sums are
    out = B.make_pack_config(rows, H, torch.float32)
    y8, pre8, up8 = (B.alloc_packed_rows(out) for _ in range(3))
    B.etr_packed_linear(B.make_linear_config(rows, d, H, E, torch.float32 if exact else torch.bfloat16, act=B.ACT_SWIGLU), block.hs8, block.offsets, block.w8["w_gate"],
                        w_up8=block.w8["w_up"], y8=y8, pre8=pre8, pre_up8=up8)
    for a, b in ((block.a8, y8), (block.pre8, pre8), (block.pre_up8, up8)):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("shape", SHAPES)
def test_after_a_change_of_the_weights(shape):
    """Refused before the changed weights are packed; then what a new block gives with them."""
    block, new = PackedBlock(shape), PackedBlock(shape)
    w_emb, w = random_weights(shape)
    x, dx_out, dh = inputs(shape)
    block.pack_weights(w)
    block.forward(x, w_emb, w)
    before = block.x_out.clone()
    for name in ("w_gate", "w_up", "w_down"):
        w[name].mul_(-1.5)
    with pytest.raises(RuntimeError, match="w_gate"):
        block.forward(x, w_emb, w)
    for b in (block, new):
        b.pack_weights(w)
        b.forward(x, w_emb, w)
        b.backward(x, w_emb, w, dx_out, dh)
    assert not torch.equal(block.x_out, before)
    for n, v in _outputs(block).items():
        assert torch.equal(v, _outputs(new)[n]), n

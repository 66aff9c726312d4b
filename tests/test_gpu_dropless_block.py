"""The operators around the layer together, as a block that drops nothing: against the block differentiated by torch in 64
bits for the same routing, under a graph, and on another stream."""
import pytest
import torch

from operator_refs import rms, scores
from paper_2406_00023_amd.dropless_block import BlockShape, DroplessBlock, random_weights

pytestmark = pytest.mark.gpu


def _reference(block, x, w_emb, w, dx_out, dh):
    s = block.s
    leaf = {"x": x.cpu().double().requires_grad_(True)}
    leaf.update({n: v.cpu().double().requires_grad_(True) for n, v in w.items()})
    topk = block.topk.cpu().long()
    h = rms(leaf["x"], 1e-5) * leaf["w_pre"]
    gate = torch.softmax(scores(h, w_emb.cpu().double(), s.D, False), 1)
    weight = torch.gather(gate, 1, topk)
    if s.gate_norm:
        weight = weight / weight.sum(1, keepdim=True)
    y = torch.zeros_like(h)
    for e in range(s.E):
        t, j = torch.where(topk == e)
        a, b = h[t] @ leaf["w_gate"][e].t(), h[t] @ leaf["w_up"][e].t()
        y = y.index_add(0, t, weight[t, j][:, None] * ((torch.nn.functional.silu(a) * b) @ leaf["w_down"][e].t()))
    x_out = leaf["x"] + rms(y, 1e-5) * leaf["w_post"]
    h_next = rms(x_out, 1e-5) * leaf["w_next"]
    grads = torch.autograd.grad([x_out, h_next], list(leaf.values()), [dx_out.cpu().double(), dh.cpu().double()])
    return x_out.detach(), h_next.detach(), dict(zip(leaf, grads))


def _off(got, want):
    return float((got.cpu().double() - want).norm() / want.norm())


# relative 2-norms: fp32 sums of up to 1408 terms through seven stages; bf16: about a dozen roundings of half a step (2^-8) at most along a
# path, which add up in squares
TOL = {torch.float32: 2e-5, torch.bfloat16: 2e-2}


@pytest.mark.parametrize("shape", [BlockShape(37, 64, 4, 8, 2, 72, torch.float32), BlockShape(300, 256, 8, 8, 3, 136, torch.float32, gate_norm=1),
                                   BlockShape(1, 256, 8, 8, 2, 128, torch.float32), BlockShape(700, 512, 16, 16, 2, 704, torch.bfloat16),
                                   BlockShape(2000, 512, 4, 16, 2, 1408, torch.bfloat16, gate_norm=1)])
def test_against_64_bits(shape):
    block = DroplessBlock(shape)
    w_emb, w = random_weights(shape)
    g = torch.Generator().manual_seed(3)
    x, dx_out, dh = (torch.randn(shape.T, shape.d, generator=g).to(shape.dtype).cuda() for _ in range(3))
    block.forward(x, w_emb, w)
    block.backward(x, w_emb, w, dx_out, dh)
    torch.cuda.synchronize()
    x_out, h_next, grads = _reference(block, x, w_emb, w, dx_out, dh)
    assert _off(block.x_out, x_out) <= TOL[shape.dtype] and _off(block.h_next, h_next) <= TOL[shape.dtype]
    assert _off(block.dx, grads.pop("x")) <= TOL[shape.dtype]
    for n, want in grads.items():
        assert _off(block.grads[n], want) <= TOL[shape.dtype], n


def _outputs(block):
    return {"x_out": block.x_out, "h_next": block.h_next, "dx": block.dx, "offsets": block.offsets, "row_of": block.row_of, **block.grads}


@pytest.mark.parametrize("shape", [BlockShape(300, 256, 8, 8, 3, 136, torch.float32), BlockShape(2000, 512, 4, 16, 2, 1408, torch.bfloat16)])
def test_graph_replays_match_eager_steps_on_another_stream(shape):
    captured, eager = DroplessBlock(shape), DroplessBlock(shape)
    w_emb, w = random_weights(shape)
    x, dx_out, dh = (torch.randn(shape.T, shape.d, device="cuda").to(shape.dtype) for _ in range(3))

    def step(block):
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
        for v in _outputs(captured).values():
            v.fill_(3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        step(eager)
        torch.cuda.synchronize()
        for n, v in _outputs(captured).items():
            assert torch.equal(v, _outputs(eager)[n]), (rep, n)

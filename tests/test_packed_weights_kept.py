"""Which weights a packed block computes with: those that were packed last, or none.  On the CPU, with the library's calls left out."""
import copy
import gc
import pickle

import pytest
import torch

from paper_2406_00023_amd import binding as B
from paper_2406_00023_amd import dropless_block as D

SHAPE = D.BlockShape(T=4, d=64, E=4, D=8, k=2, H=64, dtype=torch.float32)
EXPERTS = ("w_gate", "w_up", "w_down")


@pytest.fixture
def block(monkeypatch):
    real = D.PackedBlock(SHAPE, device="cpu")
    for name in B.EXPORTS:
        if not name.endswith("_bytes"):
            monkeypatch.setattr(B, name, lambda *a, **k: None, raising=False)
    return real


@pytest.fixture
def weights():
    return D.random_weights(SHAPE, device="cpu")


def forward(block, weights):
    return block.forward(torch.zeros(SHAPE.T, SHAPE.d), *weights)


@pytest.mark.parametrize("name", EXPERTS)
def test_weights_that_changed_in_place_are_refused_until_they_are_packed(block, weights, name):
    w = weights[1]
    block.pack_weights(w)
    forward(block, weights)
    forward(block, weights)
    w[name].mul_(1.5)
    with pytest.raises(RuntimeError, match=name):
        forward(block, weights)
    block.pack_weights(w)
    forward(block, weights)


@pytest.mark.parametrize("name", EXPERTS)
def test_an_optimizers_step_is_seen(block, weights, name):
    w = weights[1]
    block.pack_weights(w)
    leaf = torch.nn.Parameter(w[name])                         # the same memory
    leaf.grad = torch.ones_like(leaf)
    torch.optim.SGD([leaf], lr=0.1).step()
    with pytest.raises(RuntimeError, match=name):
        forward(block, (weights[0], {**w, name: leaf}))


@pytest.mark.parametrize("name", EXPERTS)
def test_other_weights_are_refused(block, weights, name):
    w = weights[1]
    block.pack_weights(w)
    with pytest.raises(RuntimeError, match=name):
        forward(block, (weights[0], {**w, name: w[name].clone()}))
    wide = torch.cat([w[name], w[name] + 1])                   # another part of the same memory
    block.pack_weights({**w, name: wide[:SHAPE.E]})
    with pytest.raises(RuntimeError, match=name):
        forward(block, (weights[0], {**w, name: wide[SHAPE.E:]}))
    # memory that was given back and is somebody else's now
    block.pack_weights({**w, name: w[name].clone()})
    for _ in range(8):
        with pytest.raises(RuntimeError, match=name):
            forward(block, (weights[0], {**w, name: w[name].clone()}))


def test_the_same_weights_are_taken_however_they_come(block, weights):
    w = weights[1]
    block.pack_weights({n: v.view(v.shape) for n, v in w.items()})
    forward(block, (weights[0], {n: v.detach() for n, v in w.items()}))
    w["w_post"].mul_(2.0)                                      # the norms' weights are not packed
    forward(block, weights)
    forward(block, (weights[0], {n: v for n, v in w.items() if n not in EXPERTS}))
    with torch.inference_mode():
        fixed = {n: v.clone() for n, v in w.items()}
    block.pack_weights(fixed)
    forward(block, (weights[0], fixed))


def test_packing_that_failed_leaves_nothing_to_compute_with(block, weights, monkeypatch):
    w = weights[1]
    block.pack_weights(w)

    def fails(*args):
        raise ValueError("strides")

    monkeypatch.setattr(B, "etr_pack_columns", fails)
    with pytest.raises(ValueError):
        block.pack_weights(w)
    with pytest.raises(RuntimeError, match="pack_weights"):
        forward(block, weights)


def test_the_weights_are_not_kept_alive(block, weights):
    w = weights[1]
    block.pack_weights({n: v.clone() for n, v in w.items()})
    gc.collect()
    assert all(block.packed[n].memory() is None for n in EXPERTS)
    norms = {n: v for n, v in w.items() if n not in EXPERTS}
    forward(block, (weights[0], norms))


@pytest.mark.parametrize("copied", [copy.copy, copy.deepcopy, lambda b: pickle.loads(pickle.dumps(b))], ids=["copy", "deepcopy", "pickle"])
def test_copies_have_the_packed_weights(block, weights, copied):
    w = weights[1]
    with pytest.raises(RuntimeError, match="pack_weights"):
        forward(copied(block), weights)
    block.pack_weights(w)
    block.w8["w_gate"][0].fill_(7)
    other = copied(block)
    assert torch.equal(other.w8["w_gate"][0], block.w8["w_gate"][0])
    forward(other, (weights[0], {n: v for n, v in w.items() if n not in EXPERTS}))
    with pytest.raises(RuntimeError, match="w_gate"):          # whose they are it cannot say
        forward(other, weights)
    other.pack_weights(w)
    forward(other, weights)
    forward(block, weights)

"""64-bit definitions of the operators around the layer, in plain torch on the CPU, and the bounds that the tests hold the
kernels to: a rounding to a type is off by half a step at most, and a sum of n terms in 32 bits by n roundings of the sum of
their magnitudes (a tree of sums by fewer)."""
import math

import torch

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U32 = 2.0 ** -24                                   # half a step of fp32


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def randn(seed, *shape, dtype=torch.float32, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(dtype)


def assert_within(got, want, bound, what):
    """|got - want| <= bound element by element (got: a GPU tensor; want, bound: 64 bits)."""
    if want.numel() == 0:
        return
    off = (got.detach().cpu().double() - want).abs()
    assert bool(torch.isfinite(off).all()), what
    worst = float((off - bound).max())
    assert worst <= 0, (what, worst, float(off.max()))


# ---- block norm

def rms(v, eps):
    return v / (v.square().mean(1, keepdim=True) + eps).sqrt()


def join(x, y, gate, w_post, eps, rs, bs):
    p = y if w_post is None else rms(y, eps) * w_post
    return rs * x + bs * (p if gate is None else gate[:, None] * p)


# ---- sorted rows

def sort_tables(topk, E, slot_of=None):
    """Pairs by expert, then by place in the flat list: sorted by Python, one after the other."""
    T, k = topk.shape
    pairs = []
    for t in range(T):
        for j in range(k):
            e = int(topk[t, j])
            if 0 <= e < E and (slot_of is None or int(slot_of[t, e]) >= 0):
                pairs.append((e, t * k + j))
    pairs.sort()
    row_of = torch.full((T * k,), -1, dtype=torch.int32)
    pair_of = torch.full((T * k,), -1, dtype=torch.int32)
    offsets = torch.zeros(E + 1, dtype=torch.int32)
    for r, (e, q) in enumerate(pairs):
        row_of[q], pair_of[r] = r, q
        offsets[e + 1:] += 1
    return offsets, row_of.reshape(T, k), pair_of


def pair_weights(gate, topk, row_of, gate_norm):
    """[T][k], 64 bits, differentiable in gate; 0 where the pair is not in use."""
    used = row_of >= 0
    w = torch.gather(gate, 1, topk.long().clamp(0, gate.shape[1] - 1)) * used
    if gate_norm:
        s = w.sum(1, keepdim=True)
        w = torch.where(s > 0, w / torch.where(s > 0, s, torch.ones_like(s)), torch.zeros_like(w))
    return w


def unsort(ys, w, row_of):
    used = (row_of >= 0)
    rows = ys[row_of.long().clamp(min=0)]
    return (torch.where(used, w, torch.zeros_like(w))[:, :, None] * torch.where(used[:, :, None], rows, torch.zeros_like(rows))).sum(1)


# ---- experts' products

def activation(act, a, b=None):
    if act == "none":
        return a
    if act == "gelu":
        return 0.5 * a * torch.special.erfc(-a / math.sqrt(2.0))
    return a / (1 + torch.exp(-a)) * (1.0 if b is None else b)


# ---- routing

def scores(x, w_emb, D, pooled):
    T, d = x.shape
    g = x.reshape(T, d // D, D).mean(2)
    n = g.norm(dim=1) if pooled else x.norm(dim=1) / math.sqrt(D)
    return g @ w_emb.t() / (n[:, None] * w_emb.norm(dim=1)[None, :])

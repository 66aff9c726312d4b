"""Four operators around and inside an MoE layer, as cases that can be timed and compared.

A case is one pass through the public entry points of the binding, of one of these kinds (`op`):

  norm     etr_block_norm: the residual join after a block and the norm before the next one; with `train` its backward too
  sort     pairs (token, choice) sorted by expert without padding, the rows taken there and the experts' rows brought
           back with their weights (etr_sort_tokens, etr_sort_rows, etr_unsort_rows); with `train` both gradients too
  linear   etr_expert_linear: the experts' products on sorted rows, with bias, activation and residual; with `train` the
           pre-activations are kept, and the backward runs
  route    etr_route_backward: the gradient of the affinities and of their softmax, joined to the one of the experts' path

The sizes are those of the workloads of `paper_2406_00023_amd.inputs`, decode batches on the same layers, and generic
ragged ones.  With `train` a pass is what a stage of a pipeline does in its steady state: the forward of one micro-batch,
and the backward of an earlier one on what its forward has kept (the joined stream, the pre-activations).  The plain forms are elementary torch operations in 32 bits, rounded to the output's type once.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "bf16": 2}
ACTS = {"none": 0, "silu": 1, "gelu": 2, "swiglu": 3}
EPS = 1e-5


def _norm(name, T, d, dtype, *, train=False, block=True, gate=True, post=True, pre=True, residual_scale=1.0, block_scale=1.0):
    """block: a block's output y joins the residual stream; gate: weighted per token; post / pre: normed after / before."""
    return {"name": name, "op": "norm", "T": T, "d": d, "dtype": dtype, "train": train, "block": block, "gate": gate and block,
            "post": post and block, "pre": pre or not block, "residual_scale": residual_scale, "block_scale": block_scale}


def _sort(name, T, d, E, k, dtype, *, train=False, gate_norm=0, bounded=False, skew=0.5):
    """bounded: a selection under a capacity has dropped some of the pairs (slot_of); skew: spread of the experts' popularity."""
    return {"name": name, "op": "sort", "T": T, "d": d, "E": E, "k": k, "dtype": dtype, "train": train, "gate_norm": gate_norm,
            "bounded": bounded, "skew": skew}


def _linear(name, rows, E, K, N, dtype, act, *, train=False, bias=False, residual=False, used=1.0, skew=0.3):
    """used: the share of the rows that belong to an expert at all (the others are dropped pairs' room)."""
    return {"name": name, "op": "linear", "rows": rows, "E": E, "K": K, "N": N, "dtype": dtype, "act": act, "train": train,
            "bias": bias, "residual": residual, "used": used, "skew": skew}


def _route(name, T, d, E, D, dtype, *, pooled=False, add=True):
    return {"name": name, "op": "route", "T": T, "d": d, "E": E, "D": D, "dtype": dtype, "pooled": pooled, "add": add}


def listed():
    return [
        # a decode step of 32 sequences: the join after one block and the norm before the next, bound by the launch
        _norm("norm_decode", 32, 2048, "bf16"),
        # a training step of the 32768-token workload's stream: everything at once, forward and backward
        _norm("norm_train", 32768, 4096, "bf16", train=True, block_scale=0.5),
        # a layer without a norm behind its block and a ragged batch, in the type that gradients are checked in
        _norm("norm_f32_ragged", 3001, 1080, "f32", train=True, gate=False, post=False, residual_scale=0.9),
        # the same decode step: 64 pairs over 16 experts
        _sort("sort_decode", 32, 2048, 16, 2, "bf16"),
        # a training step of the 32-expert workload without a capacity
        _sort("sort_train", 32768, 4096, 32, 2, "bf16", train=True),
        # what a capacity has left, weights renormalised, a ragged batch
        _sort("sort_f32_ragged", 3001, 1080, 12, 3, "f32", train=True, gate_norm=1, bounded=True),
        # the gate and up products of a decode step: every expert's weights for a few rows
        _linear("linear_decode", 64, 16, 2048, 5632, "bf16", "swiglu"),
        # the same products for 8192 tokens, top-2: a prompt or an evaluation pass
        _linear("linear_prompt", 16384, 16, 2048, 5632, "bf16", "swiglu"),
        # the down products of a training step, with a bias
        _linear("linear_train", 16384, 16, 5632, 2048, "bf16", "none", train=True, bias=True),
        # a small fp32 layer with everything in the epilogue and rows that belong to nobody
        _linear("linear_f32_ragged", 2501, 8, 520, 1048, "f32", "gelu", train=True, bias=True, residual=True, used=0.9),
        # the small fp32 layer's router, and that of 65536 tokens over 64 experts
        _route("route_small", 512, 256, 8, 8, "f32"),
        _route("route_64", 65536, 4096, 64, 64, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random):
    """A case of the same ranges: from one token to 65536, widths up to 8192, up to 64 experts, both types, both directions."""
    while True:
        op = rng.choice(["norm", "norm", "sort", "sort", "linear", "linear", "linear", "route"])
        dtype = "f32" if rng.random() < 0.3 else "bf16"
        train = rng.random() < 0.5
        d = _log_int(rng, 128, 8192) // 8 * 8
        if rng.random() < 0.5:
            d = d // 64 * 64                                   # most layers have widths of whole 64s
        if op == "norm":
            c = _norm("", _log_int(rng, 1, 65536), d, dtype, train=train, block=rng.random() < 0.8, gate=rng.random() < 0.5,
                      post=rng.random() < 0.5, pre=rng.random() < 0.8, residual_scale=rng.choice([1.0, 1.0, 0.7]),
                      block_scale=rng.choice([1.0, 0.5]))
            if c["T"] * d > 32768 * 4096:
                continue
        elif op == "sort":
            E = rng.choice([1, 4, 8, 12, 16, 32, 64])
            k = rng.randint(1, min(E, 8))
            c = _sort("", _log_int(rng, 1, 65536), d, E, k, dtype, train=train, gate_norm=int(rng.random() < 0.4),
                      bounded=rng.random() < 0.4, skew=rng.uniform(0.0, 1.0))
            if c["T"] * (k + 1) * d * SIZES[dtype] > 32768 * 3 * 4096 * 2:
                continue
        elif op == "linear":
            K, N = _log_int(rng, 128, 8192) // 8 * 8, _log_int(rng, 128, 8192) // 8 * 8
            if rng.random() < 0.6:
                K, N = max(128, K // 64 * 64), max(128, N // 64 * 64)
            c = _linear("", _log_int(rng, 1, 32768), rng.choice([1, 4, 8, 12, 16, 32, 64]), K, N, dtype, rng.choice(list(ACTS)),
                        train=train, bias=rng.random() < 0.6, residual=rng.random() < 0.3, used=rng.choice([1.0, 1.0, 0.8]),
                        skew=rng.uniform(0.0, 0.6))
            if c["E"] * K * N > 2e8 or work(c)["flops"] > (2e11 if dtype == "f32" else 1.1e12):
                continue
        else:
            D = rng.choice([8, 16, 32, 64])
            d = d // (8 * D) * (8 * D)
            if d < 8 * D:
                continue
            E = rng.choice([e for e in (4, 8, 12, 16, 32, 64) if e <= d // D])
            c = _route("", _log_int(rng, 1, 65536), d, E, D, dtype, pooled=rng.random() < 0.4, add=rng.random() < 0.7)
            if c["T"] * d > 65536 * 4096 or E * (d // D) * 4 > 120 * 1024:
                continue
        del c["name"]
        return c


# ---- inputs -----------------------------------------------------------------------------------------------------

def _generator(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + 17) % (1 << 62))
    return g


def _normal(g, shape, dtype=torch.float32, std=1.0):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).mul_(std).to(dtype)


def _prepare_norm(case, seed):
    g, T, d, dt = _generator(case, seed), case["T"], case["d"], DTYPES[case["dtype"]]
    s = {"x": _normal(g, (T, d), dt, 2.0), "x_out": None, "h": None, "y": None, "gate": None, "w_post": None, "w_pre": None}
    if case["block"]:
        s.update(y=_normal(g, (T, d), dt, 0.7), x_out=torch.zeros(T, d, dtype=dt, device=DEV))
        if case["gate"]:
            s["gate"] = torch.sigmoid(_normal(g, (T,)))
        if case["post"]:
            s["w_post"] = 1.0 + _normal(g, (d,), std=0.1)
    if case["pre"]:
        s.update(w_pre=1.0 + _normal(g, (d,), std=0.1), h=torch.zeros(T, d, dtype=dt, device=DEV))
    if case["train"]:
        # what an earlier forward has kept, and the gradients from above: along the stream, and out of the next block
        s.update(kept=_normal(g, (T, d), dt, 2.0) if case["block"] else s["x"],
                 dx_out=_normal(g, (T, d), dt, 0.01),
                 dh=_normal(g, (T, d), dt, 0.01) if case["pre"] else None,
                 dx=torch.zeros(T, d, dtype=dt, device=DEV), dy=torch.zeros(T, d, dtype=dt, device=DEV) if case["block"] else None,
                 dgate=torch.zeros(T, device=DEV) if case["gate"] else None,
                 dw_post=torch.zeros(d, device=DEV) if case["post"] else None,
                 dw_pre=torch.zeros(d, device=DEV) if case["pre"] else None)
    return s


def _prepare_sort(case, seed):
    g, T, d, E, k, dt = _generator(case, seed), case["T"], case["d"], case["E"], case["k"], DTYPES[case["dtype"]]
    logits = _normal(g, (T, E)) + case["skew"] * _normal(g, (E,))          # some experts are more popular than others
    s = {"gate": torch.softmax(logits, 1).contiguous(), "topk": torch.topk(logits, k, dim=1)[1].to(torch.int32).contiguous()}
    s["slot_of"] = None
    if case["bounded"]:
        kept = torch.rand((T, E), generator=g, device=DEV) < 0.85
        s["slot_of"] = torch.where(kept, torch.arange(T, device=DEV, dtype=torch.int32)[:, None], -1).to(torch.int32).contiguous()
    s.update(x=_normal(g, (T, d), dt), ys=_normal(g, (T * k, d), dt), xs=torch.zeros(T * k, d, dtype=dt, device=DEV),
             out=torch.zeros(T, d, dtype=dt, device=DEV), offsets=torch.zeros(E + 1, dtype=torch.int32, device=DEV),
             row_of=torch.zeros(T, k, dtype=torch.int32, device=DEV), pair_of=torch.zeros(T * k, dtype=torch.int32, device=DEV))
    if case["train"]:
        s.update(dout=_normal(g, (T, d), dt, 0.01), dxs=_normal(g, (T * k, d), dt, 0.01), dx=torch.zeros(T, d, dtype=dt, device=DEV),
                 dys=torch.zeros(T * k, d, dtype=dt, device=DEV), dgate=torch.zeros(T, E, device=DEV))
    return s


def _prepare_linear(case, seed):
    g, R, E, K, N, dt = _generator(case, seed), case["rows"], case["E"], case["K"], case["N"], DTYPES[case["dtype"]]
    # rows of each expert: shares of unlike popularity, whole numbers that add up to the rows in use
    rng = random.Random(int(seed) * 7919 + 3)
    used = max(1, int(R * case["used"])) if case["used"] < 1.0 else R
    shares = [math.exp(rng.gauss(0.0, case["skew"])) for _ in range(E)]
    ends = [int(used * sum(shares[: e + 1]) / sum(shares)) for e in range(E)]
    ends[-1] = used
    counts = [b - a for a, b in zip([0] + ends, ends)]
    glu = case["act"] == "swiglu"
    std = K ** -0.5
    s = {"offsets": torch.tensor([0] + ends, dtype=torch.int32, device=DEV), "most": max(counts),
         "x": _normal(g, (R, K), dt), "w": _normal(g, (E, N, K), dt, std), "w_up": _normal(g, (E, N, K), dt, std) if glu else None,
         "bias": _normal(g, (E, N), std=0.2) if case["bias"] else None,
         "bias_up": _normal(g, (E, N), std=0.2) if case["bias"] and glu else None,
         "residual": _normal(g, (R, N), dt) if case["residual"] else None, "y": torch.zeros(R, N, dtype=dt, device=DEV)}
    keep = case["train"] and case["act"] != "none"
    s.update(pre=torch.zeros(R, N, dtype=dt, device=DEV) if keep else None,
             pre_up=torch.zeros(R, N, dtype=dt, device=DEV) if keep and glu else None)
    if case["train"]:
        s.update(pre_kept=_normal(g, (R, N), dt) if keep else None, pre_up_kept=_normal(g, (R, N), dt) if keep and glu else None,
                 dy=_normal(g, (R, N), dt, 0.01), dx=torch.zeros(R, K, dtype=dt, device=DEV), dw=torch.zeros(E, N, K, dtype=dt, device=DEV),
                 dw_up=torch.zeros(E, N, K, dtype=dt, device=DEV) if glu else None,
                 dbias=torch.zeros(E, N, device=DEV) if case["bias"] else None,
                 dbias_up=torch.zeros(E, N, device=DEV) if case["bias"] and glu else None)
    return s


def _prepare_route(case, seed):
    g, T, d, E, D, dt = _generator(case, seed), case["T"], case["d"], case["E"], case["D"], DTYPES[case["dtype"]]
    P = d // D
    q = torch.linalg.qr(torch.randn((P, E), generator=g, device=DEV, dtype=torch.float32))[0]
    w_emb = q.t().contiguous()                                 # orthonormal rows
    # tokens near their expert's direction, as after training
    x = _normal(g, (T, d)) + 0.5 * math.sqrt(D) * torch.repeat_interleave(w_emb[torch.randint(0, E, (T,), generator=g, device=DEV)], D, dim=1)
    x = x.to(dt).contiguous()
    score = _scores(case, x.float(), w_emb).contiguous()
    return {"x": x, "w_emb": w_emb, "score": score, "gate": torch.softmax(score, 1).contiguous(), "dgate": _normal(g, (T, E), std=0.1),
            "dx_add": _normal(g, (T, d), dt, 0.01) if case["add"] else None, "dx": torch.zeros(T, d, dtype=dt, device=DEV)}


def _scores(case, x, w_emb):
    """Cosine of token and expert embedding on the mean-pooled features, in the token's own norm or the pooled one."""
    T, d, D = case["T"], case["d"], case["D"]
    pooled = x.reshape(T, d // D, D).mean(2)
    length = pooled.square().sum(1).sqrt() if case["pooled"] else x.square().sum(1).sqrt() / math.sqrt(D)
    return (pooled @ w_emb.t()) / (length[:, None] * w_emb.square().sum(1).sqrt()[None, :])


def prepare(case, seed):
    """Inputs, weights and output buffers, as a program that calls the operator again and again keeps them."""
    s = {"norm": _prepare_norm, "sort": _prepare_sort, "linear": _prepare_linear, "route": _prepare_route}[case["op"]](case, seed)
    s["case"] = case
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------

def run(s):
    return {"norm": (_plain_norm, _own_norm), "sort": (_plain_sort, _own_sort), "linear": (_plain_linear, _own_linear),
            "route": (_plain_route, _own_route)}[s["case"]["op"]][1 if own else 0](s)


def _present(s, names):
    return {n: s[n] for n in names if s.get(n) is not None}


def _rms_inverse(v):
    return torch.rsqrt(v.square().mean(1, keepdim=True) + EPS)


def _rms_backward(u, v, inv):
    """Gradient of <u, v inv(v)> with respect to v."""
    return inv * (u - v * (inv * inv) * (u * v).mean(1, keepdim=True))


def _plain_norm(s):
    c, dt, r = s["case"], s["x"].dtype, {}
    rs, bs = c["residual_scale"], c["block_scale"]
    stream = s["x"].float()
    if c["block"]:
        y = s["y"].float()
        inv_y = _rms_inverse(y) if c["post"] else None
        normed = y * inv_y * s["w_post"] if c["post"] else y
        weight = bs * s["gate"][:, None] if c["gate"] else bs
        r["x_out"] = (rs * stream + weight * normed).to(dt)
        stream = r["x_out"].float()
    if c["pre"]:
        r["h"] = (stream * _rms_inverse(stream) * s["w_pre"]).to(dt)
    if not c["train"]:
        return r
    grad = s["dx_out"].float()
    if c["pre"]:
        dh, stream = s["dh"].float(), s["kept"].float()
        inv = _rms_inverse(stream)
        r["dw_pre"] = (dh * stream * inv).sum(0)
        grad = grad + _rms_backward(dh * s["w_pre"], stream, inv)
    if not c["block"]:
        r["dx"] = grad.to(dt)
        return r
    r["dx"] = (rs * grad).to(dt)
    if c["gate"]:
        r["dgate"] = bs * (grad * normed).sum(1)
    up = weight * grad
    if c["post"]:
        r["dw_post"] = (up * y * inv_y).sum(0)
        up = _rms_backward(up * s["w_post"], y, inv_y)
    r["dy"] = up.to(dt)
    return r


def _own_norm(s):
    from paper_2406_00023_amd import binding as B
    c = s["case"]
    if "cfg" not in s:
        s["cfg"] = B.make_norm_config(c["T"], c["d"], s["x"].dtype, eps=EPS, residual_scale=c["residual_scale"], block_scale=c["block_scale"])
        if c["train"]:
            s["ws"] = B.alloc_workspace(B.etr_norm_workspace_bytes(s["cfg"]), DEV)
    B.etr_block_norm(s["cfg"], s["x"], s["y"], s["gate"], s["w_post"], s["w_pre"], s["x_out"], s["h"])
    if c["train"]:
        B.etr_block_norm_backward(s["cfg"], s["kept"], s["y"], s["gate"], s["w_post"], s["w_pre"], s["dx_out"], s["dh"], s["dx"], s["dy"],
                                  s["dgate"], s["dw_post"], s["dw_pre"], s["ws"])
    return _present(s, ("x_out", "h", "dx", "dy", "dgate", "dw_post", "dw_pre"))


def _plain_sort(s):
    c, dt = s["case"], s["x"].dtype
    T, E, k, d = c["T"], c["E"], c["k"], c["d"]
    topk = s["topk"].long()
    kept = torch.ones_like(topk, dtype=torch.bool) if s["slot_of"] is None else s["slot_of"].gather(1, topk) >= 0
    one_hot = (topk.reshape(-1, 1) == torch.arange(E, device=DEV)) & kept.reshape(-1, 1)          # [pair][expert]
    before = one_hot.cumsum(0)
    counts = before[-1]
    ends = counts.cumsum(0)
    offsets = torch.cat([ends.new_zeros(1), ends])
    row = (ends - counts)[topk.reshape(-1)] + before.gather(1, topk.reshape(-1, 1)).squeeze(1) - 1
    flat = kept.reshape(-1)
    row_of = torch.where(flat, row, -1)
    at = torch.where(flat, row, T * k)                         # a row of its own for what is not kept
    pair_of = torch.full((T * k + 1,), -1, dtype=torch.int64, device=DEV).scatter(0, at, torch.arange(T * k, device=DEV))[: T * k]
    live = (pair_of >= 0)[:, None]
    source = pair_of.clamp(min=0)
    xs = torch.where(live, s["x"][source // k], torch.zeros((), dtype=dt, device=DEV))
    weight = torch.where(kept, s["gate"].gather(1, topk), 0.0)
    total = weight.sum(1, keepdim=True)
    if c["gate_norm"]:
        scale = torch.where(total > 0, 1.0 / torch.where(total > 0, total, 1.0), 0.0)
        weight = weight * scale
    taken = row_of.clamp(min=0).reshape(T, k)
    ys = torch.where(kept[:, :, None], s["ys"][taken].float(), 0.0)
    out = (weight[:, :, None] * ys).sum(1).to(dt)
    r = {"offsets": offsets.int(), "row_of": row_of.int().reshape(T, k), "pair_of": pair_of.int(), "xs": xs, "out": out}
    if not c["train"]:
        return r
    r["dx"] = torch.where(kept[:, :, None], s["dxs"][taken].float(), 0.0).sum(1).to(dt)
    dout = s["dout"].float()
    dweight = torch.where(kept, (dout[:, None, :] * ys).sum(2), 0.0)
    del ys
    r["dys"] = torch.where(live, weight.reshape(-1)[source][:, None] * dout[source // k], 0.0).to(dt)
    if c["gate_norm"]:
        dweight = torch.where(kept, scale * (dweight - (dweight * weight).sum(1, keepdim=True)), 0.0)
    r["dgate"] = torch.zeros(T, E, device=DEV).scatter_add_(1, topk, dweight)
    return r


def _own_sort(s):
    from paper_2406_00023_amd import binding as B
    c = s["case"]
    if "cfg" not in s:
        s["cfg"] = B.make_sort_config(c["T"], c["k"], c["E"], c["d"], s["x"].dtype, gate_norm=c["gate_norm"])
        s["ws"] = B.alloc_workspace(B.etr_sort_workspace_bytes(s["cfg"]), DEV)
    B.etr_sort_tokens(s["cfg"], s["topk"], s["slot_of"], s["offsets"], s["row_of"], s["pair_of"], s["ws"])
    B.etr_sort_rows(s["cfg"], s["x"], s["row_of"], s["xs"])
    B.etr_unsort_rows(s["cfg"], s["ys"], s["gate"], s["topk"], s["row_of"], s["out"])
    if c["train"]:
        B.etr_unsort_rows_backward(s["cfg"], s["dout"], s["ys"], s["gate"], s["topk"], s["row_of"], s["dys"], s["dgate"])
        B.etr_sort_rows_backward(s["cfg"], s["dxs"], s["row_of"], s["dx"])
    return _present(s, ("offsets", "row_of", "pair_of", "xs", "out", "dx", "dys", "dgate"))


def _activation(act, a, b):
    if act == "none":
        return a
    if act == "gelu":
        return 0.5 * a * (1.0 + torch.erf(a * math.sqrt(0.5)))
    h = a * torch.sigmoid(a)
    return h * b if act == "swiglu" else h


def _plain_linear(s):
    c, dt = s["case"], s["x"].dtype
    R, E, K, N, act = c["rows"], c["E"], c["K"], c["N"], c["act"]
    glu = act == "swiglu"
    # rows laid out by expert, as many for each as the fullest has, so that the products are one batch
    offsets = s["offsets"].long()
    place = torch.arange(s["most"], device=DEV)[None, :]
    at = offsets[:-1, None] + place
    live = at < offsets[1:, None]
    source = torch.where(live, at, 0).reshape(-1)
    target = torch.where(live, at, R).reshape(-1)              # one row more takes what is no row

    def spread(v):
        return torch.where(live.reshape(-1, 1), v[source].float(), 0.0).reshape(E, s["most"], v.shape[1])

    def rows(v):
        out = torch.zeros(R + 1, v.shape[2], device=DEV)
        out[target] = v.reshape(-1, v.shape[2])
        return out[:R].to(dt)

    x = spread(s["x"])
    a = torch.bmm(x, s["w"].float().transpose(1, 2).contiguous())
    b = torch.bmm(x, s["w_up"].float().transpose(1, 2).contiguous()) if glu else None
    if c["bias"]:
        a = a + s["bias"][:, None, :]
        b = b + s["bias_up"][:, None, :] if glu else None
    y = _activation(act, a, b)
    r = {"y": rows(y + spread(s["residual"]) if c["residual"] else y)}
    if not c["train"]:
        return r
    da = spread(s["dy"])
    db = None
    if act != "none":
        r["pre"] = rows(a)
        a = spread(s["pre_kept"])
        sig = torch.sigmoid(a)
        if act == "gelu":
            da = da * (0.5 * (1.0 + torch.erf(a * math.sqrt(0.5))) + a * torch.exp(-0.5 * a * a) / math.sqrt(2.0 * math.pi))
        else:
            if glu:
                r["pre_up"] = rows(b)
                db = da * a * sig
                da = da * spread(s["pre_up_kept"])
            da = da * sig * (1.0 + a * (1.0 - sig))
    dx = torch.bmm(da, s["w"].float())
    r["dw"] = torch.bmm(da.transpose(1, 2).contiguous(), x).to(dt)
    if glu:
        dx = dx + torch.bmm(db, s["w_up"].float())
        r["dw_up"] = torch.bmm(db.transpose(1, 2).contiguous(), x).to(dt)
    r["dx"] = rows(dx)
    if c["bias"]:
        r["dbias"] = da.sum(1)
        if glu:
            r["dbias_up"] = db.sum(1)
    return r


def _own_linear(s):
    from paper_2406_00023_amd import binding as B
    c = s["case"]
    if "cfg" not in s:
        s["cfg"] = B.make_linear_config(c["rows"], c["K"], c["N"], c["E"], s["x"].dtype, act=ACTS[c["act"]])
        if c["train"]:
            s["ws"] = B.alloc_workspace(B.etr_linear_workspace_bytes(s["cfg"]), DEV)
    B.etr_expert_linear(s["cfg"], s["x"], s["offsets"], s["w"], s["y"], w_up=s["w_up"], bias=s["bias"], bias_up=s["bias_up"],
                        residual=s["residual"], pre=s["pre"], pre_up=s["pre_up"])
    if c["train"]:
        B.etr_expert_linear_backward(s["cfg"], s["x"], s["offsets"], s["w"], s["dy"], s["ws"], w_up=s["w_up"], pre=s["pre_kept"],
                                     pre_up=s["pre_up_kept"], dx=s["dx"], dw=s["dw"], dw_up=s["dw_up"], dbias=s["dbias"], dbias_up=s["dbias_up"])
    return _present(s, ("y", "pre", "pre_up", "dx", "dw", "dw_up", "dbias", "dbias_up"))


def _plain_route(s):
    c, dt = s["case"], s["x"].dtype
    T, d, D = c["T"], c["d"], c["D"]
    x, w = s["x"].float(), s["w_emb"]
    dscore = s["gate"] * (s["dgate"] - (s["dgate"] * s["gate"]).sum(1, keepdim=True))
    unit = w / w.square().sum(1, keepdim=True).sqrt()
    along = (dscore * s["score"]).sum(1, keepdim=True)
    pooled = x.reshape(T, d // D, D).mean(2)
    if c["pooled"]:
        square = pooled.square().sum(1, keepdim=True)
        grad = torch.where(square > 0, (dscore @ unit) * torch.rsqrt(square) - along * pooled / square, 0.0)
        dx = (grad / D).repeat_interleave(D, dim=1)
    else:
        square = x.square().sum(1, keepdim=True)
        dx = ((dscore @ unit) * torch.rsqrt(square) / math.sqrt(D)).repeat_interleave(D, dim=1) - along * x / square
        dx = torch.where(square > 0, dx, 0.0)
    if c["add"]:
        dx = dx + s["dx_add"].float()
    return {"dx": dx.to(dt)}


def _own_route(s):
    from paper_2406_00023_amd import binding as B
    from paper_2406_00023_amd import inputs as I
    c = s["case"]
    if "cfg" not in s:
        s["cfg"] = B.EtrConfig(c["T"], c["d"], c["E"], c["D"], 1, 1, 8, I.DT_F32 if c["dtype"] == "f32" else I.DT_BF16, I.MODE_BIDIR,
                               I.COS_POOLED if c["pooled"] else I.COS_FULL, 0)
    B.etr_route_backward(s["cfg"], s["x"], s["w_emb"], s["score"], s["gate"], s["dgate"], s["dx_add"], s["dx"])
    return {"dx": s["dx"]}


# ---- what a pass cannot do without ------------------------------------------------------------------------------

def work(case):
    c, el = case, SIZES[case["dtype"]]
    if c["op"] == "norm":
        row = c["T"] * c["d"] * el
        streams = 1 + 2 * c["block"] + c["pre"]                # x (and y in, the joined stream out), the next block's input
        if c["train"]:
            # dx_out in and dx out; dh in; dy out; what the earlier forward has kept (x itself where no block joins)
            streams += 2 + c["pre"] + c["block"] + (c["pre"] and c["block"])
        return {"bytes": streams * row + 4 * c["d"] * (c["pre"] + c["post"]), "flops": 10.0 * c["T"] * c["d"]}
    if c["op"] == "sort":
        T, k, E = c["T"], c["k"], c["E"]
        token, pairs = T * c["d"] * el, T * k * c["d"] * el * (0.85 if c["bounded"] else 1.0)
        tables = 12 * T * k + 4 * T * k + (4 * T * k if c["bounded"] else 0)
        nbytes, flops = 2 * token + 2 * pairs + tables, 2.0 * T * k * c["d"]
        if c["train"]:
            nbytes += 2 * token + 2 * pairs + 4 * T * E        # dout in, dys out, dxs in, dx out; ys is read already
            flops *= 3
        return {"bytes": nbytes, "flops": flops}
    if c["op"] == "linear":
        R, E, K, N = int(c["rows"] * c["used"]), c["E"], c["K"], c["N"]
        n = 2 if c["act"] == "swiglu" else 1
        live = min(E, max(1, R))
        weights, rows_in, rows_out = n * live * K * N * el, R * K * el, R * N * el
        nbytes = weights + rows_in + rows_out * (1 + c["residual"]) + 4 * n * E * N * c["bias"]
        flops = 2.0 * n * R * K * N
        if c["train"]:
            nbytes += rows_out + rows_in + n * E * K * N * el + 2 * rows_out * (n if c["act"] != "none" else 0)
            flops *= 3
        return {"bytes": nbytes, "flops": flops}
    row = c["T"] * c["d"] * el
    return {"bytes": (2 + c["add"]) * row + 12 * c["T"] * c["E"] + 4 * c["E"] * (c["d"] // c["D"]),
            "flops": 2.0 * c["T"] * c["E"] * (c["d"] // c["D"]) + 4.0 * c["T"] * c["d"]}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "sort": _exact_sort, "linear": _exact_linear, "route": _exact_route}[case["op"]](s)


def _chunks(n, width):
    step = max(1, (1 << 27) // max(1, width))
    return [slice(i, min(n, i + step)) for i in range(0, n, step)]


def _exact_norm(s):
    """Differentiated by torch in 64 bits, a part of the rows at a time."""
    c, dt = s["case"], s["x"].dtype
    parts, sums = {}, {}

    def normed(v):
        return v / (v.pow(2).mean(1, keepdim=True) + EPS).sqrt()

    def join(part, v):
        v = normed(v) * part["w_post"] if c["post"] else v
        return c["block_scale"] * (v * part["gate"].unsqueeze(1) if c["gate"] else v)

    for sl in _chunks(c["T"], 8 * c["d"]):
        leaf = {n: s[n][sl].double() for n in ("y", "gate") if s[n] is not None}
        leaf.update({n: s[n].double() for n in ("w_post", "w_pre") if s[n] is not None})
        got, stream = {}, s["x"][sl].double()
        if c["block"]:
            got["x_out"] = c["residual_scale"] * stream + join(leaf, leaf["y"])
            stream = got["x_out"].float().to(dt).double()      # the next norm reads the stream as it is stored
        if c["pre"]:
            got["h"] = normed(stream) * leaf["w_pre"]
        if c["train"]:
            leaf = {n: v.requires_grad_(True) for n, v in leaf.items()}
            kept = s["kept"][sl].double().requires_grad_(True)
            up = s["dx_out"][sl].double()                      # of the stream behind the join
            if c["pre"]:
                a, leaf_grad = torch.autograd.grad(normed(kept) * leaf["w_pre"], [kept, leaf["w_pre"]], s["dh"][sl].double())
                up = up + a
                sums["dw_pre"] = sums.get("dw_pre", 0.0) + leaf_grad
            got["dx"] = c["residual_scale"] * up if c["block"] else up
            names = [n for n in ("y", "gate", "w_post") if n in leaf]
            if c["block"]:
                for n, v in zip(names, torch.autograd.grad(join(leaf, leaf["y"]), [leaf[n] for n in names], up)):
                    if n == "w_post":
                        sums["dw_post"] = sums.get("dw_post", 0.0) + v
                    else:
                        got["d" + n] = v
        for n, v in got.items():
            parts.setdefault(n, []).append(v.detach())
    return {**{n: torch.cat(v) for n, v in parts.items()}, **sums}


def _exact_sort(s):
    c = s["case"]
    T, E, k, d = c["T"], c["E"], c["k"], c["d"]
    topk = s["topk"].long()
    kept = torch.ones_like(topk, dtype=torch.bool)
    if s["slot_of"] is not None:
        kept = torch.gather(s["slot_of"], 1, topk) >= 0
    key = torch.where(kept, topk, E).reshape(-1)
    key, order = torch.sort(key, stable=True)                  # pairs in their final order, those not kept last
    n = int(kept.sum())
    pair_of = torch.full((T * k,), -1, dtype=torch.int64, device=DEV)
    pair_of[:n] = order[:n]
    row_of = torch.full((T * k,), -1, dtype=torch.int64, device=DEV)
    row_of[order[:n]] = torch.arange(n, device=DEV)
    offsets = torch.searchsorted(key, torch.arange(E + 1, device=DEV))
    xs = torch.zeros(T * k, d, dtype=torch.float64, device=DEV)
    for sl in _chunks(n, d):
        xs[sl] = s["x"][pair_of[sl] // k].double()
    row_of = row_of.reshape(T, k)
    weight = (torch.gather(s["gate"], 1, topk).double() * kept).requires_grad_(c["train"])
    w = weight / weight.sum(1, keepdim=True).clamp_min(1e-300) if c["gate_norm"] else weight
    wd = w.detach()
    out, dx, dw = torch.zeros(T, d, dtype=torch.float64, device=DEV), torch.zeros(T, d, dtype=torch.float64, device=DEV), torch.zeros_like(wd)
    dys = torch.zeros(T * k, d, dtype=torch.float64, device=DEV) if c["train"] else None
    for j in range(k):
        t = kept[:, j].nonzero().squeeze(1)
        for sl in _chunks(t.numel(), d):
            tt = t[sl]
            rows, y = row_of[tt, j], s["ys"][row_of[tt, j]].double()
            out[tt] += wd[tt, j].unsqueeze(1) * y
            if c["train"]:
                go = s["dout"][tt].double()
                dw[tt, j] = (go * y).sum(1)
                dys[rows] = wd[tt, j].unsqueeze(1) * go
                dx[tt] += s["dxs"][rows].double()
    r = {"offsets": offsets.int(), "row_of": row_of.int(), "pair_of": pair_of.int(), "xs": xs, "out": out}
    if c["train"]:
        grad = torch.autograd.grad(w, weight, dw)[0] * kept
        r.update(dx=dx, dys=dys, dgate=torch.zeros(T, E, dtype=torch.float64, device=DEV).scatter_add_(1, topk, grad))
    return r


def _exact_linear(s):
    c = s["case"]
    R, E, K, N, act = c["rows"], c["E"], c["K"], c["N"], c["act"]
    if work(c)["flops"] > 4e13:
        return None
    glu, train = act == "swiglu", c["train"]
    ends = s["offsets"].tolist()

    def zeros(*n):
        return torch.zeros(*n, dtype=torch.float64, device=DEV)

    r = {"y": zeros(R, N)}
    if train:
        r.update(dx=zeros(R, K), dw=zeros(E, N, K))
        if glu:
            r["dw_up"] = zeros(E, N, K)
        if act != "none":
            r["pre"] = zeros(R, N)
            if glu:
                r["pre_up"] = zeros(R, N)
        if c["bias"]:
            r["dbias"] = zeros(E, N)
            if glu:
                r["dbias_up"] = zeros(E, N)
    for e in range(E):
        rows = slice(ends[e], ends[e + 1])
        if ends[e] == ends[e + 1]:
            continue
        x, wt = s["x"][rows].double(), s["w"][e].double()
        a = x @ wt.t() + (s["bias"][e].double() if c["bias"] else 0.0)
        b = None
        if glu:
            wu = s["w_up"][e].double()
            b = x @ wu.t() + (s["bias_up"][e].double() if c["bias"] else 0.0)
        r["y"][rows] = _activation(act, a, b) + (s["residual"][rows].double() if c["residual"] else 0.0)
        if not train:
            continue
        dy = s["dy"][rows].double()
        if act == "none":
            da, db = dy, None
        else:
            r["pre"][rows] = a
            leaf = [s["pre_kept"][rows].double().requires_grad_(True)]
            if glu:
                r["pre_up"][rows] = b
                leaf.append(s["pre_up_kept"][rows].double().requires_grad_(True))
            grads = torch.autograd.grad(_activation(act, leaf[0], leaf[1] if glu else None), leaf, dy)
            da, db = grads[0], grads[1] if glu else None
        r["dx"][rows] = da @ wt
        r["dw"][e] = da.t().contiguous() @ x
        if glu:
            r["dx"][rows] += db @ wu
            r["dw_up"][e] = db.t().contiguous() @ x
        if c["bias"]:
            r["dbias"][e] = da.sum(0)
            if glu:
                r["dbias_up"][e] = db.sum(0)
    return r


def _exact_route(s):
    """The forward scores of the tokens differentiated by torch in 64 bits; the gate and the scores that the operator is
    given stand for those of the forward call."""
    c = s["case"]
    w = s["w_emb"].double()
    parts = []
    for sl in _chunks(c["T"], 8 * c["d"]):
        x = s["x"][sl].double().requires_grad_(True)
        score = _scores({**c, "T": x.shape[0]}, x, w)
        gate, dgate = s["gate"][sl].double(), s["dgate"][sl].double()
        dscore = gate * (dgate - (dgate * gate).sum(1, keepdim=True))
        dx = torch.autograd.grad(score, x, dscore)[0]
        parts.append(dx + s["dx_add"][sl].double() if c["add"] else dx)
    return {"dx": torch.cat(parts)}

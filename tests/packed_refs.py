"""64-bit definitions of packed matrices, in plain torch on the CPU: e4m3 values with a power of two for each block of 128, laid out as the header
says.  Rounding goes by a table of the 127 magnitudes, powers by frexp: nothing of it is the kernels' way."""
import math

import torch

BLOCK = 128


def blocks(n):
    return -(-n // BLOCK)


def magnitudes():
    return torch.tensor([(m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)) for e in range(16) for m in range(8)][:127], dtype=torch.float64)


def code(v):
    """Bytes of the nearest e4m3 values, ties to the even byte, NaN for what is not finite."""
    table = magnitudes()
    a = v.abs().nan_to_num(nan=0.0, posinf=0.0)
    hi = torch.searchsorted(table, a).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    up, down = table[hi] - a, a - table[lo]
    q = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    q = torch.where(torch.isfinite(v), q, torch.full_like(q, 127))
    return (q + 128 * torch.signbit(v)).to(torch.uint8)


def decode(q):
    v = torch.cat([magnitudes(), torch.tensor([math.nan], dtype=torch.float64)])
    return torch.cat([v, -v])[q.long()]


def scale_bytes(top):
    """top: largest magnitudes (64 bits).  448 = 0.875 * 2^9."""
    m, e = torch.frexp(top)
    return torch.where(top > 0, e - 9 + (m > 0.875).int() + 127, torch.zeros_like(e)).clamp(min=0)


def pack_blocks(x):
    """x [..., rows, K] in 64 bits: codes [..., rows, blocks * 128] and scale bytes [..., rows, blocks]."""
    K = x.shape[-1]
    v = torch.nn.functional.pad(x, (0, blocks(K) * BLOCK - K)).unflatten(-1, (-1, BLOCK))
    s = scale_bytes(torch.where(torch.isfinite(v), v.abs(), torch.zeros_like(v)).amax(-1))
    return code(v / torch.exp2(s.double() - 127)[..., None]).flatten(-2), s.to(torch.uint8)


def layout(s):
    """Scale bytes [rows][blocks] as the header lays them out: [groups][rows][4]."""
    s = torch.nn.functional.pad(s, (0, -s.shape[-1] % 4), value=127)
    return s.unflatten(-1, (-1, 4)).transpose(-3, -2).contiguous()


def unlayout(s, n):
    """Back, the first n blocks: [..., rows, n]."""
    return s.transpose(-3, -2).flatten(-2)[..., :n]


def pack(x):
    q, s = pack_blocks(x)
    return q, layout(s)


def values(q, s, K):
    """What codes [..., rows, Kp] and scales [..., groups, rows, 4] stand for."""
    power = torch.exp2(unlayout(s, q.shape[-1] // BLOCK).double() - 127)
    return (decode(q).unflatten(-1, (-1, BLOCK)) * power[..., None]).flatten(-2)[..., :K]


def pack_columns(x, offsets):
    """Every expert's rows along columns, one behind the other: flat codes and flat scales."""
    q, s = [], []
    for a, b in zip(offsets[:-1], offsets[1:]):
        if b > a:
            cq, cs = pack(x[a:b].t().contiguous())
            q.append(cq.reshape(-1))
            s.append(cs.reshape(-1))
    return torch.cat(q) if q else torch.zeros(0, dtype=torch.uint8), torch.cat(s) if s else torch.zeros(0, dtype=torch.uint8)


def column_parts(flat_q, flat_s, width, offsets):
    """The experts' matrices [width][rows of e] of flat codes and scales, as values."""
    out, at, at_s = [], 0, 0
    for a, b in zip(offsets[:-1], offsets[1:]):
        n = blocks(b - a)
        if n == 0:
            out.append(torch.zeros(width, 0, dtype=torch.float64))
            continue
        q, s = flat_q[at: at + width * n * BLOCK].reshape(width, n * BLOCK), flat_s[at_s: at_s + -(-n // 4) * width * 4].reshape(-1, width, 4)
        out.append(values(q, s, b - a))
        at, at_s = at + width * n * BLOCK, at_s + -(-n // 4) * width * 4
    return out

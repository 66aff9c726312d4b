"""The definitions that the packed kernels are held to, against torch's own 8-bit type and hand-worked values. CPU only."""
import torch

import packed_refs as R


def test_codes_are_those_of_the_type():
    q = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    want = q.view(torch.float8_e4m3fn).double()
    got = R.decode(q)
    assert torch.equal(got.nan_to_num(nan=1e9), want.nan_to_num(nan=1e9))
    g = torch.Generator().manual_seed(1)
    x = torch.cat([torch.randn(20000, generator=g) * s for s in (0.003, 0.1, 3.0, 100.0)]).clamp(-448, 448)
    assert torch.equal(R.code(x.double()), x.to(torch.float8_e4m3fn).view(torch.uint8))
    ties = (R.magnitudes()[:-1] + R.magnitudes()[1:]) / 2
    assert torch.equal(R.code(ties), ties.float().to(torch.float8_e4m3fn).view(torch.uint8))


def test_powers():
    top = torch.tensor([448.0, 448.0001, 224.0, 224.0001, 1.0, 0.0, 2.0 ** -139, 3.4e38, 1.75, 1.76], dtype=torch.float64)
    s = R.scale_bytes(top)
    assert s.tolist() == [127, 128, 126, 127, 119, 0, 0, 247, 119, 120]
    for t, b in zip(top.tolist(), s.tolist()):
        assert t <= 448 * 2.0 ** (b - 127) and (b == 0 or t > 224 * 2.0 ** (b - 127))


def test_layout():
    s = torch.arange(3 * 5, dtype=torch.uint8).reshape(3, 5)
    flat = R.layout(s)
    assert flat.shape == (2, 3, 4) and flat[1, 2].tolist() == [14, 127, 127, 127] and flat[0, 1].tolist() == [5, 6, 7, 8]
    assert torch.equal(R.unlayout(flat, 5), s)
    x = torch.randn(7, 300, dtype=torch.float64)
    q, sc = R.pack(x)
    v = R.values(q, sc, 300)
    assert q.shape == (7, 384) and not q[:, 300:].any()
    assert bool(((v - x).abs() <= 2.0 ** -4 * x.abs() + 2.0 ** -10 * torch.exp2(R.unlayout(sc, 3).double() - 127).repeat_interleave(128, 1)[:, :300]).all())


def test_a_value_packed_again_stays():
    """In other blocks a packed value is what it was, unless it lies 2^13 below its new block's largest."""
    x = torch.randn(256, 256, dtype=torch.float64) * torch.exp2(torch.randint(-5, 5, (256, 256)).double())
    v = R.values(*R.pack(x), 256)
    w = R.values(*R.pack(v.t().contiguous()), 256).t()
    top = v.abs().unflatten(0, (2, 128)).amax(1).repeat_interleave(128, 0)
    assert torch.equal(w[v.abs() >= top * 2.0 ** -13], v[v.abs() >= top * 2.0 ** -13])

"""Arguments that the packed operators refuse: a status before anything is launched. CPU only: no call here gets past validation."""
import ctypes
import os

import pytest
import torch

from paper_2406_00023_amd import binding as B
from paper_2406_00023_amd.dropless_block import BlockShape, PackedBlock

NULL, SHAPE, UNSUPPORTED, WORKSPACE, ALIGN = 1, 2, 3, 4, 5
ok, odd, null = ctypes.c_void_p(4096), ctypes.c_void_p(4100), ctypes.c_void_p(0)
F, H = torch.float32, torch.bfloat16
P = lambda v=4096, s=4096: B.EtrPacked(v, s)
none = None


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2406_00023_amd.build import build
        build()
    return B.load_library()


@pytest.mark.parametrize("cfg,status", [
    (B.make_pack_config(0, 64, F), SHAPE), (B.make_pack_config(4, 0, F), SHAPE), (B.make_pack_config(4, -8, F), SHAPE), (B.make_pack_config(4, 64, F, E=0), SHAPE),
    (B.make_pack_config(4, 60, F), UNSUPPORTED), (B.make_pack_config(4, 64, 2), UNSUPPORTED), (B.make_pack_config(4, 64, F, E=65), UNSUPPORTED),
    (B.make_pack_config(4, 64, F, sorted=2), UNSUPPORTED), (B.make_pack_config(4, (1 << 20) + 8, F), UNSUPPORTED), (B.make_pack_config((1 << 28) + 1, 64, F), UNSUPPORTED),
    (B.make_pack_config(1 << 27, 64, F, E=4), UNSUPPORTED), (B.make_pack_config(1 << 28, 1 << 20, F), UNSUPPORTED)])
def test_pack_configs(lib, cfg, status):
    c = ctypes.byref(cfg)
    for f in (B.etr_packed_rows_bytes, B.etr_packed_rows_scale_bytes, B.etr_packed_columns_bytes, B.etr_packed_columns_scale_bytes):
        assert f(cfg) == 0
    assert lib.etr_pack_rows(c, ok, ok, ok, null) == status and lib.etr_unpack_rows(c, ok, ok, ok, null) == status
    assert lib.etr_pack_columns(c, ok, ok, ok, ok, null) == status and lib.etr_repack_columns(c, ok, ok, ok, ok, ok, null) == status
    assert lib.etr_pack_columns_pair(c, ok, ok, ok, ok, null) == status


def test_sizes(lib):
    cfg = B.make_pack_config(5, 136, F, E=3)
    assert B.etr_packed_rows_bytes(cfg) == 3 * 5 * 256 and B.etr_packed_rows_scale_bytes(cfg) == 3 * 5 * 4
    assert B.etr_packed_columns_bytes(cfg) == 3 * 136 * 128 and B.etr_packed_columns_scale_bytes(cfg) == 3 * 136 * 4
    cfg = B.make_pack_config(1000, 136, F, E=3, sorted=1)
    assert B.etr_packed_rows_bytes(cfg) == 1000 * 256 and B.etr_packed_rows_scale_bytes(cfg) == 1000 * 4
    assert B.etr_packed_columns_bytes(cfg) == 136 * 128 * (7 + 3) and B.etr_packed_columns_scale_bytes(cfg) == 136 * 4 * (1 + 3)
    assert B.etr_packed_columns_bytes(B.make_pack_config(2, 136, F, E=64, sorted=1)) == 136 * 128 * 2
    assert B.etr_packed_rows_scale_bytes(B.make_pack_config(7, 520, F)) == 7 * 2 * 4
    assert B.etr_packed_rows_bytes(B.make_pack_config(1 << 28, 1024, F)) == 1 << 38


def test_pack_arguments(lib):
    cfg, srt = B.make_pack_config(4, 64, F, E=2), B.make_pack_config(4, 64, F, E=2, sorted=1)
    for fn, n in ((lib.etr_pack_rows, 3), (lib.etr_unpack_rows, 3), (lib.etr_pack_columns_pair, 4)):
        assert fn(None, *[ok] * n, null) == NULL
        for i in range(n):
            assert fn(ctypes.byref(cfg), *[null if j == i else ok for j in range(n)], null) == NULL
            assert fn(ctypes.byref(cfg), *[odd if j == i else ok for j in range(n)], null) == ALIGN
    s = ctypes.byref(B.make_sort_config(4, 1, 4, 64, F))
    for i in range(4):
        assert lib.etr_pack_sorted_rows(s, *[null if j == i else ok for j in range(4)], null) == NULL
        assert lib.etr_pack_sorted_rows(s, *[odd if j == i else ok for j in range(4)], null) == ALIGN
    assert lib.etr_pack_sorted_rows(ctypes.byref(B.make_sort_config(4, 1, 65, 64, F)), ok, ok, ok, ok, null) == UNSUPPORTED
    for i in range(4):
        assert lib.etr_pack_columns(ctypes.byref(srt), *[null if j == i else ok for j in range(4)], null) == NULL
        assert lib.etr_pack_columns(ctypes.byref(srt), *[odd if j == i else ok for j in range(4)], null) == ALIGN
    for i in range(5):
        assert lib.etr_repack_columns(ctypes.byref(srt), *[null if j == i else ok for j in range(5)], null) == NULL
        assert lib.etr_repack_columns(ctypes.byref(srt), *[odd if j == i else ok for j in range(5)], null) == ALIGN
    assert lib.etr_pack_columns(ctypes.byref(cfg), ok, ok, ok, ok, null) == NULL                   # a stack has no table
    assert lib.etr_repack_columns(ctypes.byref(cfg), ok, ok, ok, ok, ok, null) == NULL
    assert lib.etr_pack_columns_pair(ctypes.byref(srt), ok, ok, ok, ok, null) == UNSUPPORTED


BAD = [(B.make_linear_config(0, 64, 64, 1, F), SHAPE), (B.make_linear_config(4, 60, 64, 1, F), UNSUPPORTED), (B.make_linear_config(4, 64, 64, 65, F), UNSUPPORTED),
       (B.make_linear_config(4, 64, 64, 1, F, act=4), UNSUPPORTED), (B.make_linear_config(4, 64, 64, 1, 2), UNSUPPORTED)]


@pytest.mark.parametrize("cfg,status", BAD)
def test_product_configs(lib, cfg, status):
    c = ctypes.byref(cfg)
    assert B.etr_packed_act_workspace_bytes(cfg) == 0
    assert lib.etr_packed_linear(c, P(), ok, P(), none, null, null, null, ok, none, none, none, null) == status
    assert lib.etr_packed_act_backward(c, ok, ok, none, none, P(), none, null, null, null, 0, null) == status
    assert lib.etr_packed_weight_gradient(c, P(), P(), ok, ok, null, null) == status


def test_linear_arguments(lib):
    plain, glu, one = (B.make_linear_config(40, 64, 64, e, F, act=a) for e, a in ((2, B.ACT_SILU), (2, B.ACT_SWIGLU), (1, B.ACT_NONE)))
    f = lambda c, *a: lib.etr_packed_linear(ctypes.byref(c), *a, null)       # x offsets w w_up bias bias_up residual y y8 pre8 pre_up8
    base = [P(), ok, P(), none, null, null, null, ok, none, none, none]
    def but(args, **kw):
        out = list(args)
        for k, v in kw.items():
            out[int(k[1:])] = v
        return out
    assert lib.etr_packed_linear(None, *base, null) == NULL
    for i in (0, 2):
        assert f(plain, *but(base, **{f"a{i}": none})) == NULL
        assert f(plain, *but(base, **{f"a{i}": P(0)})) == NULL and f(plain, *but(base, **{f"a{i}": P(s=0)})) == NULL
        assert f(plain, *but(base, **{f"a{i}": P(4100)})) == ALIGN and f(plain, *but(base, **{f"a{i}": P(s=4100)})) == ALIGN
    for i in (8, 9):
        assert f(plain, *but(base, **{f"a{i}": P(0)})) == NULL and f(plain, *but(base, **{f"a{i}": P(s=4100)})) == ALIGN
    assert f(plain, *but(base, a7=null)) == NULL               # no result asked for
    assert f(plain, *but(base, a1=null)) == NULL               # two experts and no table
    for i in (1, 4, 6, 7):
        assert f(plain, *but(base, **{f"a{i}": odd})) == ALIGN
    assert f(plain, *but(base, a3=P())) == NULL and f(plain, *but(base, a5=ok)) == NULL and f(plain, *but(base, a10=P())) == NULL
    full = [P(), ok, P(), P(), ok, ok, ok, ok, P(), P(), P()]
    assert f(glu, *but(full, a3=none)) == NULL and f(glu, *but(full, a4=null)) == NULL and f(glu, *but(full, a5=null)) == NULL
    assert f(glu, *but(full, a9=none)) == NULL and f(glu, *but(full, a10=none)) == NULL
    assert f(one, *but(base, a1=null, a0=none)) == NULL


def test_act_arguments(lib):
    none_, silu, glu = (B.make_linear_config(400, 64, 64, 2, F, act=a) for a in (B.ACT_NONE, B.ACT_SILU, B.ACT_SWIGLU))
    f = lambda c, *a, ws=ok, n=1 << 30: lib.etr_packed_act_backward(ctypes.byref(c), *a, ws, n, null)   # dy offsets pre8 pre_up8 d8 dt8 dbias dbias_up
    assert lib.etr_packed_act_backward(None, ok, ok, none, none, P(), P(), null, null, null, 0, null) == NULL
    assert f(none_, null, ok, none, none, P(), P(), null, null) == NULL and f(none_, odd, ok, none, none, P(), P(), null, null) == ALIGN
    assert f(none_, ok, null, none, none, P(), P(), null, null) == NULL
    assert f(none_, ok, ok, none, none, none, none, null, null) == NULL                            # nothing asked for
    assert f(none_, ok, ok, P(), none, P(), none, null, null) == NULL                              # a pre-activation and no activation
    assert f(silu, ok, ok, none, none, P(), none, null, null) == NULL
    assert f(silu, ok, ok, P(), P(), P(), none, null, null) == NULL and f(silu, ok, ok, P(), none, P(), none, ok, ok) == NULL
    assert f(glu, ok, ok, P(), none, P(), none, null, null) == NULL and f(glu, ok, ok, P(), P(), P(), none, ok, null) == NULL
    assert f(glu, ok, ok, P(), P(), P(), none, null, ok) == NULL
    for i in range(2, 6):
        a = [ok, ok, P(), P(), P(), P(), ok, ok]
        a[i] = P(4100)
        assert f(glu, *a) == ALIGN
        a[i] = P(s=0)
        assert f(glu, *a) == NULL
    for i in (6, 7):
        a = [ok, ok, P(), P(), P(), P(), ok, ok]
        a[i] = odd
        assert f(glu, *a) == ALIGN
    assert f(silu, ok, ok, P(), none, none, none, ok, null, ws=null) == NULL and f(silu, ok, ok, P(), none, none, none, ok, null, n=16) == WORKSPACE
    assert f(silu, ok, ok, P(), none, none, none, ok, null, ws=odd) == ALIGN


def test_weight_arguments(lib):
    plain, glu = (B.make_linear_config(40, 64, 64, 2, F, act=a) for a in (B.ACT_SILU, B.ACT_SWIGLU))
    f = lambda c, *a: lib.etr_packed_weight_gradient(ctypes.byref(c), *a, null)          # dt8 xt8 offsets dw dw_up
    assert lib.etr_packed_weight_gradient(None, P(), P(), ok, ok, null, null) == NULL
    assert f(plain, none, P(), ok, ok, null) == NULL and f(plain, P(), none, ok, ok, null) == NULL
    assert f(plain, P(4100), P(), ok, ok, null) == ALIGN and f(plain, P(), P(s=4100), ok, ok, null) == ALIGN
    assert f(plain, P(), P(), null, ok, null) == NULL and f(plain, P(), P(), ok, null, null) == NULL
    assert f(plain, P(), P(), odd, ok, null) == ALIGN and f(plain, P(), P(), ok, odd, null) == ALIGN
    assert f(plain, P(), P(), ok, ok, ok) == NULL and f(glu, P(), P(), ok, ok, null) == NULL and f(glu, P(), P(), ok, ok, odd) == ALIGN
    assert f(B.make_linear_config((1 << 24) + 1, 64, 64, 2, F), P(), P(), ok, ok, null) == UNSUPPORTED


def test_strides_that_the_binding_refuses():
    cfg = B.make_pack_config(4, 64, F)
    with pytest.raises(ValueError):
        B.etr_pack_rows(cfg, torch.zeros(4, 128)[:, ::2], (torch.zeros(512, dtype=torch.uint8), torch.zeros(16, dtype=torch.uint8)))
    with pytest.raises(ValueError):
        B.make_pack_config(4, 64, torch.float16)


def test_a_block_whose_weights_are_not_packed(lib):
    block = PackedBlock(BlockShape(4, 64, 4, 8, 2, 64, F), device="cpu")
    with pytest.raises(RuntimeError, match="pack_weights"):
        block.forward(None, None, None)

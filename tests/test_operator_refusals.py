"""Arguments that the operators around the layer refuse: a status before anything is launched. CPU only: no call here gets
past validation."""
import ctypes
import os

import pytest
import torch

from paper_2406_00023_amd import binding as B
from paper_2406_00023_amd import inputs as I

NULL, SHAPE, UNSUPPORTED, WORKSPACE, ALIGN = 1, 2, 3, 4, 5
ok, odd, null = ctypes.c_void_p(4096), ctypes.c_void_p(4100), ctypes.c_void_p(0)
F, H = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2406_00023_amd.build import build
        build()
    return B.load_library()


@pytest.mark.parametrize("cfg,status", [
    (B.make_norm_config(0, 64, F), SHAPE), (B.make_norm_config(4, -8, F), SHAPE), (B.make_norm_config(4, 64, F, eps=0.0), SHAPE),
    (B.make_norm_config(4, 64, F, eps=float("nan")), SHAPE), (B.make_norm_config(4, 64, F, eps=float("inf")), SHAPE),
    (B.make_norm_config(4, 64, F, residual_scale=float("nan")), SHAPE), (B.make_norm_config(4, 64, F, block_scale=float("inf")), SHAPE),
    (B.make_norm_config(4, 60, F), UNSUPPORTED), (B.make_norm_config(4, 64, 2), UNSUPPORTED), (B.make_norm_config(4, 16392, F), UNSUPPORTED),
    (B.make_norm_config(4, 32776, H), UNSUPPORTED)])
def test_norm_configs(lib, cfg, status):
    c = ctypes.byref(cfg)
    assert B.etr_norm_workspace_bytes(cfg) == 0
    assert lib.etr_block_norm(c, ok, null, null, null, ok, null, ok, null) == status
    assert lib.etr_block_norm_backward(c, ok, null, null, null, ok, null, ok, ok, null, null, null, null, null, 0, null) == status


def test_norm_arguments(lib):
    cfg = B.make_norm_config(4, 64, F)
    c = ctypes.byref(cfg)
    f = lambda *a: lib.etr_block_norm(c, *a, null)             # x, y, gate, w_post, w_pre, x_out, h
    assert lib.etr_block_norm(None, ok, null, null, null, ok, null, ok, null) == NULL
    assert f(null, null, null, null, ok, null, ok) == NULL     # no x
    assert f(ok, null, null, null, null, null, null) == NULL   # neither y nor a norm
    assert f(ok, null, null, null, ok, null, null) == NULL     # a norm and no place for it
    assert f(ok, null, null, null, null, null, ok) == NULL
    assert f(ok, ok, null, null, null, null, null) == NULL     # a join and no place for it
    assert f(ok, null, null, null, ok, ok, ok) == NULL         # a place and no join
    assert f(ok, null, ok, null, ok, null, ok) == NULL and f(ok, null, null, ok, ok, null, ok) == NULL
    assert f(odd, null, null, null, ok, null, ok) == ALIGN and f(ok, ok, odd, null, null, ok, null) == ALIGN
    g = lambda *a, ws=ok, n=1 << 30: lib.etr_block_norm_backward(c, *a, ws, n, null)   # x_out y gate w_post w_pre dx_out dh dx dy dgate dw_post dw_pre
    full = [ok] * 12
    assert g(ok, ok, ok, ok, ok, ok, ok, null, ok, ok, ok, ok) == NULL
    assert g(null, ok, ok, ok, ok, ok, ok, ok, ok, ok, ok, ok) == NULL                  # a norm's gradient needs its input
    assert g(ok, null, null, null, null, ok, null, ok, null, null, null, null) == NULL
    assert g(ok, ok, null, ok, ok, ok, null, ok, ok, null, ok, ok) == NULL              # w_pre and no dh
    assert g(ok, ok, null, ok, ok, ok, ok, ok, ok, ok, ok, ok) == NULL                  # dgate and no gate
    assert g(ok, ok, ok, null, ok, ok, ok, ok, ok, ok, ok, ok) == NULL                  # dw_post and no w_post
    assert g(ok, ok, ok, ok, null, ok, null, ok, ok, ok, ok, ok) == NULL                # dw_pre and no w_pre
    assert g(ok, ok, ok, ok, ok, ok, ok, ok, null, ok, ok, ok) == NULL                  # y and no dy
    assert g(*full, ws=null) == NULL and g(*full, n=16) == WORKSPACE and g(*full, ws=odd) == ALIGN
    assert g(*full[:-1], odd) == ALIGN


@pytest.mark.parametrize("cfg,status", [
    (B.make_sort_config(0, 1, 4, 64, F), SHAPE), (B.make_sort_config(4, 0, 4, 64, F), SHAPE), (B.make_sort_config(4, 5, 4, 64, F), SHAPE),
    (B.make_sort_config(4, 1, 0, 64, F), SHAPE), (B.make_sort_config(4, 1, 4, 0, F), SHAPE), (B.make_sort_config(4, 1, 65, 64, F), UNSUPPORTED),
    (B.make_sort_config(4, 1, 4, 60, F), UNSUPPORTED), (B.make_sort_config(4, 1, 4, 64, 2), UNSUPPORTED),
    (B.make_sort_config(4, 1, 4, 64, F, gate_norm=2), UNSUPPORTED), (B.make_sort_config((1 << 29) + 1, 2, 4, 8, F), UNSUPPORTED),
    (B.make_sort_config(4, 1, 4, 32776, F), UNSUPPORTED)])
def test_sort_configs(lib, cfg, status):
    c = ctypes.byref(cfg)
    assert B.etr_sort_workspace_bytes(cfg) == 0
    assert lib.etr_sort_tokens(c, ok, null, ok, ok, ok, ok, 1 << 30, null) == status
    assert lib.etr_sort_rows(c, ok, ok, ok, null) == status and lib.etr_sort_rows_backward(c, ok, ok, ok, null) == status
    assert lib.etr_unsort_rows(c, ok, ok, ok, ok, ok, null) == status
    assert lib.etr_unsort_rows_backward(c, ok, ok, ok, ok, ok, ok, ok, null) == status


def test_sort_arguments(lib):
    cfg = B.make_sort_config(100, 2, 4, 64, F)
    c = ctypes.byref(cfg)
    assert lib.etr_sort_tokens(None, ok, null, ok, ok, ok, ok, 1 << 30, null) == NULL
    for fn, n in ((lib.etr_sort_rows, 3), (lib.etr_sort_rows_backward, 3), (lib.etr_unsort_rows, 5), (lib.etr_unsort_rows_backward, 7)):
        for i in range(n):
            assert fn(c, *[null if j == i else ok for j in range(n)], null) == NULL
            assert fn(c, *[odd if j == i else ok for j in range(n)], null) == ALIGN
    f = lambda *a: lib.etr_sort_tokens(c, *a, null)
    for i in (0, 2, 3, 4, 5):
        assert f(*[null if j == i else ok for j in range(6)], 1 << 30) == NULL
    assert f(ok, odd, ok, ok, ok, ok, 1 << 30) == ALIGN and f(ok, null, ok, ok, ok, ok, 0) == WORKSPACE


def test_route_backward_arguments(lib):
    cfg = B.make_config(I.CONFIGS["cfg1"])
    c = ctypes.byref(cfg)
    for i in (0, 1, 2, 3, 4, 6):
        assert lib.etr_route_backward(c, *[null if j == i else ok for j in range(7)], null) == NULL
    assert lib.etr_route_backward(c, ok, ok, ok, ok, ok, odd, ok, null) == ALIGN
    big = B.make_config(I.CONFIGS["cfg1"].with_(E=64, d=4096, D=8, k=1))
    assert lib.etr_route_backward(ctypes.byref(big), *([ok] * 7), null) == UNSUPPORTED
    bad = B.make_config(I.CONFIGS["cfg1"].with_(T=0))
    assert lib.etr_route_backward(ctypes.byref(bad), *([ok] * 7), null) == SHAPE


def test_types_and_strides_that_the_binding_refuses():
    with pytest.raises(ValueError):
        B.make_norm_config(4, 64, torch.float16)
    with pytest.raises(ValueError):
        B.make_sort_config(4, 1, 4, 64, torch.int32)
    cfg = B.make_norm_config(4, 64, F)
    with pytest.raises(ValueError):                            # a strided view
        B.etr_block_norm(cfg, torch.zeros(4, 128)[:, ::2], w_pre=torch.ones(64), h=torch.zeros(4, 64))


@pytest.mark.parametrize("cfg,status", [
    (B.make_linear_config(0, 64, 64, 1, F), SHAPE), (B.make_linear_config(4, 0, 64, 1, F), SHAPE), (B.make_linear_config(4, 64, -8, 1, F), SHAPE),
    (B.make_linear_config(4, 64, 64, 0, F), SHAPE), (B.make_linear_config(4, 60, 64, 1, F), UNSUPPORTED), (B.make_linear_config(4, 64, 60, 1, F), UNSUPPORTED),
    (B.make_linear_config(4, 64, 64, 65, F), UNSUPPORTED), (B.make_linear_config(4, 64, 64, 1, 2), UNSUPPORTED),
    (B.make_linear_config(4, 64, 64, 1, F, act=4), UNSUPPORTED), (B.make_linear_config(4, 64, 64, 1, F, act=-1), UNSUPPORTED),
    (B.make_linear_config(4, (1 << 20) + 8, 64, 1, F), UNSUPPORTED), (B.make_linear_config((1 << 28) + 1, 64, 64, 1, F), UNSUPPORTED),
    (B.make_linear_config(4, 1 << 20, 1 << 20, 64, F), UNSUPPORTED)])
def test_linear_configs(lib, cfg, status):
    c = ctypes.byref(cfg)
    assert B.etr_linear_workspace_bytes(cfg) == 0
    assert lib.etr_expert_linear(c, ok, ok, ok, null, null, null, null, ok, null, null, null) == status
    assert lib.etr_expert_linear_backward(c, ok, ok, ok, null, ok, null, ok, ok, ok, null, ok, null, ok, 1 << 40, null) == status


def test_linear_arguments(lib):
    plain, glu, one = (ctypes.byref(B.make_linear_config(40, 64, 64, e, F, act=a)) for e, a in ((2, B.ACT_SILU), (2, B.ACT_SWIGLU), (1, B.ACT_NONE)))
    f = lambda c, *a: lib.etr_expert_linear(c, *a, null)       # x offsets w w_up bias bias_up residual y pre pre_up
    assert lib.etr_expert_linear(None, ok, ok, ok, null, null, null, null, ok, null, null, null) == NULL
    for i in (0, 1, 2, 7):
        assert f(plain, *[null if j == i else (ok if j in (0, 1, 2, 7) else null) for j in range(10)]) == NULL
    assert f(one, null, null, ok, null, null, null, null, ok, null, null) == NULL
    assert f(plain, ok, ok, ok, ok, null, null, null, ok, null, null) == NULL           # w_up and nothing to do with it
    assert f(plain, ok, ok, ok, null, null, ok, null, ok, null, null) == NULL           # bias_up likewise
    assert f(plain, ok, ok, ok, null, null, null, null, ok, null, ok) == NULL
    assert f(glu, ok, ok, ok, null, null, null, null, ok, null, null) == NULL           # no w_up
    assert f(glu, ok, ok, ok, ok, ok, null, null, ok, null, null) == NULL               # one bias of two
    assert f(glu, ok, ok, ok, ok, null, null, null, ok, ok, null) == NULL               # one pre-activation of two
    for i in range(10):
        assert f(glu, *[odd if j == i else ok for j in range(10)]) == ALIGN
    b = lambda c, *a, ws=ok, n=1 << 30: lib.etr_expert_linear_backward(c, *a, ws, n, null)   # x off w w_up pre pre_up dy dx dw dw_up dbias dbias_up
    full = [ok] * 12
    for i in (0, 1, 2, 3, 4, 5, 6, 9, 11):
        assert b(glu, *[null if j == i else ok for j in range(12)]) == NULL, i
    for i in range(12):
        assert b(glu, *[odd if j == i else ok for j in range(12)]) == ALIGN
    assert b(glu, *full, ws=null) == NULL and b(glu, *full, n=16) == WORKSPACE
    assert b(glu, ok, ok, ok, ok, ok, ok, ok, null, null, null, null, null) == NULL     # nothing asked for
    assert b(plain, ok, ok, ok, null, ok, null, ok, ok, ok, ok, null, null) == NULL     # dw_up and no second weight
    assert b(plain, ok, ok, ok, null, null, null, ok, ok, ok, null, null, null) == NULL # an activation and no pre-activation

"""The operators around the layer at the ends of what their configs allow. CPU only: workspace queries, nothing is launched."""
import pytest
import torch

from paper_2406_00023_amd import binding as B


@pytest.mark.parametrize("T", [4096, 100000, 2 ** 31 - 4, 2 ** 31 - 3, 2 ** 31 - 1])
def test_norm_workspace_of_many_tokens(T):
    """From 4096 tokens on all numbers of tokens have as many workgroups."""
    assert B.etr_norm_workspace_bytes(B.make_norm_config(T, 64, torch.float32)) == 1024 * 2 * 64 * 4


@pytest.mark.parametrize("inside,past", [
    # w (rows / 32 + E) <= 2^30, w = ceil(max(K, N) / 32)
    ((1 << 28, 64, 4064, 8), (1 << 28, 64, 4096, 8)), ((1 << 25, (1 << 15) - 32, 64, 1), (1 << 25, 1 << 15, 64, 1)),
    ((((1 << 20) - 1) * 32, 64, 1 << 15, 1), ((1 << 20) * 32, 64, 1 << 15, 1)),
    # w^2 E <= 2^30
    ((64, 64, 1 << 17, 64), (64, 64, (1 << 17) + 8, 64)), ((64, 1 << 20, 64, 1), (64, 1 << 20, 64, 2)),
    # the plain ones
    ((64, 1 << 20, 8, 1), (64, (1 << 20) + 8, 8, 1)), ((1 << 28, 8, 8, 64), ((1 << 28) + 1, 8, 8, 64)), ((64, 64, 64, 64), (64, 64, 64, 65))])
def test_linear_limits_are_those_of_the_header(inside, past):
    for dtype in (torch.float32, torch.bfloat16):
        for act in (B.ACT_NONE, B.ACT_SWIGLU):
            assert B.etr_linear_workspace_bytes(B.make_linear_config(*inside, dtype, act=act)) > 0
            assert B.etr_linear_workspace_bytes(B.make_linear_config(*past, dtype, act=act)) == 0

"""The operators around the layer at the ends of what their configs allow. CPU only: workspace queries, nothing is launched."""
import pytest
import torch

from paper_2406_00023_amd import binding as B


@pytest.mark.parametrize("T", [4096, 100000, 2 ** 31 - 4, 2 ** 31 - 3, 2 ** 31 - 1])
def test_norm_workspace_of_many_tokens(T):
    """From 4096 tokens on all numbers of tokens have as many workgroups."""
    assert B.etr_norm_workspace_bytes(B.make_norm_config(T, 64, torch.float32)) == 1024 * 2 * 64 * 4

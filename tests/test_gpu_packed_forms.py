"""Each form of the products of packed operands element by element, with everything in the epilogue, in both types of results."""
import pytest

import packed_forms as F
from test_gpu_packed_backward import weights_case
from test_gpu_packed_linear import case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("product,act,form,rows,E,K,N", F.listed(F.FORWARD, F.PACKING))
def test_forward(product, act, form, rows, E, K, N, dtype):
    assert F.plan(product, act, rows, E, K, N, dtype) == form
    counts, spare = F.counts(rows, E)
    keep = product == F.PACKING
    case(counts, K, N, dtype, act, bias=True, residual=True, keep=keep, extra=spare, seed=K)
    if act == "none":                                          # (every activation has a pass of its own)
        for other in ("silu", "gelu"):
            case(counts, K, N, dtype, other, keep=keep, extra=spare, seed=N)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("product,act,form,rows,E,K,N", F.listed(F.WEIGHT))
def test_weights(product, act, form, rows, E, K, N, dtype):
    assert F.plan(product, act, rows, E, K, N, dtype) == form
    counts, spare = F.counts(rows, E)
    weights_case(counts, K, N, act == "swiglu", dtype, extra=spare)

"""The row kernels (block norm, sorted rows, router gradient) at the widths and numbers of tokens on both sides of what chooses their forms: 16-byte
pieces to a row (a quarter of its fp32 values, an eighth of its bf16 ones), and more than 2048 tokens or fewer."""
import pytest

import test_gpu_block_norm as N
import test_gpu_route_backward as R
import test_gpu_sorted_rows as S

pytestmark = pytest.mark.gpu
VALUES = {"f32": 4, "bf16": 8}
FULL, JOIN, PRE = N.PARTS[0], N.PARTS[2], N.PARTS[4]       # everything; a block and no norm behind it; a norm alone


def _widths(dtype, pieces):
    return [(dtype, p * VALUES[dtype]) for p in pieces if p * VALUES[dtype] % 8 == 0]


FEW = [c for t in VALUES for c in _widths(t, (64, 66, 130, 256, 258, 512, 514, 1024, 1026, 2048, 2050, 4096))]
MANY = [c for t in VALUES for c in _widths(t, (64, 66, 128, 130, 256, 258, 512, 514))]


@pytest.mark.parametrize("parts", [FULL, JOIN, PRE])
@pytest.mark.parametrize("dtype,d", FEW)
def test_norm_of_few_tokens(dtype, d, parts):
    print(f"norm 6 x {d} {dtype} {parts}", flush=True)
    N.test_forward(6, d, dtype, parts)
    N.test_backward(6, d, dtype, parts)


@pytest.mark.parametrize("parts", [FULL, PRE])
@pytest.mark.parametrize("dtype,d", MANY)
def test_norm_of_many_tokens(dtype, d, parts):
    print(f"norm 2051 x {d} {dtype} {parts}", flush=True)
    N.test_forward(2051, d, dtype, parts)
    N.test_backward(2051, d, dtype, parts)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,k,E,d", [(2100, 2, 8, 1000), (2048, 2, 8, 520), (2049, 2, 8, 1032), (6, 3, 8, 1024), (6, 3, 8, 16392)])
def test_sorted_rows(T, k, E, d, dtype):
    print(f"sorted rows {T} x {k} of {E}, {d} {dtype}", flush=True)
    S.test_rows_and_gradients(T, k, E, d, "holes", dtype)


@pytest.mark.parametrize("pooled", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,d,E,D", [(70, 1024, 8, 16), (70, 768, 8, 16), (70, 1032, 6, 24), (33, 2064, 8, 16), (9, 4128, 5, 32)])
def test_router_gradient(T, d, E, D, dtype, pooled):
    print(f"router gradient {T} x {d}, {E} of {D} {dtype} pooled {pooled}", flush=True)
    R.test_against_64_bits(T, d, E, D, dtype, pooled)

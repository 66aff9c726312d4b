"""Which form each product on sorted rows takes, asked from the library on the host (no GPU): every form that is compiled has a product
that takes it, the element-wise tests run one of each, and no size takes a form that they do not."""
import random
import re

import pytest

import linear_forms as F
from paper_2406_00023_amd import binding as B


@pytest.mark.parametrize("product,dtype,act,form,rows,E,K,N", F.listed(F.FORWARD, F.INPUT, F.WEIGHT, F.JOINT))
def test_listed_products_take_their_forms(product, dtype, act, form, rows, E, K, N):
    assert F.plan(product, dtype, act, rows, E, K, N) == form


def test_no_size_takes_a_form_that_is_not_listed():
    rng, grid = random.Random(1), lambda most: int(2 ** rng.uniform(0, most))
    for _ in range(6000):
        dtype, act, E = rng.choice(["f32", "bf16"]), rng.choice(["none", "swiglu"]), rng.choice([1, 2, 4, 8, 12, 16, 32, 64])
        rows, K, N = grid(17), 8 * grid(11), 8 * grid(11)
        for product in (F.FORWARD, F.INPUT, F.WEIGHT, F.JOINT):
            assert F.plan(product, dtype, act, rows, E, K, N) in F.CASES[product, dtype, act], (product, dtype, act, rows, E, K, N)


def test_every_compiled_form_is_listed():
    F.plan(F.FORWARD, "f32", "none", 1, 1, 8, 8)               # the library is there
    with open(B.LIB_PATH, "rb") as f:
        names = f.read()
    kernels = set(re.findall(rb"linear_kernelILb([01])ELi(\d+)ELi\d+ELi\d+ELi\d+ELi\d+ELi(\d+)ELi(\d)ELb([01])E", names))
    assert kernels
    for bf16, rows, shared, product, glu in kernels:
        product, dtype, form = int(product), "bf16" if bf16 == b"1" else "f32", rows.decode() + ("+" if int(shared) > 1 else "")
        assert form in F.CASES[product, dtype, "swiglu" if glu == b"1" else "none"], (product, dtype, form, glu)

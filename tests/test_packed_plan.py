"""Which form each product of packed operands takes, asked from the library on the host (no GPU): every form that is compiled has a product that
takes it, the element-wise tests run one of each, and no size takes a form that they do not."""
import random
import re

import pytest

import packed_forms as F
from paper_2406_00023_amd import binding as B


@pytest.mark.parametrize("product,act,form,rows,E,K,N", F.listed(F.FORWARD, F.PACKING, F.WEIGHT))
def test_listed_products_take_their_forms(product, act, form, rows, E, K, N):
    assert F.plan(product, act, rows, E, K, N) == form and F.plan(product, act, rows, E, K, N, "f32") == form


def test_no_size_takes_a_form_that_is_not_listed():
    rng, grid = random.Random(1), lambda most: int(2 ** rng.uniform(0, most))
    for _ in range(6000):
        act, E = rng.choice(["none", "swiglu"]), rng.choice([1, 2, 4, 8, 12, 16, 32, 64])
        rows, K, N = grid(17), 8 * grid(11), 8 * grid(11)
        for product in (F.FORWARD, F.PACKING, F.WEIGHT):
            assert F.plan(product, act, rows, E, K, N) in F.CASES[product, act], (product, act, rows, E, K, N)


def test_every_compiled_form_is_listed():
    F.plan(F.FORWARD, "none", 1, 1, 8, 8)                      # the library is there
    with open(B.LIB_PATH, "rb") as f:
        names = f.read()
    tiles = set(re.findall(rb"packed_tiles_kernelILb([01])ELi(\d+)ELi\d+ELi\d+ELi\d+ELi([01])ELb([01])E", names))
    assert tiles
    for _, rows, weight, glu in tiles:
        for product in ((F.WEIGHT,) if weight == b"1" else (F.FORWARD, F.PACKING)):
            assert rows.decode() in F.CASES[product, "swiglu" if glu == b"1" else "none"], (product, rows, glu)
    few = set(re.findall(rb"packed_rows_kernelILb([01])ELi(\d)ELi\dELb([01])ELb([01])E", names))
    assert few
    for _, waves, glu, packs in few:
        assert f"rows{16 * int(waves)}" in F.CASES[F.PACKING if packs == b"1" else F.FORWARD, "swiglu" if glu == b"1" else "none"]

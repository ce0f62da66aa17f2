"""Which tiles the products' sizes lead to (a rule on the host), and that the GPU's tests reach
every one of them."""
import random

import pytest

import paper_2103_16716_amd as pb
from test_gpu_expert_tiles import BEFORE, BEHIND, CASES, DTYPES, PRODUCTS
from test_gpu_experts import IN_PARTS, SHAPES, test_large_products as large


def kind(product, dtype, N, E, K, O):
    rows, cols, parts = pb.expert_linear_tile(PRODUCTS[product], N, E, K, O, DTYPES[dtype][0])
    return product, dtype, rows, cols, parts > 1


def reached():
    for product in PRODUCTS:
        for dtype in DTYPES:
            for sizes in SHAPES + IN_PARTS:
                yield kind(product, dtype, *sizes)
        for counts, K, O in large.pytestmark[0].args[1]:
            yield kind(product, "bf16", sum(counts) + 8, len(counts), K, O)
    for product, dtype, N, E, K, O, _ in CASES:
        yield kind(product, dtype, N + BEFORE + BEHIND, E, K, O)


def test_every_tile_has_a_test():
    r = random.Random(1)

    def size(most):
        return int(most ** r.random())

    found = {kind(p, d, size(100000), size(2048), 8 * size(1024), 8 * size(1024))
             for _ in range(8000) for p in PRODUCTS for d in DTYPES}
    assert len(found) >= 20
    assert found <= set(reached())


def test_the_tiles_are_those_of_the_cases():
    for product, dtype, N, E, K, O, tile in CASES:
        assert kind(product, dtype, N + BEFORE + BEHIND, E, K, O) == (product, dtype, *tile, False)


def test_refusals():
    good = (pb.BASE_PRODUCT_Y, 64, 2, 64, 64, pb.BASE_BF16)
    assert pb.expert_linear_tile(*good)[2] >= 1
    for i, bad, status in ((0, -1, pb.BASE_ERR_INVALID_ARG), (0, 3, pb.BASE_ERR_INVALID_ARG),
                           (1, 0, pb.BASE_ERR_INVALID_ARG), (3, 12, pb.BASE_ERR_INVALID_ARG),
                           (2, 2049, pb.BASE_ERR_RANGE), (4, (1 << 20) + 8, pb.BASE_ERR_RANGE),
                           (5, pb.BASE_I16, pb.BASE_ERR_UNSUPPORTED_DTYPE)):
        with pytest.raises(pb.BaseError) as err:
            pb.expert_linear_tile(*good[:i], bad, *good[i + 1:])
        assert err.value.status == status
    assert pb.lib().base_expert_linear_tile(*good, None, None, None) == pb.BASE_ERR_INVALID_ARG

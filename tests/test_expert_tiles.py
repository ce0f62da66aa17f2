"""Which tiles the products' sizes lead to: a rule on the host."""
import pytest

import paper_2103_16716_amd as pb
from test_gpu_expert_tiles import BEFORE, BEHIND, CASES, DTYPES, PRODUCTS


def kind(product, dtype, N, E, K, O):
    rows, cols, parts = pb.expert_linear_tile(PRODUCTS[product], N, E, K, O, DTYPES[dtype][0])
    return product, dtype, rows, cols, parts > 1


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

"""Routing with k experts a token at sizes that lead to each form of the choice: 16 or 64 lanes
a token with 4 to 32 scores each, sorted lists of two or eight or rounds, in one block or two
launches."""
import pytest

from test_gpu_experts import test_topk_assign as check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,E,k", [
    # rounds (k > 8) by 16 lanes, in one block and not
    (40, 64, 10), (3000, 64, 16), (30, 100, 12), (700, 128, 9), (20, 250, 20), (900, 250, 20),
    (1, 9, 9), (256, 33, 9), (70, 64, 64),
    # by 64 lanes
    (50, 400, 17), (200, 1000, 33), (9, 1025, 40), (600, 1999, 11),
    # one or two choices, more than 128 experts
    (100, 200, 2), (5000, 256, 1), (60, 500, 2), (600, 512, 2), (3, 2048, 1), (300, 2047, 2),
    (100, 100, 2),
    # three to eight: one token and two tokens by 16 lanes in one block, and by 64 lanes
    (33, 200, 6), (120, 256, 8), (40, 300, 5), (64, 512, 8), (300, 1500, 8), (1025, 1025, 3)])
def test_every_form(T, E, k):
    check(T, E, k)

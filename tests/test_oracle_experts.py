"""Pins of the oracle's expert layer: a hand-worked routing, moves as adjoints,
gradients against central differences, planted mistakes that the pins reject."""
import numpy as np
import pytest

from oracle import experts as ex


def rng_of(seed):
    return np.random.Generator(np.random.PCG64(seed))


def test_routing_by_hand():
    inf, nan = np.inf, np.nan
    S = np.array([[1, 3, 2], [5, 5, 5], [-inf, 0, nan], [-inf, nan, -inf], [0.0, -0.0, inf]])
    a, v = ex.topk(S, 2)
    assert a.tolist() == [[1, 2], [0, 1], [1, -1], [-1, -1], [2, 0]]
    assert v.tolist() == [[3, 2], [5, 5], [0, -inf], [-inf, -inf], [inf, 0]]
    perm, slots, off = ex.sort_pairs(a, 3)
    # pairs 0..9: experts 1 2 0 1 1 - - - 2 0
    assert perm.tolist() == [2, 9, 0, 3, 4, 1, 8, -1, -1, -1]
    assert off.tolist() == [0, 2, 5, 7]
    assert slots.tolist() == [[2, 5], [0, 3], [4, -1], [-1, -1], [6, 1]]


def test_sort_is_stable_and_k1_is_the_sort_vector():
    a = rng_of(0).integers(0, 7, (50, 1))
    perm, slots, off = ex.sort_pairs(a, 7)
    np.testing.assert_array_equal(perm, np.argsort(a[:, 0], kind="stable"))
    np.testing.assert_array_equal(np.diff(off), np.bincount(a[:, 0], minlength=7))
    np.testing.assert_array_equal(perm[slots[:, 0]], np.arange(50))


def test_moves_are_adjoint():
    """<dispatch(x, w), F> = <x, combine(F, w)>, and the backward is its gradient."""
    r = rng_of(1)
    a = r.integers(-1, 4, (9, 3))
    _, slots, _ = ex.sort_pairs(a, 4)
    x, F, w = r.standard_normal((9, 5)), r.standard_normal((27, 5)), r.standard_normal((9, 3))
    left = np.sum(ex.dispatch(x, slots, w) * F)
    assert left == pytest.approx(np.sum(x * ex.combine(F, slots, w)), rel=1e-12)
    dF, dw = ex.combine_backward(x, F, slots, w)
    assert np.sum(dw * w) == pytest.approx(left, rel=1e-12)
    assert np.sum(dF * F) == pytest.approx(left, rel=1e-12)
    assert np.all(dw[slots < 0] == 0)


def differences(f, x, dy, n=12, h=1e-5):
    """Directional derivatives of <f(x), dy> at n random directions, and the directions."""
    r = rng_of(7)
    for _ in range(n):
        v = r.standard_normal(x.shape)
        yield (np.sum((f(x + h * v) - f(x - h * v)) * dy)) / (2 * h), v


def test_gradients_against_differences():
    r = rng_of(2)
    N, E, K, O = 11, 3, 6, 5
    off = np.array([0, 4, 4, 11])
    e = ex.row_experts(off, N)
    x, w, b = r.standard_normal((N, K)), r.standard_normal((E, K)), r.standard_normal((E, K))
    dy = r.standard_normal((N, K))
    dx, dw, db = ex.norm_backward(dy, x, w, e, 1e-5)
    for got, f, at in ((dx, lambda z: ex.norm(z, w, b, e, 1e-5)[0], x),
                       (dw, lambda z: ex.norm(x, z, b, e, 1e-5)[0], w),
                       (db, lambda z: ex.norm(x, w, z, e, 1e-5)[0], b)):
        for want, v in differences(f, at, dy):
            assert np.sum(got * v) == pytest.approx(want, rel=1e-6, abs=1e-7)
    # planted mistakes: the mean's term left out, the weight's gradient of rows one off
    want, v = next(differences(lambda z: ex.norm(z, w, b, e, 1e-5)[0], x, dy))
    assert abs(np.sum((dx + (dy * w[e]).mean(axis=1, keepdims=True)) * v) - want) > 1e-3
    want, v = next(differences(lambda z: ex.norm(x, z, b, e, 1e-5)[0], w, dy))
    off_by_one = ex.norm_backward(dy, x, w, np.roll(e, 1), 1e-5)[1]
    assert abs(np.sum(off_by_one * v) - want) > 1e-3
    W, B, dy = r.standard_normal((E, O, K)), r.standard_normal((E, O)), r.standard_normal((N, O))
    u = np.maximum(x, 0)
    gw, gb = ex.linear_dw(dy, u, e, E)
    for got, f, at in ((ex.linear_dx(dy, W, e, relu_of=u),
                        lambda z: ex.linear(np.maximum(z, 0), W, B, e), x),
                       (gw, lambda z: ex.linear(u, z, B, e), W),
                       (gb, lambda z: ex.linear(u, W, z, e), B)):
        for want, v in differences(f, at, dy):
            assert np.sum(got * v) == pytest.approx(want, rel=1e-6, abs=1e-7)
    assert np.all(gw[1] == 0) and np.all(gb[1] == 0)      # an expert without rows

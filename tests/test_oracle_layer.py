"""Pins of the oracle's whole layer with k experts a token: its gradients against central
differences of the layer computed token by token, along each gradient itself, and mistakes
that both these pins and the bounds of the GPU's results have to reject."""
import numpy as np
import pytest

from layer_common import PARAMETERS, layer_bounds, own_directions
from oracle import experts as ex
from test_gpu_experts import EPS, block_inputs, block_loss

STEP = 1e-5


def inputs(k):
    H, S, p, dOut = block_inputs(T=60, E=5, d=32, inner=64, seed=k)
    f64 = lambda z: np.asarray(z, dtype=np.float64)
    return f64(H), f64(S), {n: f64(v) for n, v in p.items()}, f64(dOut)


def slope(H, S, k, p, dOut, name, v):
    """Central difference of <layer, dOut> along direction v of `name`."""
    at = []
    for h in (STEP, -STEP):
        if name in PARAMETERS:
            at.append(block_loss(H, S, k, {**p, name: p[name] + h * v}, dOut))
        else:
            at.append(block_loss(H + h * v if name == "H" else H, S + h * v if name == "S" else S,
                                 k, p, dOut))
    return (at[0] - at[1]) / (2 * STEP)


@pytest.mark.parametrize("k", [1, 2, 4])
def test_gradients_along_themselves(k):
    """Steps of 10^-5: the difference's own error is about 10^-10 of the slope, 10^-9 by the
    loss's rounding, and of the order of the step where a ReLU switches inside it."""
    H, S, p, dOut = inputs(k)
    c, g = ex.layer_backward(H, S, k, p, dOut, EPS)
    total = (c["out"] * dOut).sum()
    assert block_loss(H, S, k, p, dOut) == pytest.approx(total, rel=1e-10, abs=1e-9)
    seen = set()
    for name, v in own_directions(g):
        seen.add(name)
        want = slope(H, S, k, p, dOut, name, v)
        assert (g[name] * v).sum() == pytest.approx(want, rel=1e-3), name
        for factor in (0.5, 0.9, 1.1, 2.0):   # what is off by a factor, or not there, is seen
            assert not (factor * g[name] * v).sum() == pytest.approx(want, rel=1e-3), name
        assert abs(want) > 0
    assert seen == set(PARAMETERS + (("H", "S") if k > 1 else ("H",)))   # (k = 1: weights are 1)
    if k == 1:
        assert not np.any(g["S"])
    assert not np.any(g["S"][S == -np.inf])


@pytest.mark.parametrize("k", [1, 2, 4])
def test_bounds_reject_mistakes(k):
    """The bounds that the GPU's results are held to pass none of: a factor of 0.9 or 1.1, an
    expert's gradient left out, experts exchanged, a row's gradient added to its neighbour."""
    H, S, p, dOut = inputs(k)
    c, g, bound = layer_bounds(H, S, k, p, dOut)
    assert set(bound) == set(PARAMETERS) | {"out", "w", "H", "S"}

    def passes(name, got):
        return np.all(np.abs(got - g[name]) <= bound[name])

    for name in PARAMETERS + ("w", "H", "S"):
        assert passes(name, g[name])
        if not np.any(g[name]):
            continue
        for factor in (0.9, 1.1):
            assert not passes(name, factor * g[name]), name
        assert not passes(name, np.roll(g[name], 1, axis=0)), name
    for name in PARAMETERS:
        for e in range(len(g[name])):
            if np.any(g[name][e]):
                less = g[name].copy()
                less[e] = 0.0
                assert not passes(name, less), (name, e)
    assert not np.all(np.abs(c["out"] - H) <= bound["out"])

"""Helpers of the tests of a whole layer with k experts a token: how far its fp32 results
may be from the oracle's, and the directions its gradients are differenced along. Nothing
here computes a step of the layer."""
from __future__ import annotations

import numpy as np

from oracle import experts as ex
from test_gpu_experts import EPS, SUM, U, norm_bounds

PARAMETERS = ("g", "b", "W1", "b1", "W2", "b2")


def layer_bounds(H, S, k, p, dOut):
    """(results, gradients, bounds by name) of the layer in fp32: every step's own rounding
    ((n + 3) U for a sum of n products, U for a stored value) and what the errors of its
    operands become. With d and b an operand's value and bound, a product's error is at most
    |d1| b2 + b1 (|d2| + b2). A ReLU may switch where its argument is within its own bound
    of zero; there a gradient may be there or not."""
    c, g = ex.layer_backward(H, S, k, p, dOut, EPS)
    H, dOut = np.asarray(H, dtype=np.float64), np.asarray(dOut, dtype=np.float64)
    q = {n: np.abs(np.asarray(v, dtype=np.float64)) for n, v in p.items()}
    e, token, slots, w = c["e"], c["token"], c["slots"], c["w"]
    E, d, inner = q["W1"].shape[0], H.shape[1], q["W1"].shape[1]
    a = {n: np.abs(v) for n, v in g.items()}
    out = {}

    b_y, _, b_rstd, b_xh = norm_bounds(H[token], p["g"], p["b"], e, EPS, U)
    y = np.abs(c["y"])
    b_u = ex.linear(b_y, q["W1"], None, e)
    b_u = b_u + (d + 3) * U * ex.linear(y + b_y, q["W1"], q["b1"], e) + U * np.abs(c["z"])
    u = c["u"] + b_u
    b_f = ex.linear(b_u, q["W2"], None, e)
    b_f = b_f + (inner + 3) * U * ex.linear(u, q["W2"], q["b2"], e) + U * np.abs(c["f"])
    f = np.abs(c["f"]) + b_f
    # softmax: the difference to the largest score, exp, k terms, a quotient
    v = ex.topk(S, k)[1].astype(np.float64)
    there = v > -np.inf
    far = np.where(there, v.max(axis=1, keepdims=True) - np.where(there, v, 0.0), 0.0)
    b_w = w * (16 + k + far) * U
    out["out"] = ex.combine(b_f, slots, w) + ex.combine(f, slots, b_w) + \
        (k + 3) * U * ex.combine(f, slots, w, np.abs(H))

    n = np.maximum(np.bincount(e, minlength=E), 1)
    of_n = (n + 3) * U
    rows = np.zeros((len(token), d))
    b_df = ex.dispatch(np.abs(dOut), slots, b_w, rows) + 2 * U * a["f"]
    out["w"] = ex.combine_backward(np.abs(dOut), b_f, slots, w, rows)[1] + \
        (d + 2) * U * ex.combine_backward(np.abs(dOut), f, slots, w, rows)[1]

    def by_weights(dy, b_dy, x, b_x):
        one, two = ex.linear_dw(b_dy, x + b_x, e, E), ex.linear_dw(dy, b_x, e, E)
        sums = ex.linear_dw(dy + b_dy, x + b_x, e, E)
        return (one[0] + two[0] + of_n[:, None, None] * sums[0],
                one[1] + of_n[:, None] * sums[1])

    out["W2"], out["b2"] = by_weights(a["f"], b_df, c["u"], b_u)
    whole = np.abs(ex.linear_dx(g["f"], p["W2"], e))
    b_dz = ex.linear_dx(b_df, q["W2"], e)
    b_dz = b_dz + (d + 3) * U * ex.linear_dx(a["f"] + b_df, q["W2"], e) + U * whole
    b_dz = np.where(c["z"] > b_u, b_dz, np.where(c["z"] < -b_u, 0.0, whole + b_dz))
    out["W1"], out["b1"] = by_weights(a["z"], b_dz, y, b_y)
    b_dy = ex.linear_dx(b_dz, q["W1"], e)
    b_dy = b_dy + (inner + 3) * U * ex.linear_dx(a["z"] + b_dz, q["W1"], e) + U * a["y"]

    mean, rs = c["mean"][:, None], c["rstd"][:, None]
    xh = np.abs((H[token] - mean) * rs)
    h, b_h = a["y"] * q["g"][e], b_dy * q["g"][e]
    b_h = b_h + U * h
    s1, s2 = h.mean(axis=1, keepdims=True), (h * xh).mean(axis=1, keepdims=True)
    b_s1 = b_h.mean(axis=1, keepdims=True) + SUM * s1
    b_s2 = (b_h * xh + h * b_xh).mean(axis=1, keepdims=True) + (SUM + 2 * U) * s2
    b_dx = rs * (b_h + b_s1 + xh * b_s2 + b_xh * s2 + 4 * U * (h + s1 + xh * s2)) + \
        (b_rstd / c["rstd"])[:, None] * a["x"] + U * a["x"]
    out["g"], out["b"] = np.zeros((E, d)), np.zeros((E, d))
    np.add.at(out["g"], e, b_dy * xh + a["y"] * b_xh + (of_n[e])[:, None] * a["y"] * xh)
    np.add.at(out["b"], e, b_dy + (of_n[e])[:, None] * a["y"])
    out["H"] = (k + 3) * U * np.abs(dOut)
    np.add.at(out["H"], token, b_dx + (k + 3) * U * a["x"])

    m = a["w"] + (w * a["w"]).sum(axis=1, keepdims=True)
    b_v = b_w * m + w * (out["w"] + (b_w * a["w"] + w * out["w"]).sum(axis=1, keepdims=True)) + \
        (k + 6) * U * w * m
    out["S"] = np.zeros(np.asarray(S).shape)
    for (t, j), i in np.ndenumerate(c["assign"]):
        if i >= 0:
            out["S"][t, i] = b_v[t, j]
    # (products of two bounds that the sums above leave out are below 2 % of them)
    return c, g, {name: 1.02 * b for name, b in out.items()}


def own_directions(grads):
    """(name, direction) along every gradient itself, for parameters one expert at a time:
    the difference along it is the gradient's whole length."""
    for name in PARAMETERS + ("H", "S"):
        g = grads[name]
        for i in range(len(g)) if name in PARAMETERS else [slice(None)]:
            v = np.zeros(g.shape)
            v[i] = g[i]
            if np.any(v):
                yield name, v / np.linalg.norm(v)

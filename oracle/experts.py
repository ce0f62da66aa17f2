"""Oracle (test infrastructure only): routing with k experts a token and the
experts' feed-forward block, forward and backward, in fp64.

The paper's comparison layers send a token to its k best experts; an expert is a
stack of residual blocks of layer norm, projection, ReLU and projection (Sec. 3.1).
Pair p = t k + j is choice j of token t; the routed order lists the pairs expert
after expert, ascending within one (Fig. 2's sort vector with k choices).
Inputs are the exact values the device receives.
"""
from __future__ import annotations

import numpy as np


def topk(S, k):
    """(assign, scores) [T, k]: highest score first, lowest index on ties; -inf and
    NaN are never chosen (assign -1, score -inf)."""
    S = np.asarray(S)
    T, E = S.shape
    a = np.full((T, k), -1, dtype=np.int32)
    v = np.full((T, k), -np.inf, dtype=S.dtype)
    for t in range(T):
        allowed = [e for e in range(E) if S[t, e] > -np.inf]
        best = sorted(allowed, key=lambda e: (-S[t, e], e))[:k]
        a[t, :len(best)] = best
        v[t, :len(best)] = S[t, best]
    return a, v


def sort_pairs(assign, E):
    """(perm, slots, offsets) of choices [T, k]; entries outside [0, E) have no row."""
    a = np.asarray(assign)
    flat = a.reshape(-1).astype(np.int64)
    perm = np.full(flat.size, -1, dtype=np.int32)
    slots = np.full(flat.size, -1, dtype=np.int32)
    offsets = np.zeros(E + 1, dtype=np.int32)
    r = 0
    for e in range(E):
        for p in np.nonzero(flat == e)[0]:
            perm[r], slots[p] = p, r
            r += 1
        offsets[e + 1] = r
    return perm, slots.reshape(a.shape), offsets


def combine(F, slots, weights=None, residual=None):
    """out[t] = residual[t] + sum_j weights[t, j] F[slots[t, j]]."""
    F = np.asarray(F, dtype=np.float64)
    T, k = slots.shape
    out = np.zeros((T, F.shape[1])) if residual is None else np.array(residual, dtype=np.float64)
    for t in range(T):
        for j in range(k):
            if slots[t, j] >= 0:
                w = 1.0 if weights is None else float(weights[t, j])
                out[t] += w * F[slots[t, j]]
    return out


def dispatch(x, slots, weights=None, into=None):
    """into[slots[t, j]] = weights[t, j] x[t], the other rows of `into` as they were."""
    x = np.asarray(x, dtype=np.float64)
    T, k = slots.shape
    out = np.zeros((T * k, x.shape[1])) if into is None else np.array(into, dtype=np.float64)
    for t in range(T):
        for j in range(k):
            if slots[t, j] >= 0:
                out[slots[t, j]] = (1.0 if weights is None else float(weights[t, j])) * x[t]
    return out


def combine_backward(dY, F, slots, weights, into=None):
    """(dF, dweights) of combine."""
    dY, F = np.asarray(dY, dtype=np.float64), np.asarray(F, dtype=np.float64)
    dw = np.zeros(slots.shape)
    for (t, j), r in np.ndenumerate(slots):
        if r >= 0:
            dw[t, j] = dY[t] @ F[r]
    return dispatch(dY, slots, weights, into), dw


def row_experts(offsets, N):
    """Expert of each of N rows, -1 for rows in no range."""
    e = np.full(N, -1, dtype=np.int64)
    for i in range(len(offsets) - 1):
        e[offsets[i]:offsets[i + 1]] = i
    return e


def norm(x, weight, bias, e, eps):
    """Layer norm of rows x with the weights of experts e: (y, mean, rstd)."""
    x = np.asarray(x, dtype=np.float64)
    mean = x.mean(axis=1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(axis=1) + eps)
    xh = (x - mean[:, None]) * rstd[:, None]
    y = xh * np.asarray(weight, dtype=np.float64)[e]
    if bias is not None:
        y = y + np.asarray(bias, dtype=np.float64)[e]
    return y, mean, rstd


def norm_backward(dy, x, weight, e, eps):
    """(dx, dweight, dbias) of norm."""
    dy, x = np.asarray(dy, dtype=np.float64), np.asarray(x, dtype=np.float64)
    w = np.asarray(weight, dtype=np.float64)
    _, mean, rstd = norm(x, w, None, e, eps)
    xh = (x - mean[:, None]) * rstd[:, None]
    h = dy * w[e]
    dx = rstd[:, None] * (h - h.mean(axis=1, keepdims=True)
                          - xh * (h * xh).mean(axis=1, keepdims=True))
    dw, db = np.zeros(w.shape), np.zeros(w.shape)
    np.add.at(dw, e, dy * xh)
    np.add.at(db, e, dy)
    return dx, dw, db


def linear(x, w, bias, e, relu=False, residual=None):
    """y[r] = act(x[r] w[e]^T + bias[e]) + residual[r]."""
    x, w = np.asarray(x, dtype=np.float64), np.asarray(w, dtype=np.float64)
    y = np.zeros((x.shape[0], w.shape[1]))
    for i in np.unique(e):
        r = e == i
        y[r] = x[r] @ w[i].T
    if bias is not None:
        y += np.asarray(bias, dtype=np.float64)[e]
    if relu:
        y = np.where(y < 0, 0.0, y)
    return y if residual is None else y + np.asarray(residual, dtype=np.float64)


def linear_dx(dy, w, e, relu_of=None):
    """dx[r] = dy[r] w[e], 0 where relu_of is not > 0."""
    dy, w = np.asarray(dy, dtype=np.float64), np.asarray(w, dtype=np.float64)
    dx = np.zeros((dy.shape[0], w.shape[2]))
    for i in np.unique(e):
        r = e == i
        dx[r] = dy[r] @ w[i]
    return dx if relu_of is None else np.where(np.asarray(relu_of) > 0, dx, 0.0)


def linear_dw(dy, x, e, E):
    """(dw [E, O, K], db [E, O])."""
    dy, x = np.asarray(dy, dtype=np.float64), np.asarray(x, dtype=np.float64)
    dw, db = np.zeros((E, dy.shape[1], x.shape[1])), np.zeros((E, dy.shape[1]))
    for i in np.unique(e):
        r = e == i
        dw[i] = dy[r].T @ x[r]
        db[i] = dy[r].sum(axis=0)
    return dw, db


def routed_weights(v):
    """Softmax over a token's chosen scores v [T, k]; 0 for a choice of score -inf."""
    v = np.asarray(v, dtype=np.float64)
    top = v.max(axis=1, keepdims=True)
    w = np.exp(v - np.where(top > -np.inf, top, 0.0))
    return w / np.maximum(w.sum(axis=1, keepdims=True), 1e-300)


def layer(H, S, k, p, eps):
    """A layer of such experts, p their parameters g, b, W1, b1, W2, b2:
        out[t] = H[t] + sum_j w[t, j] f_e(H[t]),  e = assign[t, j],
        f_e(h) = W2_e max(W1_e norm_e(h) + b1_e, 0) + b2_e,  w[t] = softmax(scores[t]).
    Every intermediate result, those on routed rows for the n rows there are."""
    H = np.asarray(H, dtype=np.float64)
    assign, scores = topk(S, k)
    perm, slots, offsets = sort_pairs(assign, np.asarray(S).shape[1])
    n = offsets[-1]
    e, token = row_experts(offsets, n), perm[:n] // k
    w = routed_weights(scores)
    y, mean, rstd = norm(H[token], p["g"], p["b"], e, eps)
    z = linear(y, p["W1"], p["b1"], e)
    u = np.maximum(z, 0.0)
    f = linear(u, p["W2"], p["b2"], e)
    return dict(assign=assign, slots=slots, e=e, token=token, w=w, y=y, mean=mean, rstd=rstd, z=z,
                u=u, f=f, out=combine(f, slots, w, H))


def layer_backward(H, S, k, p, dOut, eps):
    """(layer's results, the gradients of <out, dOut> by H, S, w, each parameter and each
    intermediate result, named d and it)."""
    H, dOut = np.asarray(H, dtype=np.float64), np.asarray(dOut, dtype=np.float64)
    c = layer(H, S, k, p, eps)
    e, token, E = c["e"], c["token"], np.asarray(S).shape[1]
    df, dw = combine_backward(dOut, c["f"], c["slots"], c["w"], np.zeros((len(token), H.shape[1])))
    dW2, db2 = linear_dw(df, c["u"], e, E)
    dz = linear_dx(df, p["W2"], e, relu_of=c["u"])
    dW1, db1 = linear_dw(dz, c["y"], e, E)
    dy = linear_dx(dz, p["W1"], e)
    dx, dg, db = norm_backward(dy, H[token], p["g"], e, eps)
    dH = dOut.copy()
    np.add.at(dH, token, dx)
    dv = c["w"] * (dw - (c["w"] * dw).sum(axis=1, keepdims=True))
    dS = np.zeros(np.asarray(S).shape)
    for (t, j), a in np.ndenumerate(c["assign"]):
        if a >= 0:
            dS[t, a] = dv[t, j]
    return c, dict(f=df, w=dw, W2=dW2, b2=db2, z=dz, W1=dW1, b1=db1, y=dy, x=dx, g=dg, b=db, H=dH,
                   S=dS)

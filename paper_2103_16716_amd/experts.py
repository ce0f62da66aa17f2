"""k experts a token and the experts themselves: routing; row moves, layer norm
and products on routed rows, and their gradients.

    r = topk_assign(S, 2)                       # 2 experts a token, rows by expert
    y, mean, rstd = expert_norm(H, g, b, r.offsets, perm=r.perm, k=2)
    u = expert_linear(y, W1, r.offsets, bias=b1, relu=True)
    f = expert_linear(u, W2, r.offsets, bias=b2)
    some = r.assign[:, :1] >= 0                 # (a softmax over no expert at all is NaN)
    weights = torch.softmax(r.scores.where(some, 0.0), 1)
    out = combine(f, r.slots, weights=weights, residual=H)

and back, for an upstream dOut:

    df, dweights = combine_backward(dOut, f, r.slots, weights)
    dW2, db2 = expert_linear_dw(df, u, r.offsets)
    du = expert_linear_dx(df, W2, r.offsets, relu_of=u)
    dW1, db1 = expert_linear_dw(du, y, r.offsets)
    dy = expert_linear_dx(du, W1, r.offsets)
    dx, dg, db = expert_norm_backward(dy, H, g, mean, rstd, r.offsets, perm=r.perm, k=2)
    dH = combine(dx, r.slots, residual=dOut)
    ds = weights * (dweights - (weights * dweights).sum(1, keepdim=True))
    dS = torch.zeros_like(S).scatter_add_(1, r.assign.clamp(min=0).long(), ds)

A token without an expert has scores of -inf, weights that nothing uses and dweights of 0;
so have the choices that a token has no expert for, and their ds is 0.

Marshals torch tensors into the C calls of include/base.h. Tensors are contiguous
and, as `stream`, on the current device. Work goes to the current stream, or to `stream`, in
whose memory pool outputs that are not given are then allocated. Rows that no pair
has (behind offsets[-1]) are left as they are in outputs that are given, and are
unspecified in ones that are not.
"""
from __future__ import annotations

import contextlib
import ctypes
import dataclasses

from . import (BASE_PRODUCT_DW, BASE_PRODUCT_DX, BASE_PRODUCT_Y, _check, _dtype_code, _stream_ptr,
               _torch, lib)


@dataclasses.dataclass
class Routing:
    assign: object      # int32 [T, k], -1: no expert
    scores: object      # float32 [T, k] (None from sort_by_expert)
    perm: object        # int32 [T k]: pair t k + j of each routed row
    slots: object       # int32 [T, k]: routed row of each pair, -1: none
    offsets: object     # int32 [E + 1]: expert e's rows are [offsets[e], offsets[e + 1])


def _need(**tensors) -> None:
    """Every given tensor contiguous and on the current device."""
    here = -1
    for t in tensors.values():
        if t is None:
            continue
        d = t.get_device()
        if d != here or d < 0:
            if here < 0 <= d:
                here = _torch().cuda.current_device()
            if d != here or d < 0:
                _refuse(tensors, here)
        if not t.is_contiguous():
            _refuse(tensors, here)


def _refuse(tensors, here) -> None:
    for name, t in tensors.items():
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError(f"{name} must be on the GPU")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        if t.get_device() != here:
            raise ValueError(f"{name} is on {t.device}, the current device is cuda:{here}")


def _empty(rows, cols, dtype, device):
    return _torch().empty_strided((rows, cols), (cols, 1), dtype=dtype, device=device)


def _like(name, t, shape, dtype) -> None:
    if t is not None and (t.shape != shape or t.dtype != dtype):
        raise ValueError(f"{name} must be {dtype} {list(shape)}, not {t.dtype} {list(t.shape)}")


def _dims(name, t, n) -> None:
    if t.dim() != n:
        raise ValueError(f"{name} must have {n} dimensions")


def _on(stream):
    """Where outputs are allocated: the pool of the stream that writes them."""
    if stream is None:
        return _current
    torch = _torch()
    here = torch.cuda.current_device()
    if stream.device_index != here:
        raise ValueError(f"stream is on cuda:{stream.device_index}, the current device is "
                         f"cuda:{here}")
    return torch.cuda.stream(stream)


_current = contextlib.nullcontext()


def _ptr(t):
    return None if t is None else t.data_ptr()


def _workspace(nbytes, device):
    torch = _torch()
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


def topk_workspace_size(T: int, E: int, k: int) -> int:
    return int(lib().base_topk_workspace_size(T, E, k))


def _routing(T, E, k, dev, out_perm, out_slots, out_offsets, out_assign=None, choose=False):
    """assign (if choose), perm, slots and offsets: those given, the others cut from one
    allocation (a small call's time is the host's)."""
    torch = _torch()
    i32 = torch.int32
    if out_perm is None and out_slots is None and out_offsets is None and out_assign is None:
        n = T * k
        buf = torch.empty((3 if choose else 2) * n + E + 1, dtype=i32, device=dev)
        assign = buf.as_strided((T, k), (k, 1), 2 * n + E + 1) if choose else None
        return (assign, buf.as_strided((n,), (1,), 0), buf.as_strided((T, k), (k, 1), n),
                buf.as_strided((E + 1,), (1,), 2 * n))
    _need(out_perm=out_perm, out_slots=out_slots, out_offsets=out_offsets, out_assign=out_assign)
    out = []
    for name, t, shape in (("out_assign", out_assign, (T, k)), ("out_perm", out_perm, (T * k,)),
                           ("out_slots", out_slots, (T, k)),
                           ("out_offsets", out_offsets, (E + 1,))):
        if t is None and (choose or name != "out_assign"):
            t = torch.empty(shape, dtype=i32, device=dev)
        _like(name, t, shape, i32)
        out.append(t)
    return out


def topk_assign(S, k: int, workspace=None, stream=None, out_assign=None, out_scores=None,
                out_perm=None, out_slots=None, out_offsets=None) -> Routing:
    """The k best experts of each row of S (float32 [T, E]), highest first, lowest
    index on ties, never one of score -inf or NaN; and the sort of the pairs by
    expert (base_topk_assign)."""
    torch = _torch()
    _need(S=S, out_scores=out_scores, workspace=workspace)
    _dims("S", S, 2)
    if S.dtype != torch.float32:
        raise TypeError("S must be float32")
    T, E = S.shape
    k = int(k)
    if not 0 < k <= min(E, 64):
        raise ValueError(f"k must be in 1 .. {min(E, 64)}")
    with _on(stream):
        dev = S.device
        assign, perm, slots, offsets = _routing(T, E, k, dev, out_perm, out_slots, out_offsets,
                                                out_assign, True)
        _like("out_scores", out_scores, (T, k), torch.float32)
        scores = out_scores
        if scores is None:
            scores = _empty(T, k, torch.float32, dev)
        ws = workspace
        if ws is None:
            ws = _workspace(topk_workspace_size(T, E, k), dev)
        _check(lib().base_topk_assign(S.data_ptr(), T, E, k, assign.data_ptr(), scores.data_ptr(),
                                      perm.data_ptr(), slots.data_ptr(), offsets.data_ptr(),
                                      ws.data_ptr(), ws.nbytes, _stream_ptr(stream)),
               "base_topk_assign")
    return Routing(assign, scores, perm, slots, offsets)


def sort_by_expert(assign, E: int, workspace=None, stream=None, out_perm=None, out_slots=None,
                   out_offsets=None) -> Routing:
    """The sort of topk_assign for given choices, int32 [T, k] (or [T]: one
    choice); entries outside [0, E) have no expert (base_sort_by_expert)."""
    torch = _torch()
    _need(assign=assign, workspace=workspace)
    if assign.dtype != torch.int32:
        raise TypeError("assign must be int32")
    if assign.dim() == 1:
        assign = assign.unsqueeze(1)
    _dims("assign", assign, 2)
    T, k = assign.shape
    E = int(E)
    with _on(stream):
        _, perm, slots, offsets = _routing(T, E, k, assign.device, out_perm, out_slots,
                                           out_offsets)
        ws = workspace
        if ws is None:
            ws = _workspace(topk_workspace_size(T, E, k), assign.device)
        _check(lib().base_sort_by_expert(assign.data_ptr(), T, E, k, perm.data_ptr(),
                                         slots.data_ptr(), offsets.data_ptr(), ws.data_ptr(),
                                         ws.nbytes, _stream_ptr(stream)),
               "base_sort_by_expert")
    return Routing(assign, None, perm, slots, offsets)


def _slots_of(slots, weights, **others):
    torch = _torch()
    _need(slots=slots, weights=weights, **others)
    _dims("slots", slots, 2)
    if slots.dtype != torch.int32:
        raise TypeError("slots must be int32")
    _like("weights", weights, slots.shape, torch.float32)
    return slots.shape


def dispatch(x, slots, weights=None, out=None, stream=None):
    """Token rows to their routed rows, out[slots[t, j]] = weights[t, j] x[t]
    (base_dispatch); out has T k rows. Without weights a copy bit for bit, the
    gradient of combine without weights."""
    torch = _torch()
    T, k = _slots_of(slots, weights, x=x, out=out)
    _dims("x", x, 2)
    d = x.shape[1]
    _like("x", x, (T, d), x.dtype)
    _like("out", out, (T * k, d), x.dtype)
    with _on(stream):
        if out is None:
            out = _empty(T * k, d, x.dtype, x.device)
        _check(lib().base_dispatch(x.data_ptr(), _ptr(weights), slots.data_ptr(), out.data_ptr(),
                                   T, k, d, _dtype_code(x), _stream_ptr(stream)), "base_dispatch")
    return out


def combine(F, slots, weights=None, residual=None, out=None, stream=None):
    """Routed rows back to their tokens, out[t] = residual[t] + sum over j of
    weights[t, j] F[slots[t, j]] (base_combine). Pairs without a row add nothing."""
    torch = _torch()
    T, k = _slots_of(slots, weights, F=F, residual=residual, out=out)
    _dims("F", F, 2)
    d = F.shape[1]
    _like("F", F, (T * k, d), F.dtype)
    _like("residual", residual, (T, d), F.dtype)
    _like("out", out, (T, d), F.dtype)
    with _on(stream):
        if out is None:
            out = _empty(T, d, F.dtype, F.device)
        _check(lib().base_combine(F.data_ptr(), _ptr(weights), slots.data_ptr(), _ptr(residual),
                                  out.data_ptr(), T, k, d, _dtype_code(F), _stream_ptr(stream)),
               "base_combine")
    return out


def combine_backward(dY, F, slots, weights, out=None, stream=None):
    """Gradient of combine with weights (base_combine_backward): (dF in routed
    order, dweights [T, k]). The residual's gradient is dY."""
    torch = _torch()
    T, k = _slots_of(slots, weights, dY=dY, F=F, out=out)
    _dims("F", F, 2)
    d = F.shape[1]
    _like("F", F, (T * k, d), F.dtype)
    _like("dY", dY, (T, d), F.dtype)
    _like("out", out, (T * k, d), F.dtype)
    if weights is None:
        raise ValueError("weights are needed (without them the gradient is dispatch(dY, slots))")
    with _on(stream):
        if out is None:
            out = torch.empty_like(F)
        dw = _empty(T, k, torch.float32, F.device)
        _check(lib().base_combine_backward(dY.data_ptr(), F.data_ptr(), weights.data_ptr(),
                                           slots.data_ptr(), out.data_ptr(), dw.data_ptr(), T, k,
                                           d, _dtype_code(F), _stream_ptr(stream)),
               "base_combine_backward")
    return out, dw


def _norm_args(x, weight, offsets, perm, k, **others):
    """(N, E, d) of a norm's arguments."""
    torch = _torch()
    _need(x=x, weight=weight, offsets=offsets, perm=perm, **others)
    _dims("x", x, 2)
    d = x.shape[1]
    if weight.dim() == 1:
        weight = weight.unsqueeze(0)
    E = weight.shape[0]
    _like("weight", weight, (E, d), x.dtype)
    _like("offsets", offsets, (E + 1,), torch.int32)
    if offsets is None and E != 1:
        raise ValueError("weights of several experts need offsets")
    if perm is None and k != 1:
        raise ValueError("k needs perm")
    if perm is not None:
        _dims("perm", perm, 1)
        _like("perm", perm, perm.shape, torch.int32)
    return (x.shape[0] if perm is None else perm.shape[0]), E, d


def expert_norm(x, weight, bias=None, offsets=None, eps: float = 1e-5, perm=None, k: int = 1,
                out=None, stream=None):
    """Layer norm of routed rows with their experts' weights [E, d] (base_expert_norm):
    (y, mean, rstd). With perm, routed row r is row perm[r] // k of x. Without
    offsets one norm, weight [d] or [1, d], for every row."""
    torch = _torch()
    N, E, d = _norm_args(x, weight, offsets, perm, k, bias=bias, out=out)
    if bias is not None:
        _like("bias", bias, weight.shape, x.dtype)
    _like("out", out, (N, d), x.dtype)
    with _on(stream):
        if out is None:
            out = _empty(N, d, x.dtype, x.device)
        mean = torch.empty(N, dtype=torch.float32, device=x.device)
        rstd = torch.empty(N, dtype=torch.float32, device=x.device)
        _check(lib().base_expert_norm(x.data_ptr(), _ptr(perm), x.shape[0], k, weight.data_ptr(),
                                      _ptr(bias), _ptr(offsets), out.data_ptr(), mean.data_ptr(),
                                      rstd.data_ptr(), N, E, d, float(eps), _dtype_code(x),
                                      _stream_ptr(stream)), "base_expert_norm")
    return out, mean, rstd


def expert_norm_workspace_size(N: int, E: int, d: int) -> int:
    return int(lib().base_expert_norm_workspace_size(N, E, d))


def expert_norm_backward(dy, x, weight, mean, rstd, offsets=None, perm=None, k: int = 1,
                         residual=None, out=None, workspace=None, stream=None):
    """Gradient of expert_norm (base_expert_norm_backward): (dx, dweight, dbias), dx
    in routed order with `residual` added, the others float32 of weight's shape."""
    torch = _torch()
    N, E, d = _norm_args(x, weight, offsets, perm, k, dy=dy, mean=mean, rstd=rstd,
                         residual=residual, out=out, workspace=workspace)
    _like("dy", dy, (N, d), x.dtype)
    _like("mean", mean, (N,), torch.float32)
    _like("rstd", rstd, (N,), torch.float32)
    _like("residual", residual, (N, d), x.dtype)
    _like("out", out, (N, d), x.dtype)
    with _on(stream):
        if out is None:
            out = _empty(N, d, x.dtype, x.device)
        dweight = torch.empty(weight.shape, dtype=torch.float32, device=x.device)
        dbias = torch.empty(weight.shape, dtype=torch.float32, device=x.device)
        ws = workspace
        if ws is None:
            ws = _workspace(expert_norm_workspace_size(N, E, d), x.device)
        _check(lib().base_expert_norm_backward(
            dy.data_ptr(), x.data_ptr(), _ptr(perm), x.shape[0], k, weight.data_ptr(),
            mean.data_ptr(), rstd.data_ptr(), _ptr(offsets), _ptr(residual), out.data_ptr(),
            dweight.data_ptr(), dbias.data_ptr(), N, E, d, _dtype_code(x), ws.data_ptr(),
            ws.nbytes, _stream_ptr(stream)), "base_expert_norm_backward")
    return out, dweight, dbias


def expert_linear_workspace_size(product: int, N: int, E: int, K: int, O: int, dtype: int) -> int:
    """Bytes for a BASE_PRODUCT_* of these sizes and BASE_* type; 0 for most."""
    return int(lib().base_expert_linear_workspace_size(product, N, E, K, O, dtype))


def expert_linear_tile(product: int, N: int, E: int, K: int, O: int, dtype: int):
    """(rows, columns, parts): the tiles and the parts of the sum that a BASE_PRODUCT_* of
    these sizes and BASE_* type is computed in (base_expert_linear_tile)."""
    out = (ctypes.c_int32 * 3)()
    at = ctypes.addressof(out)
    _check(lib().base_expert_linear_tile(product, N, E, K, O, dtype, at, at + 4, at + 8),
           "base_expert_linear_tile")
    return tuple(out)


def _linear_workspace(workspace, product, N, E, K, O, dtype, device):
    """(tensor or None, address, bytes)."""
    if workspace is None:
        n = expert_linear_workspace_size(product, N, E, K, O, dtype)
        if n == 0:
            return None, None, 0
        workspace = _workspace(n, device)
    return workspace, workspace.data_ptr(), workspace.nbytes


def _linear_args(w, offsets, **others):
    torch = _torch()
    _need(w=w, offsets=offsets, **others)
    _dims("w", w, 3)
    E, O, K = w.shape
    _like("offsets", offsets, (E + 1,), torch.int32)
    return E, O, K


def expert_linear(x, w, offsets, bias=None, relu: bool = False, residual=None, out=None,
                  workspace=None, stream=None):
    """Routed rows x [N, K] times their experts' matrices w [E, O, K]: y = act(x w^T +
    bias) + residual, act the ReLU with `relu` (base_expert_linear)."""
    torch = _torch()
    E, O, K = _linear_args(w, offsets, x=x, bias=bias, residual=residual, out=out,
                           workspace=workspace)
    _dims("x", x, 2)
    N = x.shape[0]
    _like("x", x, (N, K), w.dtype)
    _like("bias", bias, (E, O), w.dtype)
    _like("residual", residual, (N, O), w.dtype)
    _like("out", out, (N, O), w.dtype)
    with _on(stream):
        if out is None:
            out = _empty(N, O, x.dtype, x.device)
        code = _dtype_code(x)
        ws, at, n = _linear_workspace(workspace, BASE_PRODUCT_Y, N, E, K, O, code, x.device)
        _check(lib().base_expert_linear(x.data_ptr(), w.data_ptr(), _ptr(bias), _ptr(residual),
                                        offsets.data_ptr(), out.data_ptr(), N, E, K, O,
                                        1 if relu else 0, code, at, n, _stream_ptr(stream)),
               "base_expert_linear")
    return out


def expert_linear_dx(dy, w, offsets, relu_of=None, out=None, workspace=None, stream=None):
    """Gradient of expert_linear by its rows, dy w (base_expert_linear_dx). With relu_of
    (the ReLU's result that was x) the gradient before that ReLU: 0 where it is not > 0."""
    torch = _torch()
    E, O, K = _linear_args(w, offsets, dy=dy, relu_of=relu_of, out=out, workspace=workspace)
    _dims("dy", dy, 2)
    N = dy.shape[0]
    _like("dy", dy, (N, O), w.dtype)
    _like("relu_of", relu_of, (N, K), w.dtype)
    _like("out", out, (N, K), w.dtype)
    with _on(stream):
        if out is None:
            out = _empty(N, K, dy.dtype, dy.device)
        code = _dtype_code(dy)
        ws, at, n = _linear_workspace(workspace, BASE_PRODUCT_DX, N, E, K, O, code, dy.device)
        _check(lib().base_expert_linear_dx(dy.data_ptr(), w.data_ptr(), _ptr(relu_of),
                                           offsets.data_ptr(), out.data_ptr(), N, E, K, O, code,
                                           at, n, _stream_ptr(stream)),
               "base_expert_linear_dx")
    return out


def expert_linear_dw(dy, x, offsets, workspace=None, stream=None):
    """Gradient of expert_linear by its matrices and bias (base_expert_linear_dw):
    (dw float32 [E, O, K], db float32 [E, O]), summed over each expert's rows."""
    torch = _torch()
    _need(dy=dy, x=x, offsets=offsets, workspace=workspace)
    _dims("dy", dy, 2)
    _dims("x", x, 2)
    _dims("offsets", offsets, 1)
    (N, O), K, E = dy.shape, x.shape[1], offsets.shape[0] - 1
    _like("x", x, (N, K), dy.dtype)
    _like("offsets", offsets, (E + 1,), torch.int32)
    with _on(stream):
        dw = torch.empty((E, O, K), dtype=torch.float32, device=dy.device)
        db = _empty(E, O, torch.float32, dy.device)
        code = _dtype_code(dy)
        ws, at, n = _linear_workspace(workspace, BASE_PRODUCT_DW, N, E, K, O, code, dy.device)
        _check(lib().base_expert_linear_dw(dy.data_ptr(), x.data_ptr(), offsets.data_ptr(),
                                           dw.data_ptr(), db.data_ptr(), N, E, K, O, code, at, n,
                                           _stream_ptr(stream)),
               "base_expert_linear_dw")
    return dw, db

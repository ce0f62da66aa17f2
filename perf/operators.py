"""Measured cases of an expert layer around the routing: k experts a token,
the experts' layer norm and the experts' products.

A mixture-of-experts layer with k experts a token picks them from the scores
and sorts the pairs by expert (topk_assign), moves the token rows into that
order and back with weights, and in training takes the gradient of both
(dispatch, combine, combine_backward). The experts are feed-forward blocks:
a layer norm whose weights are the expert's own (expert_norm and its backward
pass), then products with the expert's matrices (expert_linear, and in training
expert_linear_dx and expert_linear_dw). Routed rows stand expert after expert;
expert e's are [offsets[e], offsets[e + 1]), and offsets live on the GPU.

T tokens, E experts, k experts a token, N = T k routed rows, width d; the
products take K inputs to O outputs. Sizes are the package's workloads, the
ranges around them and the four-fold inner width of the experts.

With `own` false every operator is computed in its plain form from elementary
torch operations; with `own` true by this package.
"""
from __future__ import annotations

import torch

own = False
DEV = "cuda"
KINDS = ("route", "move", "norm", "linear")
EPS = 1e-5


def listed():
    return [
        # Serving: one step of 48 running sequences, top-2 of 64 experts.
        dict(name="route-decode", kind="route", T=48, E=64, k=2, masked=False),
        # A training batch: 32768 tokens, top-2 of 128 experts.
        dict(name="route-train", kind="route", T=32768, E=128, k=2, masked=False),
        # The widest routing: eight of 256 experts, a padded batch (tokens
        # behind a sequence's end have no expert).
        dict(name="route-wide", kind="route", T=65536, E=256, k=8, masked=True),
        # A training step's rows to the experts and back, with the gradients.
        dict(name="move-train", kind="move", T=32768, E=128, k=2, d=2048, dtype="bf16",
             masked=False),
        # The same in fp32 at odd sizes, with padded tokens.
        dict(name="move-ragged", kind="move", T=6001, E=100, k=3, d=1000, dtype="f32",
             masked=True),
        # Serving: the layer norm of the 96 routed rows of 48 tokens, read
        # through the sort vector.
        dict(name="norm-decode", kind="norm", N=96, E=64, k=2, d=1024, dtype="bf16",
             train=False, gather=True, shared=False),
        # A training step: each expert's norm and its backward pass.
        dict(name="norm-train", kind="norm", N=32768, E=128, k=1, d=2048, dtype="bf16",
             train=True, gather=False, shared=False),
        # One norm for all rows, in fp32, at the widest model dimension.
        dict(name="norm-shared", kind="norm", N=16384, E=1, k=1, d=4096, dtype="f32",
             train=True, gather=False, shared=True),
        # Serving: 64 rows through the first product of 64 experts (width
        # 1024, inner width 4096), where the weights' bytes count.
        dict(name="linear-decode", kind="linear", N=64, E=64, K=1024, O=4096, dtype="bf16",
             train=False, relu=True, residual=False),
        # A training batch through the first product of 32 experts.
        dict(name="linear-train", kind="linear", N=32768, E=32, K=2048, O=8192, dtype="bf16",
             train=False, relu=True, residual=False),
        # The gradients of the second product (inner width back to the model's).
        dict(name="linear-grad", kind="linear", N=16384, E=16, K=8192, O=2048, dtype="bf16",
             train=True, relu=True, residual=False),
        # fp32, sizes that fill no tile: the second product with its residual,
        # forward and backward.
        dict(name="linear-ragged", kind="linear", N=1501, E=10, K=2056, O=520, dtype="f32",
             train=True, relu=False, residual=True),
    ]


def _log_int(rng, lo, hi):
    """A whole number of [lo, hi], even over its logarithm."""
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(KINDS)
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    E = _log_int(rng, 4, 256)
    if kind == "route":
        return dict(kind=kind, T=_log_int(rng, 1, 65536), E=E, k=rng.randint(1, min(8, E)),
                    masked=rng.random() < 0.5)
    if kind == "move":
        k = rng.randint(1, min(8, E))
        d = 8 * _log_int(rng, 16, 512)
        most = 32768 * 2 * 2048 // (k * d * (2 if dtype == "f32" else 1))
        return dict(kind=kind, T=_log_int(rng, 1, min(32768, most)), E=E, k=k, d=d, dtype=dtype,
                    masked=rng.random() < 0.5)
    if kind == "norm":
        shared = rng.random() < 0.25
        gather = rng.random() < 0.4
        k = rng.randint(1, 2) if gather else 1
        d = 8 * _log_int(rng, 16, 512)
        most = 32768 * 2048 // (d * (2 if dtype == "f32" else 1))
        return dict(kind=kind, N=k * _log_int(rng, 1, min(32768, most) // k),
                    E=1 if shared else E, k=k, d=d, dtype=dtype, train=rng.random() < 0.6,
                    gather=gather, shared=shared)
    E = _log_int(rng, 2, 64)
    K = 8 * _log_int(rng, 16, 1024)
    O = 8 * _log_int(rng, 16, min(1024, 32 * 2048 * 1024 // (E * K)))
    train = rng.random() < 0.5
    # fp32 products run at about an eighth of the bf16 rate
    most = 32768 * 2048 * 8192 // (K * O * (2 if train else 1) * (8 if dtype == "f32" else 1))
    return dict(kind=kind, N=_log_int(rng, 1, min(32768, most)), E=E, K=K, O=O, dtype=dtype,
                train=train, relu=rng.random() < 0.5, residual=rng.random() < 0.3)


# ------------------------------------------------------------------ inputs --

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) + 2103_16716)
    return g


def _randn(shape, g, dtype="f32", scale=1.0):
    """N(0, scale^2), drawn in fp32 and rounded to the storage type."""
    x = torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)
    if scale != 1.0:
        x *= scale
    return x.to(torch.bfloat16) if dtype == "bf16" else x


def _scores(T, E, g, masked):
    """Unit-variance scores with some experts liked more than others. masked:
    about a tenth of the tokens are padding and have no expert, and a tenth of
    the others may not use the first half of the experts."""
    S = torch.randn((T, E), generator=g, device=DEV)
    S += 0.5 * torch.randn((E,), generator=g, device=DEV)
    if masked:
        u = torch.rand((T,), generator=g, device=DEV)
        S[(u >= 0.1) & (u < 0.2), :E // 2] = float("-inf")
        S[u < 0.1] = float("-inf")
    return S


def _offsets(N, E, g):
    """Row ranges of N rows that choose among E experts, unevenly."""
    p = torch.softmax(0.5 * torch.randn((E,), generator=g, device=DEV), dim=0)
    e = torch.multinomial(p, N, replacement=True, generator=g)
    off = torch.zeros(E + 1, dtype=torch.int32, device=DEV)
    off[1:] = torch.cumsum(torch.bincount(e, minlength=E), dim=0).to(torch.int32)
    return off


def prepare(case, seed):
    if own:
        import paper_2103_16716_amd as pb
    g = _gen(seed)
    kind = case["kind"]
    st = dict(case=case)
    if kind == "route":
        T, E, k = case["T"], case["E"], case["k"]
        st["S"] = _scores(T, E, g, case["masked"])
        if own:
            st["ws"] = torch.empty(pb.topk_workspace_size(T, E, k), dtype=torch.uint8, device=DEV)
        return st
    dt = case["dtype"]
    if kind == "move":
        T, E, k, d = case["T"], case["E"], case["k"], case["d"]
        r = _plain_route(_scores(T, E, g, case["masked"]), k)
        st["perm"], st["slots"] = r["perm"], r["slots"]
        st["w"] = torch.softmax(r["scores"], dim=1).nan_to_num_(0.0)
        st["x"], st["dY"] = _randn((T, d), g, dt), _randn((T, d), g, dt)
        st["F"], st["dX"] = _randn((T * k, d), g, dt), _randn((T * k, d), g, dt)
        # Routed rows that no token has (padding) keep what the buffers hold.
        st["X"], st["dF"] = torch.zeros_like(st["F"]), torch.zeros_like(st["F"])
        return st
    if kind == "norm":
        N, E, k, d = case["N"], case["E"], case["k"], case["d"]
        st["offsets"] = None if case["shared"] else _offsets(N, E, g)
        st["perm"] = None
        if case["gather"]:
            st["perm"] = torch.randperm(N, generator=g, device=DEV).to(torch.int32)
        x = _randn((N // k, d), g, "f32") + 0.5 * _randn((N // k, 1), g, "f32")
        st["x"] = x.to(torch.bfloat16) if dt == "bf16" else x
        st["weight"] = (1.0 + 0.1 * _randn((E, d), g)).to(st["x"].dtype)
        st["bias"] = _randn((E, d), g, dt, 0.1)
        if case["train"]:
            st["dy"] = _randn((N, d), g, dt)
        if own and case["train"]:
            st["ws"] = torch.empty(pb.expert_norm_workspace_size(N, E, d), dtype=torch.uint8,
                                   device=DEV)
        return st
    N, E, K, O = case["N"], case["E"], case["K"], case["O"]
    st["offsets"] = _offsets(N, E, g)
    st["w"] = _randn((E, O, K), g, dt, K ** -0.5)
    st["x"] = _randn((N, K), g, dt)
    if case["train"]:
        st["dy"] = _randn((N, O), g, dt)
        if case["relu"]:   # x is the result of the product before, and its ReLU's
            st["x"].clamp_(min=0)
    if not case["train"] or case["residual"]:
        st["bias"] = _randn((E, O), g, dt, 0.1)
    st["residual"] = _randn((N, O), g, dt) if case["residual"] else None
    return st


# ------------------------------------------------------------- plain forms --

def _plain_route(S, k):
    """The k best experts of each token, lowest index on ties, -inf and NaN
    never chosen; the pairs sorted by expert, in order within an expert."""
    T, E = S.shape
    s = torch.where(S == S, S, float("-inf"))
    col = torch.arange(E, device=S.device)
    assign = torch.empty((T, k), dtype=torch.int64, device=S.device)
    scores = torch.empty((T, k), dtype=torch.float32, device=S.device)
    for j in range(k):
        best = s.amax(dim=1)
        e = torch.where(s == best[:, None], col, E).amin(dim=1)
        scores[:, j] = best
        assign[:, j] = torch.where(best == float("-inf"), -1, e)
        s = torch.where(col == e[:, None], float("-inf"), s)
    flat = assign.view(-1)
    key = torch.where(flat < 0, E, flat)
    order = torch.sort(key, stable=True).indices
    offsets = torch.searchsorted(key[order], torch.arange(E + 1, device=S.device))
    row = torch.arange(T * k, device=S.device)
    here = row < offsets[E]
    perm = torch.where(here, order, -1)
    slots = torch.empty_like(row)
    slots[order] = torch.where(here, row, -1)
    i32 = torch.int32
    return dict(assign=assign.to(i32), scores=scores, perm=perm.to(i32),
                slots=slots.view(T, k).to(i32), offsets=offsets.to(i32))


def _plain_dispatch(x, slots, into):
    out = into.clone()
    for j in range(slots.shape[1]):
        sel = slots[:, j] >= 0
        out[slots[sel, j].long()] = x[sel]
    return out


def _plain_combine(F, slots, w, residual):
    y = residual.float()
    for j in range(slots.shape[1]):
        s = slots[:, j]
        f = F[torch.where(s < 0, 0, s.long())].float()
        if w is not None:
            f = f * w[:, j, None]
        y = y + torch.where((s >= 0)[:, None], f, 0.0)
    return y.to(residual.dtype)


def _plain_combine_backward(dY, F, slots, w, into):
    dF, dw = into.clone(), torch.zeros_like(w)
    for j in range(slots.shape[1]):
        s = slots[:, j]
        sel = s >= 0
        r = torch.where(sel, s.long(), 0)
        dw[:, j] = torch.where(sel, (dY.float() * F[r].float()).sum(dim=1), 0.0)
        dF[r[sel]] = (w[:, j, None] * dY.float()).to(dF.dtype)[sel]
    return dF, dw


def _row_experts(offsets, N):
    row = torch.arange(N, device=DEV, dtype=torch.int32)
    return torch.searchsorted(offsets[1:], row, right=True)


def _plain_norm(st):
    case = st["case"]
    N, E, k = case["N"], case["E"], case["k"]
    e = (torch.zeros(N, dtype=torch.int64, device=DEV) if st["offsets"] is None
         else _row_experts(st["offsets"], N))
    x = st["x"] if st["perm"] is None else st["x"][st["perm"].long() // k]
    x = x.float()
    mean = x.mean(dim=1)
    c = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((c * c).mean(dim=1) + EPS)
    xh = c * rstd[:, None]
    w = st["weight"].float()[e]
    y = (xh * w + st["bias"].float()[e]).to(st["x"].dtype)
    if not case["train"]:
        return dict(y=y, mean=mean, rstd=rstd)
    dy = st["dy"].float()
    g = dy * w
    dx = rstd[:, None] * (g - g.mean(dim=1)[:, None] - xh * (g * xh).mean(dim=1)[:, None])
    hot = (e == torch.arange(E, device=DEV)[:, None]).float()
    return dict(y=y, mean=mean, rstd=rstd, dx=dx.to(st["x"].dtype), dweight=hot @ (dy * xh),
                dbias=hot @ dy)


def _plain_linear(st):
    case = st["case"]
    N, E, K, O = case["N"], case["E"], case["K"], case["O"]
    x, w, dt = st["x"], st["w"], st["x"].dtype
    off = st["offsets"].tolist()
    forward = not case["train"] or case["residual"]
    out = {}
    if forward:
        out["y"] = torch.empty((N, O), dtype=dt, device=DEV)
    if case["train"]:
        out["dx"] = torch.empty((N, K), dtype=dt, device=DEV)
        out["dw"] = torch.zeros((E, O, K), device=DEV)
        out["db"] = torch.zeros((E, O), device=DEV)
    for e in range(E):
        r = slice(off[e], off[e + 1])
        if off[e] == off[e + 1]:
            continue
        we, xe = w[e].float(), x[r].float()
        if forward:
            y = xe @ we.t() + st["bias"][e].float()
            if case["relu"]:
                y = y.clamp(min=0)
            if st["residual"] is not None:
                y = y + st["residual"][r].float()
            out["y"][r] = y.to(dt)
        if case["train"]:
            dy = st["dy"][r].float()
            dx = dy @ we
            if case["relu"]:
                dx = torch.where(x[r] > 0, dx, 0.0)
            out["dx"][r] = dx.to(dt)
            out["dw"][e] = dy.t() @ xe
            out["db"][e] = dy.sum(dim=0)
    return out


def _plain(st):
    case = st["case"]
    if case["kind"] == "route":
        return _plain_route(st["S"], case["k"])
    if case["kind"] == "move":
        X = _plain_dispatch(st["x"], st["slots"], st["X"])
        Y = _plain_combine(st["F"], st["slots"], st["w"], st["x"])
        dF, dw = _plain_combine_backward(st["dY"], st["F"], st["slots"], st["w"], st["dF"])
        return dict(X=X, Y=Y, dF=dF, dw=dw,
                    dx=_plain_combine(st["dX"], st["slots"], None, st["dY"]))
    return _plain_norm(st) if case["kind"] == "norm" else _plain_linear(st)


# -------------------------------------------------------------------- pass --

def run(st):
    if not own:
        return _plain(st)
    import paper_2103_16716_amd as pb
    case = st["case"]
    kind = case["kind"]
    if kind == "route":
        r = pb.topk_assign(st["S"], case["k"], workspace=st["ws"])
        return dict(assign=r.assign, scores=r.scores, perm=r.perm, slots=r.slots,
                    offsets=r.offsets)
    if kind == "move":
        X = pb.dispatch(st["x"], st["slots"], out=st["X"])
        Y = pb.combine(st["F"], st["slots"], weights=st["w"], residual=st["x"])
        dF, dw = pb.combine_backward(st["dY"], st["F"], st["slots"], st["w"], out=st["dF"])
        dx = pb.combine(st["dX"], st["slots"], residual=st["dY"])
        return dict(X=X, Y=Y, dF=dF, dw=dw, dx=dx)
    if kind == "norm":
        where = dict(offsets=st["offsets"], perm=st["perm"], k=case["k"])
        y, mean, rstd = pb.expert_norm(st["x"], st["weight"], st["bias"], eps=EPS, **where)
        if not case["train"]:
            return dict(y=y, mean=mean, rstd=rstd)
        dx, dweight, dbias = pb.expert_norm_backward(st["dy"], st["x"], st["weight"], mean, rstd,
                                                     workspace=st["ws"], **where)
        return dict(y=y, mean=mean, rstd=rstd, dx=dx, dweight=dweight, dbias=dbias)
    x, w, offsets = st["x"], st["w"], st["offsets"]
    out = {}
    if not case["train"] or case["residual"]:
        out["y"] = pb.expert_linear(x, w, offsets, bias=st["bias"], relu=case["relu"],
                                    residual=st["residual"])
    if case["train"]:
        out["dx"] = pb.expert_linear_dx(st["dy"], w, offsets, relu_of=x if case["relu"] else None)
        out["dw"], out["db"] = pb.expert_linear_dw(st["dy"], x, offsets)
    return out


# ------------------------------------------------------- work and accuracy --

def work(case):
    kind = case["kind"]
    if kind == "route":   # scores in; assign, scores, perm, slots and offsets out
        T, E, k = case["T"], case["E"], case["k"]
        return dict(bytes=4 * T * E + 16 * T * k + 4 * E, flops=T * E * k)
    sz = 2 if case["dtype"] == "bf16" else 4
    if kind == "move":
        # Each call's own rows: dispatch T in, N out; combine N and T in, T out,
        # twice; its backward T and N in, N out. (A padded batch has fewer.)
        T, k, d = case["T"], case["k"], case["d"]
        return dict(bytes=(6 * T + 5 * T * k) * d * sz + 28 * T * k, flops=8 * T * k * d)
    if kind == "norm":
        N, E, k, d = case["N"], case["E"], case["k"], case["d"]
        rows, b = (N // k + N) * d, 8 * N + 4 * E
        if not case["train"]:
            return dict(bytes=sz * (rows + 2 * E * d) + b, flops=8 * N * d)
        # and again for the backward: dy and x in, dx out; dweight and dbias
        return dict(bytes=sz * (rows + 2 * E * d + (N // k + 2 * N) * d + E * d) + 8 * E * d + 2 * b,
                    flops=24 * N * d)
    N, E, K, O = case["N"], case["E"], case["K"], case["O"]
    experts = min(E, N)   # at most so many have rows
    forward = not case["train"] or case["residual"]
    by, fl = 4 * E, 0
    if forward:
        by += sz * (N * K + experts * (K + 1) * O + N * O * (2 if case["residual"] else 1))
        fl += 2 * N * K * O
    if case["train"]:
        by += sz * (N * O + experts * K * O + N * K * (2 if case["relu"] else 1))
        by += sz * N * (K + O) + 4 * E * (K + 1) * O
        fl += 4 * N * K * O
    return dict(bytes=by, flops=fl)


def _exact_route(S, k):
    T, E = S.shape
    s = torch.where(torch.isnan(S), float("-inf"), S.double())
    v, a = torch.sort(s, dim=1, descending=True, stable=True)
    v, a = v[:, :k], torch.where(v[:, :k].isinf() & (v[:, :k] < 0), E, a[:, :k]).reshape(-1)
    count = torch.bincount(a, minlength=E + 1)[:E]
    offsets = torch.cat([count.new_zeros(1), count.cumsum(0)])
    n = int(offsets[E])
    # (expert, position) as one number: its order is the routed order
    rank = torch.sort(a * (T * k) + torch.arange(T * k, device=S.device)).values % (T * k)
    perm = rank.clone()
    perm[n:] = -1
    slots = torch.full_like(rank, -1)
    slots[rank[:n]] = torch.arange(n, device=S.device)
    i32 = torch.int32
    return dict(assign=torch.where(a == E, -1, a).view(T, k).to(i32), scores=v, perm=perm.to(i32),
                slots=slots.view(T, k).to(i32), offsets=offsets.to(i32))


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "route":
        return _exact_route(st["S"], case["k"])
    if kind == "move":
        k, d = case["k"], case["d"]
        perm, slots = st["perm"].long(), st["slots"].long()
        n = int((perm >= 0).sum())   # routed rows come first
        pairs = perm[:n]
        tok = pairs // k
        w = st["w"].double().view(-1)[pairs]
        x, dY, F = st["x"].double(), st["dY"].double(), st["F"].double()
        X, dF = st["X"].double(), st["dF"].double()
        X[:n] = x[tok]
        dF[:n] = w[:, None] * dY[tok]
        dw = torch.zeros(slots.numel(), dtype=torch.float64, device=DEV)
        dw[pairs] = (dY[tok] * F[:n]).sum(dim=1)
        Y = x.index_add(0, tok, w[:, None] * F[:n])
        return dict(X=X, Y=Y, dF=dF, dw=dw.view(slots.shape),
                    dx=dY.index_add(0, tok, st["dX"][:n].double()))
    if kind == "norm":
        N, E, k, d = case["N"], case["E"], case["k"], case["d"]
        bounds = [0, N] if st["offsets"] is None else st["offsets"].tolist()
        x = st["x"].double()
        if st["perm"] is not None:
            x = x[torch.div(st["perm"].long(), k, rounding_mode="floor")]
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = (var + EPS).rsqrt()
        xh = (x - mean[:, None]) * rstd[:, None]
        out = dict(y=torch.empty_like(x), mean=mean, rstd=rstd)
        if case["train"]:
            out.update(dx=torch.empty_like(x), dweight=x.new_zeros((E, d)),
                       dbias=x.new_zeros((E, d)))
        for e in range(E):
            r = slice(bounds[e], bounds[e + 1])
            w = st["weight"][e].double()
            out["y"][r] = torch.addcmul(st["bias"][e].double(), xh[r], w)
            if case["train"]:
                dy = st["dy"][r].double()
                h = dy * w
                h -= h.mean(dim=1, keepdim=True) + xh[r] * (h * xh[r]).mean(dim=1, keepdim=True)
                out["dx"][r] = h * rstd[r, None]
                out["dweight"][e] = (dy * xh[r]).sum(dim=0)
                out["dbias"][e] = dy.sum(dim=0)
        return out
    N, E, K, O = case["N"], case["E"], case["K"], case["O"]
    bounds = st["offsets"].tolist()
    f64 = dict(dtype=torch.float64, device=DEV)
    out = {}
    if not case["train"] or case["residual"]:
        out["y"] = torch.empty((N, O), **f64)
    if case["train"]:
        out.update(dx=torch.empty((N, K), **f64), dw=torch.zeros((E, O, K), **f64),
                   db=torch.zeros((E, O), **f64))
    for e in range(E):
        r = slice(bounds[e], bounds[e + 1])
        w, x = st["w"][e].double(), st["x"][r].double()
        if "y" in out:
            y = torch.addmm(st["bias"][e].double(), x, w.t())
            y = torch.relu(y) if case["relu"] else y
            out["y"][r] = y if st["residual"] is None else y + st["residual"][r]
        if case["train"]:
            dy = st["dy"][r].double()
            out["dx"][r] = torch.mm(dy, w) * ((x > 0) if case["relu"] else 1.0)
            out["dw"][e] = torch.mm(dy.t(), x)
            out["db"][e] = dy.sum(dim=0)
    return out

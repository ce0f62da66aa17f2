"""k experts a token, the experts' norm and products, through the C ABI against the
oracle in fp64.

Bounds: a fp32 sum of n terms in any order is off by at most n u sum |terms|, u =
2^-24 (products of bf16 are exact, a fp32 product adds one more u); a result stored
in bf16 is off by at most 2^-8 of its value more (half a step). Each test adds up the
roundings its formula makes. Integers are equal."""
import threading

import numpy as np
import pytest
import torch

import paper_2103_16716_amd as pb
import workloads as wl
from gpu_common import dev, host
from oracle import experts as ex

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
EPS = 1e-5
STEP = {"bf16": 2.0 ** -8, "f32": U}


def rng_of(*seed):
    return np.random.Generator(np.random.PCG64(list(seed)))


def rows(rng, shape, dtype, scale=1.0):
    """(values, what the device receives)."""
    x = rng.standard_normal(shape, dtype=np.float32) * np.float32(scale)
    if dtype == "f32":
        return x, x
    bits = wl.f32_to_bf16_bits(x)
    return wl.bf16_bits_to_f32(bits), bits


def values(t):
    h = host(t)
    with np.errstate(invalid="ignore"):   # (NaN in rows that no expert has)
        return (wl.bf16_bits_to_f32(h) if h.dtype == np.uint16 else h).astype(np.float64)


def close(got, want, bound):
    got, want = values(got) if torch.is_tensor(got) else got, np.asarray(want, dtype=np.float64)
    assert np.all(np.isfinite(got))
    over = np.abs(got - want) - bound
    assert np.all(over <= 0), f"off by {np.abs(got - want).max()}, {over.max()} over the bound"


def some_offsets(rng, N, E, first=0, last=None):
    """Uneven ranges with empty experts, covering [first, last)."""
    last = N if last is None else last
    cut = np.sort(rng.integers(first, last + 1, E - 1)) if E > 1 else np.zeros(0, dtype=np.int64)
    cut[: E // 3] = first    # the first third of the experts but one have no rows
    return np.concatenate([[first], np.sort(cut), [last]]).astype(np.int32)


# ------------------------------------------------------------------ routing --

@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 8, 8), (5, 3, 2), (48, 64, 2), (300, 100, 7),
                                   (1000, 128, 2), (2049, 256, 8), (513, 257, 3), (777, 512, 4),
                                   (130, 1021, 5), (64, 2048, 64), (70000, 16, 2), (4097, 6, 6),
                                   (65, 40, 3), (255, 128, 8), (255, 100, 4), (20001, 256, 8),
                                   (17000, 90, 5), (16385, 200, 3), (33000, 60, 8)])
def test_topk_assign(T, E, k):
    r = rng_of(T, E, k)
    S = r.standard_normal((T, E), dtype=np.float32)
    S[::3] = np.round(S[::3])                     # ties: the lowest index first; both zeros
    S[1::5, : E // 2] = -np.inf                   # experts that are forbidden
    S[2::7] = -np.inf                             # padding: no expert at all
    S[3::11, E // 3] = np.nan
    S[4::13, E - 1] = np.inf
    got = pb.topk_assign(dev(S), k)
    if T * E <= 400000:
        a, v = ex.topk(S, k)
    else:   # the same by numpy's stable sort
        key = np.where(S > -np.inf, S, -np.inf)
        a = np.argsort(-key, axis=1, kind="stable")[:, :k].astype(np.int32)
        v = np.take_along_axis(key, a, axis=1)
        a[v == -np.inf] = -1
    perm, slots, off = ex.sort_pairs(a, E)
    np.testing.assert_array_equal(host(got.assign), a)
    np.testing.assert_array_equal(host(got.scores), v)
    np.testing.assert_array_equal(host(got.offsets), off)
    np.testing.assert_array_equal(host(got.perm), perm)
    np.testing.assert_array_equal(host(got.slots), slots)


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (9, 5, 3), (100, 2048, 5), (3000, 64, 1),
                                   (50001, 33, 4)])
def test_sort_by_expert(T, E, k):
    r = rng_of(T, E, k, 1)
    a = r.integers(-2, E + 2, (T, k)).astype(np.int32)     # some have no expert
    a[0, 0] = np.iinfo(np.int32).max
    if T > 1:
        a[1] = np.iinfo(np.int32).min
    a[T // 2:] = np.where(r.random((T - T // 2, 1)) < 0.5, E - 1, a[T // 2:])   # a crowded expert
    perm, slots, off = ex.sort_pairs(a, E)
    ws = torch.full((pb.topk_workspace_size(T, E, k),), 0xA5, dtype=torch.uint8, device="cuda")
    for _ in range(2):   # a used workspace serves again
        got = pb.sort_by_expert(dev(a), E, workspace=ws)
        np.testing.assert_array_equal(host(got.offsets), off)
        np.testing.assert_array_equal(host(got.perm), perm)
        np.testing.assert_array_equal(host(got.slots), slots)


def test_one_choice_is_the_greedy_routing():
    S = dev(rng_of(3).standard_normal((5000, 96), dtype=np.float32))
    a, perm, off = pb.greedy_assign(S)
    r = pb.topk_assign(S, 1)
    s = pb.sort_by_expert(a, 96)
    for got in (r, s):
        assert torch.equal(got.assign.view(-1), a) and torch.equal(got.perm, perm)
        assert torch.equal(got.offsets, off)


# -------------------------------------------------------------------- moves --

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,k,d", [(1, 1, 8), (3, 2, 24), (65, 3, 1000), (200, 8, 264), (7, 64, 16),
                                   (130, 2, 2048), (31, 1, 4104), (9, 5, 8200), (40, 17, 520)])
def test_moves(T, k, d, dtype):
    r = rng_of(T, k, d)
    E = 5
    _, slots, off = ex.sort_pairs(r.integers(-1, E, (T, k)), E)
    w = r.standard_normal((T, k)).astype(np.float32)
    w[slots < 0] = np.nan                     # pairs without a row add nothing, whatever this is
    (x, xd), (F, Fd) = rows(r, (T, d), dtype), rows(r, (T * k, d), dtype)
    n = off[-1]
    F[n:] = 0
    sd, wd = dev(slots), dev(w)
    step = STEP[dtype]
    keep = torch.full((T * k, d), 7.0, dtype=dev(xd).dtype, device="cuda")
    seven = np.full((T * k, d), 7.0)
    close(pb.dispatch(dev(xd), sd, out=keep.clone()), ex.dispatch(x, slots, into=seven), 0.0)
    want = ex.dispatch(x, slots, w, into=seven)
    close(pb.dispatch(dev(xd), sd, weights=wd, out=keep.clone()), want, (step + U) * np.abs(want))
    for weights, residual in ((None, None), (w, None), (w, x), (None, x)):
        got = pb.combine(dev(Fd), sd, weights=None if weights is None else wd,
                         residual=None if residual is None else dev(xd))
        want = ex.combine(F, slots, weights, residual)
        mag = ex.combine(np.abs(F), slots, None if weights is None else np.abs(weights),
                         None if residual is None else np.abs(residual))
        close(got, want, (k + 2) * U * mag + step * (np.abs(want) + (k + 2) * U * mag))
    dF, dw = pb.combine_backward(dev(xd), dev(Fd), sd, wd, out=keep.clone())
    want, want_w = ex.combine_backward(x, F, slots, w, into=seven)
    mag = ex.combine_backward(np.abs(x), np.abs(F), slots, np.abs(w))[1]
    close(dF, want, (step + U) * np.abs(want))
    close(dw, want_w, (d + 2) * U * mag)


def test_combine_into_its_residual_and_bad_slots():
    """out may be the residual; slots out of range are no rows, and the same slot
    twice is read twice."""
    r = rng_of(5)
    T, k, d = 33, 3, 64
    (x, xd), (F, Fd) = rows(r, (T, d), "f32"), rows(r, (T * k, d), "f32")
    slots = r.integers(0, T * k, (T, k)).astype(np.int32)
    slots[3, 1] = slots[4, 0] = slots[4, 1]
    bad = slots.copy()
    bad[0], bad[1, 1], bad[2, 2] = -5, T * k, np.iinfo(np.int32).max
    ok = np.where((bad >= 0) & (bad < T * k), bad, -1)
    out = dev(xd)
    assert pb.combine(dev(Fd), dev(bad), residual=out, out=out) is out
    close(out, ex.combine(F, ok, None, x),
          (k + 2) * U * (np.abs(x) + ex.combine(np.abs(F), ok)))
    dF, dw = pb.combine_backward(dev(xd), dev(Fd), dev(bad), torch.ones(T, k, device="cuda"))
    assert torch.all(dw[torch.from_numpy(ok < 0).cuda()] == 0)


# --------------------------------------------------------------------- norm --

SUM = 64 * U    # a row's sums: at most 32 terms a lane and lanes and waves joined in a tree


def norm_bounds(x, w, b, e, eps, step):
    """Bounds of y, mean and rstd, and of xh: the mean is off by SUM mean |x|, the
    squares by SUM (and by the mean's own error squared), the root halves that."""
    x = x.astype(np.float64)
    y, mean, rstd = ex.norm(x, w, b, e, eps)
    c = x - mean[:, None]
    d_mean = SUM * np.abs(x).mean(axis=1) + 1e-37
    d_c = d_mean[:, None] + U * np.abs(c)
    var = (c * c).mean(axis=1)
    d_var = SUM * var + 2 * U * var + d_mean ** 2 + U * (var + eps)
    d_rstd = rstd * (0.5 * d_var / (var + eps) * 1.01 + 3 * U)
    d_xh = d_c * rstd[:, None] + np.abs(c) * d_rstd[:, None] + U * np.abs(c * rstd[:, None])
    wa = np.abs(w.astype(np.float64))[e]
    d_y = 1.01 * d_xh * wa + 2 * U * np.abs(y) + U * np.abs(c * rstd[:, None]) * wa
    return d_y + step * (np.abs(y) + d_y), d_mean, d_rstd, 1.01 * d_xh


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,E,d,mode", [
    (1, 1, 8, "shared"), (3, 1, 136, "shared"), (700, 1, 2048, "shared"), (257, 9, 512, "plain"),
    (130, 64, 1024, "plain"), (90, 5, 1000, "gather"), (64, 3, 2056, "plain"),
    (100, 7, 4096, "gather"), (40, 4, 8200, "plain"), (21, 2, 16384, "gather"),
    (600, 200, 264, "ragged"), (300, 3, 4096, "ragged"), (35, 2048, 64, "plain")])
def test_norm(N, E, d, mode, dtype):
    r = rng_of(N, E, d)
    k = 3 if mode == "gather" else 1
    n = N // k * k
    src = np.arange(n)
    perm = None
    T = n // k
    if mode == "gather":
        perm = r.permutation(n).astype(np.int32)
        src = perm // k
    step = STEP[dtype]
    x0 = r.standard_normal((T, d), dtype=np.float32) + 3 * r.standard_normal((T, 1), dtype=np.float32)
    x0[T // 2] = 1.5                              # a constant row: y = b
    xd = x0 if dtype == "f32" else wl.f32_to_bf16_bits(x0)
    x = x0 if dtype == "f32" else wl.bf16_bits_to_f32(xd)
    (w, wd), (b, bd), (dy, dyd), (res, resd) = (rows(r, s, dtype) for s in
                                                ((E, d), (E, d), (n, d), (n, d)))
    first, last = (7, n - 9) if mode == "ragged" else (0, n)
    off = some_offsets(r, n, E, first, last)
    e = ex.row_experts(off, n)
    live = e >= 0
    e = e[live]
    kw = dict(offsets=None if mode == "shared" else dev(off), perm=None if perm is None else dev(perm),
              k=k)
    keep = torch.full((n, d), 7.0, dtype=dev(dyd).dtype, device="cuda")
    y, mean, rstd = pb.expert_norm(dev(xd), dev(wd), dev(bd), eps=EPS, out=keep.clone(), **kw)
    xs = x[src][live]
    b_y, b_mean, b_rstd, b_xh = norm_bounds(xs, w, b, e, EPS, step)
    want_y, want_mean, want_rstd = ex.norm(xs, w, b, e, EPS)
    close(values(y)[live], want_y, b_y)
    close(values(mean)[live], want_mean, b_mean)
    close(values(rstd)[live], want_rstd, b_rstd)
    assert np.all(values(y)[~live] == 7.0)        # rows of no expert
    y2 = pb.expert_norm(dev(xd), dev(wd), eps=EPS, **kw)[0]
    close(values(y2)[live], ex.norm(xs, w, None, e, EPS)[0], b_y + step * np.abs(b).max())

    want, want_w, want_b = ex.norm_backward(dy[live], xs, w, e, EPS)
    dya, wa = np.abs(dy[live].astype(np.float64)), np.abs(w.astype(np.float64))[e]
    xh = np.abs((xs - want_mean[:, None]) * want_rstd[:, None])
    h = dya * wa
    d_s1 = (SUM + U) * h.mean(axis=1, keepdims=True)
    d_s2 = ((SUM + 2 * U) * h * xh + h * b_xh).mean(axis=1, keepdims=True)
    s1, s2 = h.mean(axis=1, keepdims=True), (h * xh).mean(axis=1, keepdims=True)
    rs = want_rstd[:, None]
    b_dx = rs * (d_s1 + xh * d_s2 + b_xh * s2 + 4 * U * (h + s1 + xh * s2)) + \
        (b_rstd / want_rstd)[:, None] * np.abs(want)
    b_dx = 1.05 * b_dx
    m = np.maximum(np.bincount(e, minlength=E), 1)[:, None]
    b_w, b_b = np.zeros((E, d)), np.zeros((E, d))
    np.add.at(b_w, e, dya * b_xh + (m[e] + 2) * U * dya * xh)
    np.add.at(b_b, e, m[e] * U * dya)
    ws = torch.full((pb.expert_norm_workspace_size(n, E, d),), 0xA5, dtype=torch.uint8, device="cuda")
    for add in (None, res):
        dx, dw, db = pb.expert_norm_backward(dev(dyd), dev(xd), dev(wd), mean, rstd, workspace=ws,
                                             residual=None if add is None else dev(resd),
                                             out=keep.clone(), **kw)
        total = want if add is None else want + add[live]
        more = 0.0 if add is None else U * np.abs(total)
        close(values(dx)[live], total, b_dx + more + step * (np.abs(total) + b_dx))
        assert np.all(values(dx)[~live] == 7.0)
        close(dw, want_w, 1.05 * b_w)
        close(db, want_b, b_b)
    # in place of its gradient or of the added rows; the same bits as before
    for name in ("dy", "residual"):
        a, c = dev(dyd), dev(resd)
        into = a if name == "dy" else c
        got = pb.expert_norm_backward(a, dev(xd), dev(wd), mean, rstd, residual=c, out=into, **kw)
        assert torch.equal(got[0][torch.from_numpy(live).cuda()], dx[torch.from_numpy(live).cuda()])
        assert torch.equal(got[1], dw) and torch.equal(got[2], db)


# ----------------------------------------------------------------- products --

SHAPES = [(1, 1, 8, 8), (5, 3, 16, 24), (64, 8, 128, 72), (100, 7, 264, 200), (300, 2, 1000, 136),
          (33, 40, 520, 64), (257, 4, 64, 520), (700, 3, 192, 328), (1500, 5, 256, 512),
          (2000, 9, 512, 256), (600, 1, 2056, 264), (16, 2048, 32, 16), (90, 6, 2048, 1024)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,E,K,O", SHAPES)
def test_products(N, E, K, O, dtype):
    r = rng_of(N, E, K, O)
    ragged = N >= 100
    off = some_offsets(r, N, E, *((3, N - 5) if ragged else (0, N)))
    e = ex.row_experts(off, N)
    live = e >= 0
    e = e[live]
    step = STEP[dtype]
    (x, xd), (w, wd) = rows(r, (N, K), dtype), rows(r, (E, O, K), dtype, K ** -0.5)
    (b, bd), (res, resd), (dy, dyd) = rows(r, (E, O), dtype), rows(r, (N, O), dtype), \
        rows(r, (N, O), dtype)
    x[~live] = np.nan     # rows of no expert are not read as input that matters
    dy[~live] = np.nan
    xd, dyd = (a if dtype == "f32" else wl.f32_to_bf16_bits(a) for a in (x, dy))
    X, W, D, G = dev(xd), dev(wd), dev(dyd), dev(off)
    xl, dl = x[live], dy[live]
    keep = dict(y=torch.full((N, O), 7.0, dtype=X.dtype, device="cuda"),
                dx=torch.full((N, K), 7.0, dtype=X.dtype, device="cuda"))
    mag = ex.linear(np.abs(xl), np.abs(w), None, e)
    for bias, relu, residual in ((None, False, None), (b, True, None), (b, False, res),
                                 (None, True, res)):
        got = pb.expert_linear(X, W, G, bias=None if bias is None else dev(bd), relu=relu,
                               residual=None if residual is None else dev(resd),
                               out=keep["y"].clone())
        want = ex.linear(xl, w, bias, e, relu, None if residual is None else residual[live])
        m = (K + 3) * U * (mag + (0 if bias is None else np.abs(b[e])))
        m = m + (0 if residual is None else U * (np.abs(res[live]) + mag))
        close(values(got)[live], want, m + step * (np.abs(want) + m))
        assert np.all(values(got)[~live] == 7.0)
    u, ud = rows(r, (N, K), dtype)
    u[:, ::5] = 0.0
    u[:, 1::7] = np.nan
    ud = u if dtype == "f32" else wl.f32_to_bf16_bits(u)
    mag = ex.linear_dx(np.abs(dl), np.abs(w), e)
    for relu_of in (None, u):
        got = pb.expert_linear_dx(D, W, G, relu_of=None if relu_of is None else dev(ud),
                                  out=keep["dx"].clone())
        want = ex.linear_dx(dl, w, e, None if relu_of is None else relu_of[live])
        m = (O + 3) * U * mag
        close(values(got)[live], want, m + step * (np.abs(want) + m))
        assert np.all(values(got)[~live] == 7.0)
    dw, db = pb.expert_linear_dw(D, X, G)
    want, want_b = ex.linear_dw(dl, xl, e, E)
    mag, mag_b = ex.linear_dw(np.abs(dl), np.abs(xl), e, E)
    n = np.bincount(e, minlength=E)
    close(dw, want, (n + 3)[:, None, None] * U * mag)
    close(db, want_b, (n + 3)[:, None] * U * mag_b)
    again = pb.expert_linear_dw(D, X, G)
    assert torch.equal(again[0], dw) and torch.equal(again[1], db)


# Few outputs and long sums: cut into parts (the number of them is in the comment, a product's
# in bf16 and fp32).
IN_PARTS = [(1, 1, 8192, 512),      # y 32, 32; one row, parts of four chunks
            (70, 1, 8192, 264),     # y 25, 25; uneven parts, columns behind 256
            (40, 3, 4104, 72),      # y 16, 32; a part of part of a chunk, the last ones empty
            (130, 1, 8, 4096),      # dx 16, 32
            (150, 2, 1032, 6152),   # dx 7, 7; three groups of columns in the join
            (300, 2, 8192, 136),    # y 14, 14; several tiles of rows
            (5000, 3, 264, 40),     # dw 6, 13
            (5000, 1, 64, 200)]     # dw 19, 32


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,E,K,O", IN_PARTS)
def test_products_in_parts(N, E, K, O, dtype):
    code = pb.BASE_F32 if dtype == "f32" else pb.BASE_BF16
    sizes = [pb.expert_linear_workspace_size(p, N, E, K, O, code)
             for p in (pb.BASE_PRODUCT_Y, pb.BASE_PRODUCT_DX, pb.BASE_PRODUCT_DW)]
    assert max(sizes) > 0
    test_products(N, E, K, O, dtype)
    # the workspace's contents do not matter, and another expert's rows may be none or all
    r = rng_of(N, E, K, O, 1)
    x, w, dy = (dev(rows(r, n, dtype)[1]) for n in ((N, K), (E, O, K), (N, O)))
    off = dev(np.array([0] * E + [N], dtype=np.int32))
    got = []
    for fill in (0, 255):
        ws = [torch.full((max(n, 256),), fill, dtype=torch.uint8, device="cuda") for n in sizes]
        got.append((pb.expert_linear(x, w, off, workspace=ws[0]),
                    pb.expert_linear_dx(dy, w, off, workspace=ws[1]),
                    *pb.expert_linear_dw(dy, x, off, workspace=ws[2])))
    for a, b in zip(*got):
        assert torch.equal(a, b) and bool(torch.isfinite(a).all())
    y, dx, dw, db = got[0]
    assert bool((dw[:-1] == 0).all()) and bool((db[:-1] == 0).all())
    step = STEP[dtype]
    near_product(y, x, w[-1].t().contiguous(), K, step)
    near_product(dx, dy, w[-1], O, step)
    near_product(dw[-1], dy.t().contiguous(), x, N, U)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,E,K,O", [(7, 3, 16, 24), (90, 1, 4096, 264), (150, 2, 520, 4104),
                                     (3000, 2, 136, 72), (2500, 3, 520, 2056)])
def test_a_batch_of_padding(N, E, K, O, dtype):
    """No token has an expert: the router says so, results and gradients by the rows stay as
    they were, those by the weights are zero."""
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    route = pb.topk_assign(torch.full((N, E), -float("inf"), device="cuda"), 1)
    assert bool((route.assign == -1).all()) and bool((route.slots == -1).all())
    assert bool((route.perm == -1).all()) and bool((route.offsets == 0).all())
    off = route.offsets
    x, dy = (torch.full((N, n), float("nan"), dtype=t, device="cuda") for n in (K, O))
    w = torch.randn(E, O, K, device="cuda").to(t)
    y, dx = torch.full_like(dy, 7.0), torch.full_like(x, 7.0)
    pb.expert_linear(x, w, off, out=y)
    pb.expert_linear_dx(dy, w, off, out=dx)
    dw, db = pb.expert_linear_dw(dy, x, off)
    _, mean, rstd = pb.expert_norm(x, w[:, 0].contiguous(), None, off, out=dx)
    dg, dbias = pb.expert_norm_backward(x, x, w[:, 0].contiguous(), mean, rstd, off, out=dx)[1:]
    assert bool((y == 7).all()) and bool((dx == 7).all())
    for z in (dw, db, dg, dbias):
        assert bool((z == 0).all())
    h = torch.randn(N, K, device="cuda").to(t)
    assert torch.equal(pb.combine(x, route.slots, residual=h), h)
    w1 = torch.full((N, 1), float("nan"), device="cuda")
    assert torch.equal(pb.combine(x, route.slots, weights=w1, residual=h), h)
    dF, dwt = pb.combine_backward(h, x, route.slots, w1, out=torch.full_like(x, 7.0))
    assert bool((dF == 7).all()) and bool((dwt == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,E,K,O", [(90, 1, 4096, 264), (150, 2, 520, 4104), (3000, 2, 136, 72),
                                     (33, 40, 520, 64), (2500, 3, 520, 2056)])
def test_products_in_place_captured_and_at_once(N, E, K, O, dtype):
    """The bits of a plain call: with y in the residual's place and dx in relu_of's, in every
    replay of a graph (a workspace of its own, other work between the replays), and by two
    streams at once."""
    r = rng_of(N, E, K, O, 2)
    x, w, dy, res, u = (dev(rows(r, n, dtype)[1])
                        for n in ((N, K), (E, O, K), (N, O), (N, O), (N, K)))
    b = dev(rows(r, (E, O), dtype)[1])
    off = dev(some_offsets(r, N, E, 0, N))

    def run():
        return (pb.expert_linear(x, w, off, bias=b, relu=True, residual=res),
                pb.expert_linear_dx(dy, w, off, relu_of=u), *pb.expert_linear_dw(dy, x, off))

    want = run()
    a, c = res.clone(), u.clone()
    assert pb.expert_linear(x, w, off, bias=b, relu=True, residual=a, out=a) is a
    assert pb.expert_linear_dx(dy, w, off, relu_of=c, out=c) is c
    assert torch.equal(a, want[0]) and torch.equal(c, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for _ in range(3):
        for t in got:
            t.fill_(float("nan"))
        graph.replay()
        again = run()
        torch.cuda.synchronize()
        for p, q, s in zip(want, got, again):
            assert torch.equal(p, q) and torch.equal(p, s)
    streams = [torch.cuda.Stream() for _ in range(2)]
    out = []
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    for _ in range(4):
        for st in streams:
            with torch.cuda.stream(st):
                out.append(run())
    torch.cuda.synchronize()
    for got in out:
        assert all(torch.equal(p, q) for p, q in zip(want, got))


def test_products_keep_infinities_and_nan_in_their_rows():
    """A row of NaN or infinities spoils its own results only, and the ReLU keeps a NaN."""
    r = rng_of(11)
    N, E, K, O = 200, 3, 256, 136
    x, w = r.standard_normal((N, K), dtype=np.float32), r.standard_normal((E, O, K), dtype=np.float32)
    off = np.array([0, 90, 91, 200], dtype=np.int32)
    clean = pb.expert_linear(dev(x), dev(w), dev(off), relu=True)
    x[90] = np.nan
    x[5, 3] = np.inf
    y = pb.expert_linear(dev(x), dev(w), dev(off), relu=True)
    assert torch.isnan(y[90]).all() and not torch.isfinite(y[5]).all()
    rest = [i for i in range(N) if i not in (5, 90)]
    assert torch.equal(y[rest], clean[rest])


def test_offsets_out_of_order_stay_in_bounds():
    """Offsets beyond the rows, negative or falling are no fault: ranges are cut to
    the rows there are, and what they do not cover is left alone."""
    N, E, K, O = 64, 4, 32, 40
    x = torch.ones(N, K, device="cuda")
    w = torch.ones(E, O, K, device="cuda")
    off = torch.tensor([-7, 20, 10, 1 << 30, 5], dtype=torch.int32, device="cuda")
    out = torch.full((N, O), 7.0, device="cuda")
    y = pb.expert_linear(x, w, off, out=out)
    assert torch.equal(y, torch.full_like(y, float(K)))
    pb.expert_linear_dx(y, w, off)
    pb.expert_linear_dw(y, x, off)
    y, mean, rstd = pb.expert_norm(x, w[:, 0].contiguous(), None, off)
    pb.expert_norm_backward(x, x, w[:, 0].contiguous(), mean, rstd, off)
    torch.cuda.synchronize()


def near_product(got, a, b, terms, step):
    """got against a b in fp64 on the GPU: a fp32 sum of so many terms, stored with `step`."""
    a, b = a.double(), b.double()
    want = a @ b
    bound = (terms + 3) * U * (a.abs() @ b.abs())
    assert bool(((got.double() - want).abs() <= bound + step * (want.abs() + bound)).all())


@pytest.mark.parametrize("counts,K,O", [
    # (1) many tiles of one size for every unit: the tiles that blocks go through in turn, ends
    # of 1 to 255 rows, empty experts, a last round of few tiles
    ([2816, 0, 2561, 2623], 72, 6152), ([1800, 900, 1300, 1, 3999, 0], 72, 6152),
    ([8000], 200, 6144), ([4097, 4000], 1032, 2056), ([700, 64, 0, 129, 2200, 3000], 64, 8200),
    ([2816, 0, 2561, 2623], 6152, 72), ([700, 64, 0, 129, 2200, 3000], 8200, 64),
    # (2) 128 x 128 and 64 x 128 tiles, one expert and several
    ([128] * 40, 264, 2056), ([90, 30, 64, 65] * 16, 520, 1032), ([513], 2056, 1032)])
def test_large_products(counts, K, O):
    """Every expert's block of y, dx and dW in bf16, in the tiles of larger calls, with the
    results of rows before and behind left alone."""
    g = torch.Generator(device="cuda").manual_seed(K + O)
    before, behind = 5, 3
    N, E = sum(counts) + before + behind, len(counts)
    x, dy = (torch.randn(N, n, generator=g, device="cuda").bfloat16() for n in (K, O))
    w = (torch.randn(E, O, K, generator=g, device="cuda") * K ** -0.5).bfloat16()
    ends = np.cumsum([before] + counts)
    off = torch.tensor(ends, dtype=torch.int32, device="cuda")
    for back in (x, dy):
        back[:before], back[N - behind:] = float("nan"), float("inf")
    y = pb.expert_linear(x, w, off, out=torch.full((N, O), 7.0, dtype=x.dtype, device="cuda"))
    dx = pb.expert_linear_dx(dy, w, off, out=torch.full_like(x, 7.0))
    dw, db = pb.expert_linear_dw(dy, x, off)
    for e, n in enumerate(counts):
        r = slice(int(ends[e]), int(ends[e + 1]))
        near_product(y[r], x[r], w[e].t().contiguous(), K, 2.0 ** -8)
        near_product(dx[r], dy[r], w[e], O, 2.0 ** -8)
        near_product(dw[e], dy[r].t().contiguous(), x[r], n, U)
        want, mag = dy[r].double().sum(dim=0), dy[r].double().abs().sum(dim=0)
        assert bool(((db[e].double() - want).abs() <= (n + 1) * U * mag).all())
    for got in (y, dx):
        assert bool((got[:before] == 7).all()) and bool((got[N - behind:] == 7).all())


def test_matrices_beyond_32_bits():
    """More than 2^32 bytes and 2^31 elements in the rows, then in the matrices: the last
    rows and the last expert have their results."""
    g = torch.Generator(device="cuda").manual_seed(1)
    N, n, K, O, E = 270000, 200, 8192, 64, 3
    m = 130                                            # rows of expert 0; expert 2 the others
    x = torch.empty(N, K, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(n, K, generator=g, device="cuda").bfloat16()
    x[N - n:] = tail
    dy = torch.randn(N, O, generator=g, device="cuda").bfloat16()
    dt = dy[N - n:]
    w = (torch.randn(E, O, K, generator=g, device="cuda") * K ** -0.5).bfloat16()
    off = torch.tensor([N - n, N - n + m, N - n + m, N], dtype=torch.int32, device="cuda")
    y = pb.expert_linear(x, w, off)[N - n:]
    near_product(y[:m], tail[:m], w[0].t().contiguous(), K, 2.0 ** -8)
    near_product(y[m:], tail[m:], w[2].t().contiguous(), K, 2.0 ** -8)
    dx = torch.empty_like(x)
    pb.expert_linear_dx(dy, w, off, out=dx)
    near_product(dx[N - n:N - n + m], dt[:m], w[0], O, 2.0 ** -8)
    near_product(dx[N - n + m:], dt[m:], w[2], O, 2.0 ** -8)
    dw = pb.expert_linear_dw(dy, x, off)[0]
    near_product(dw[0], dt[:m].t().contiguous(), tail[:m], m, U)
    near_product(dw[2], dt[m:].t().contiguous(), tail[m:], n - m, U)
    assert not torch.any(dw[1])
    gain = w[:, 0].contiguous()
    y, mean, rstd = pb.expert_norm(x, gain, None, off, out=dx)
    want, mean_t, _ = pb.expert_norm(tail, gain, None, off - (N - n))
    assert torch.equal(y[N - n:], want) and torch.equal(mean[N - n:], mean_t)
    slots = torch.full((N, 1), -1, dtype=torch.int32, device="cuda")
    slots[N - n:, 0] = torch.arange(N - 1, N - n - 1, -1, device="cuda", dtype=torch.int32)
    moved = pb.dispatch(x, slots, out=dx)
    assert torch.equal(moved[N - n:], tail.flip(0))
    back = pb.combine(moved, slots)
    assert torch.equal(back[N - n:], tail) and not torch.any(back[0])
    del x, dx, y, moved, back
    E, O = 300, 1024
    w = torch.empty(E, O, K, dtype=torch.bfloat16, device="cuda")
    w[E - 1] = (torch.randn(O, K, generator=g, device="cuda") * K ** -0.5).bfloat16()
    off = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    off[E] = n
    dy = torch.randn(n, O, generator=g, device="cuda").bfloat16()
    near_product(pb.expert_linear(tail, w, off), tail, w[E - 1].t().contiguous(), K, 2.0 ** -8)
    near_product(pb.expert_linear_dx(dy, w, off), dy, w[E - 1], O, 2.0 ** -8)
    dw, db = pb.expert_linear_dw(dy, tail, off)
    near_product(dw[E - 1], dy.t().contiguous(), tail, n, U)
    assert not torch.any(dw[E - 2]) and not torch.any(db[:E - 1])


# ----------------------------------------------------------------- together --

def block(H, S, k, p, dOut):
    """A whole layer with k experts a token, forward and backward, as a program runs it."""
    r = pb.topk_assign(S, k)
    weights = torch.softmax(r.scores, dim=1)
    y, mean, rstd = pb.expert_norm(H, p["g"], p["b"], r.offsets, eps=EPS, perm=r.perm, k=k)
    u = pb.expert_linear(y, p["W1"], r.offsets, bias=p["b1"], relu=True)
    f = pb.expert_linear(u, p["W2"], r.offsets, bias=p["b2"])
    out = pb.combine(f, r.slots, weights=weights, residual=H)
    df, dweights = pb.combine_backward(dOut, f, r.slots, weights)
    dW2, db2 = pb.expert_linear_dw(df, u, r.offsets)
    du = pb.expert_linear_dx(df, p["W2"], r.offsets, relu_of=u)
    dW1, db1 = pb.expert_linear_dw(du, y, r.offsets)
    dy = pb.expert_linear_dx(du, p["W1"], r.offsets)
    dx, dg, db = pb.expert_norm_backward(dy, H, p["g"], mean, rstd, r.offsets, perm=r.perm, k=k)
    dH = pb.combine(dx, r.slots, residual=dOut)
    return dict(out=out, dH=dH, dw=dweights, W1=dW1, b1=db1, W2=dW2, b2=db2, g=dg, b=db)


def block_inputs(T=96, E=6, d=64, inner=256, seed=0):
    r = rng_of(T, E, d, seed)
    p = dict(g=1 + 0.1 * r.standard_normal((E, d)), b=0.1 * r.standard_normal((E, d)),
             W1=r.standard_normal((E, inner, d)) * d ** -0.5, b1=0.1 * r.standard_normal((E, inner)),
             W2=r.standard_normal((E, d, inner)) * inner ** -0.5, b2=0.1 * r.standard_normal((E, d)))
    p = {k: v.astype(np.float32) for k, v in p.items()}
    H, dOut = (r.standard_normal((T, d)).astype(np.float32) for _ in range(2))
    S = r.standard_normal((T, E)).astype(np.float32)
    S[::9] = -np.inf            # padding
    S[1::9, 1:] = -np.inf       # one expert allowed
    return H, S, p, dOut


def block_loss(H, S, k, p, dOut, weights=None):
    """<layer(H), dOut> in fp64 from the definition, without a sort: each token by each
    of its experts."""
    a, v = ex.topk(S, k)
    total = 0.0
    for t in range(H.shape[0]):
        h = H[t]
        out = h.copy()
        s = np.exp(v[t] - v[t].max()) if a[t, 0] >= 0 else np.zeros(k)
        s = s / max(s.sum(), 1e-300) if weights is None else weights[t]
        for j in range(k):
            i = a[t, j]
            if i < 0:
                continue
            z = (h - h.mean()) / np.sqrt(h.var() + EPS) * p["g"][i] + p["b"][i]
            u = np.maximum(p["W1"][i] @ z + p["b1"][i], 0)
            out = out + s[j] * (p["W2"][i] @ u + p["b2"][i])
        total += out @ dOut[t]
    return total


@pytest.mark.parametrize("k", [1, 2, 4])
def test_layer_gradients_against_differences(k):
    """The layer in fp32: its result and every gradient along random directions, against
    the definition in fp64 and its central differences. Sums of up to N d terms of size
    one agree to a part in 10^4 by far; a wrong factor or row is off by its whole share."""
    H, S, p, dOut = block_inputs()
    got = block(dev(H), dev(S), k, {n: dev(v) for n, v in p.items()}, dev(dOut))
    f64 = lambda z: np.asarray(z, dtype=np.float64)
    H, S, dOut, p = f64(H), f64(S), f64(dOut), {n: f64(v) for n, v in p.items()}
    want = block_loss(H, S, k, p, dOut)
    scale = np.abs(dOut * H).sum()
    assert abs((values(got["out"]) * dOut).sum() - want) <= 1e-5 * scale
    r = rng_of(k, 99)
    h = 1e-4
    for name in ("W1", "b1", "W2", "b2", "g", "b", "dH"):
        v = r.standard_normal(H.shape if name == "dH" else p[name].shape)
        v /= np.linalg.norm(v)
        if name == "dH":
            d = block_loss(H + h * v, S, k, p, dOut) - block_loss(H - h * v, S, k, p, dOut)
        else:
            d = (block_loss(H, S, k, {**p, name: p[name] + h * v}, dOut)
                 - block_loss(H, S, k, {**p, name: p[name] - h * v}, dOut))
        g = values(got[name])
        assert abs((g * v).sum() - d / (2 * h)) <= 1e-3 * np.linalg.norm(g), name
    # the weights' gradient, one token's choices at a time
    a, sc = ex.topk(S, k)
    w = np.where(a >= 0, np.exp(np.where(a >= 0, sc - np.where(a >= 0, sc, 0).max(), 0)), 0)
    w /= np.maximum(w.sum(axis=1, keepdims=True), 1e-300)
    v = r.standard_normal(w.shape) * (a >= 0)
    d = block_loss(H, S, k, p, dOut, w + h * v) - block_loss(H, S, k, p, dOut, w - h * v)
    assert abs((values(got["dw"]) * v).sum() - d / (2 * h)) <= \
        1e-3 * np.linalg.norm(values(got["dw"])) * np.linalg.norm(v)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layer_captured_and_replayed(dtype):
    """The whole layer captured into a graph: every replay, between eager runs on other
    data, gives the bits of the eager run on the same data."""
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    sets = []
    for seed in range(3):
        H, S, p, dOut = block_inputs(T=200, E=12, d=128, inner=512, seed=seed)
        sets.append([dev(H).to(t), dev(S), {n: dev(v).to(t) for n, v in p.items()}, dev(dOut).to(t)])
    H, S, p, dOut = (x.clone() if torch.is_tensor(x) else {n: v.clone() for n, v in x.items()}
                     for x in sets[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block(H, S, 2, p, dOut)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = block(H, S, 2, p, dOut)
    for i in (0, 1, 2, 1, 0):
        want = block(*sets[i][:2], 2, *sets[i][2:])
        H.copy_(sets[i][0])
        S.copy_(sets[i][1])
        dOut.copy_(sets[i][3])
        for n, v in sets[i][2].items():
            p[n].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        routed = int(pb.topk_assign(S, 2).offsets[-1])
        assert 0 < routed < 400
        for n in want:
            assert torch.equal(got[n], want[n]), n


def test_layer_from_two_threads():
    """Threads with streams of their own: the library keeps nothing between calls."""
    H, S, p, dOut = block_inputs(T=700, E=8, d=256, inner=1024)
    H, S, dOut, p = dev(H), dev(S), dev(dOut), {n: dev(v) for n, v in p.items()}
    want = block(H, S, 2, p, dOut)
    torch.cuda.synchronize()
    wrong, done = [], []

    def work():
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(6):
                got = block(H, S, 2, p, dOut)
                torch.cuda.current_stream().synchronize()
                wrong.extend(n for n in want if not torch.equal(got[n], want[n]))
        done.append(1)

    threads = [threading.Thread(target=work) for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(done) == 2 and not wrong


def test_layer_on_a_stream_of_its_own():
    """With stream= the work and its outputs belong to that stream, whatever is current."""
    H, S, p, dOut = block_inputs(T=500, E=8, d=256, inner=512)
    H, S, dOut, p = dev(H), dev(S), dev(dOut), {n: dev(v) for n, v in p.items()}
    want = block(H, S, 2, p, dOut)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    r = pb.topk_assign(S, 2, stream=st)
    y, mean, rstd = pb.expert_norm(H, p["g"], p["b"], r.offsets, eps=EPS, perm=r.perm, k=2, stream=st)
    u = pb.expert_linear(y, p["W1"], r.offsets, bias=p["b1"], relu=True, stream=st)
    f = pb.expert_linear(u, p["W2"], r.offsets, bias=p["b2"], stream=st)
    with torch.cuda.stream(st):
        weights = torch.softmax(r.scores, dim=1)
    out = pb.combine(f, r.slots, weights=weights, residual=H, stream=st)
    df, dw = pb.combine_backward(dOut, f, r.slots, weights, stream=st)
    dW2, db2 = pb.expert_linear_dw(df, u, r.offsets, stream=st)
    x = pb.dispatch(H, r.slots, stream=st)
    st.synchronize()
    assert torch.equal(out, want["out"]) and torch.equal(dw, want["dw"])
    assert torch.equal(dW2, want["W2"]) and torch.equal(db2, want["b2"])
    n = int(r.offsets[-1])
    assert torch.equal(x[:n], H[r.perm[:n].long() // 2])


def test_binding_refusals():
    f = torch.zeros(4, 16, device="cuda")
    b = f.bfloat16()
    i = torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    o = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    w = torch.zeros(2, 16, 16, device="cuda")
    for call in (lambda: pb.topk_assign(f, 0), lambda: pb.topk_assign(f, 17),
                 lambda: pb.topk_assign(f.t(), 2), lambda: pb.sort_by_expert(i[None], 4),
                 lambda: pb.dispatch(f[:3], i), lambda: pb.dispatch(f, i, out=f),
                 lambda: pb.dispatch(f, i, weights=f), lambda: pb.combine(f, i),
                 lambda: pb.combine(torch.zeros(8, 16, device="cuda"), i, residual=b),
                 lambda: pb.combine_backward(f, torch.zeros(8, 16, device="cuda"), i, None),
                 lambda: pb.expert_norm(f, f[:2]), lambda: pb.expert_norm(f, b[0]),
                 lambda: pb.expert_norm(f, f[:2], offsets=o[:2]),
                 lambda: pb.expert_norm(f, f[0], perm=f[0]),
                 lambda: pb.expert_norm(f, f[0], k=2),
                 lambda: pb.expert_linear(f, w, o[:2]), lambda: pb.expert_linear(b, w, o),
                 lambda: pb.expert_linear(f, w, o, bias=f[:2, :8]),
                 lambda: pb.expert_linear(f, w[0], o), lambda: pb.expert_linear_dx(f, w, i[0]),
                 lambda: pb.expert_linear_dw(f, b, o),
                 lambda: pb.expert_linear_dx(f[:, ::2], w, o)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: pb.topk_assign(b, 2), lambda: pb.sort_by_expert(o.long(), 4),
                 lambda: pb.dispatch(f, i.long()), lambda: pb.dispatch(f.half(), i)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(pb.BaseError) as err:
        pb.topk_assign(f, 2, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    assert err.value.status == pb.BASE_ERR_WORKSPACE
    with pytest.raises(pb.BaseError) as err:
        pb.expert_linear(f, w, o, out=f)
    assert err.value.status == pb.BASE_ERR_INVALID_ARG

"""The expert layer's calls at numbers of rows near 2^31 and of blocks that a launch has no room
for. Values are whole numbers whose sums are exact in fp32, so that results are equal."""
import pytest
import torch

import paper_2103_16716_amd as pb

pytestmark = pytest.mark.gpu

STEP = 1 << 24   # rows compared at a time


@pytest.fixture(autouse=True)
def memory():
    yield
    torch.cuda.empty_cache()


def steps(n):
    for a in range(0, n, STEP):
        yield slice(a, min(n, a + STEP))


def signs(g, *shape, dtype):
    """-1, 0 or 1."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    for r in steps(shape[0]):
        out[r] = torch.randint(-1, 2, out[r].shape, generator=g, device="cuda",
                               dtype=torch.int8).to(dtype)
    return out


def test_routing_of_most_pairs():
    """2^31 - 2 pairs, the last tokens without an expert: choices against a stable sort, then
    perm and slots: each row's pair has the row's expert, rises within an expert, and has the
    row as its slot."""
    g = torch.Generator(device="cuda").manual_seed(0)
    T, E, k, padded = (1 << 30) - 1, 3, 2, 1000
    S = torch.rand(T, E, generator=g, device="cuda")
    S[T - padded:] = -float("inf")
    got = pb.topk_assign(S, k)
    count = torch.zeros(E, dtype=torch.int64, device="cuda")
    for r in steps(T - padded):
        v, a = torch.sort(S[r], dim=1, descending=True, stable=True)
        assert torch.equal(got.assign[r].long(), a[:, :k]) and torch.equal(got.scores[r], v[:, :k])
        count += torch.bincount(a[:, :k].reshape(-1), minlength=E)
    assert bool((got.assign[T - padded:] == -1).all() and (got.slots[T - padded:] == -1).all())
    del S
    off = [0] + count.cumsum(0).tolist()
    assert got.offsets.tolist() == off and off[E] == k * (T - padded)
    flat, slots = got.assign.view(-1), got.slots.view(-1)
    for e in range(E):
        last = -1
        for r in steps(off[e + 1] - off[e]):
            row = torch.arange(off[e] + r.start, off[e] + r.stop, device="cuda")
            pair = got.perm[off[e] + r.start:off[e] + r.stop].long()
            assert bool((pair[1:] > pair[:-1]).all()) and int(pair[0]) > last
            last = int(pair[-1])
            assert bool((flat[pair] == e).all()) and bool((slots[pair] == row).all())
    assert bool((got.perm[off[E]:] == -1).all())
    again = pb.sort_by_expert(got.assign, E)
    assert all(torch.equal(a, b) for a, b in ((again.perm, got.perm), (again.slots, got.slots),
                                              (again.offsets, got.offsets)))


def test_moves_of_many_tokens():
    g = torch.Generator(device="cuda").manual_seed(1)
    T, d, t = (1 << 30) + 5, 8, torch.bfloat16
    x = signs(g, T, d, dtype=t)
    slots = torch.arange(T - 1, -1, -1, dtype=torch.int32, device="cuda")[:, None]
    w = torch.ones(T, 1, device="cuda")
    w[::3] = 2.0
    X = pb.dispatch(x, slots)
    for r in steps(T):
        assert torch.equal(X[T - r.stop:T - r.start].flip(0), x[r])
    Y = pb.combine(X, slots, weights=w, residual=x)
    for r in steps(T):
        assert torch.equal(Y[r], (w[r] + 1) * x[r])
    del Y
    dF, dw = pb.combine_backward(x, X, slots, w)
    for r in steps(T):
        assert torch.equal(dF[T - r.stop:T - r.start].flip(0), (w[r] * x[r]).to(t))
        assert torch.equal(dw[r, 0], x[r].float().square().sum(dim=1))


def test_norm_of_many_rows():
    """Rows of as many 1 as -1 are their own normalised rows with eps 0."""
    g = torch.Generator(device="cuda").manual_seed(2)
    N, d, E, t = (1 << 28) + 77, 8, 3, torch.bfloat16
    ends = [3, 1 << 27, 1 << 27, N - 5]
    off = torch.tensor(ends, dtype=torch.int32, device="cuda")
    x = torch.tensor([1, -1, -1, 1, 1, 1, -1, -1], dtype=t, device="cuda").repeat(N, 1)
    for r in steps(N):
        x[r] *= 2 * torch.randint(0, 2, (len(x[r]), 1), generator=g, device="cuda",
                                  dtype=torch.int8).to(t) - 1
    w = torch.randint(1, 3, (E, d), generator=g, device="cuda").to(t)
    b = signs(g, E, d, dtype=t)
    y, mean, rstd = pb.expert_norm(x, w, b, off, eps=0.0, out=torch.full_like(x, 7.0))
    dy = signs(g, N, d, dtype=t)
    dx, dw, db = pb.expert_norm_backward(dy, x, w, mean, rstd, off, out=torch.full_like(x, 7.0))
    for z in (y, dx):
        assert bool((z[:3] == 7).all()) and bool((z[N - 5:] == 7).all())
    for e in range(E):
        want_w, want_b = torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")
        for r in steps(ends[e + 1] - ends[e]):
            r = slice(ends[e] + r.start, ends[e] + r.stop)
            xr, dr = x[r].float(), dy[r].float()
            assert torch.equal(y[r], (xr * w[e].float() + b[e].float()).to(t))
            assert not torch.any(mean[r]) and bool((rstd[r] == 1).all())
            h = dr * w[e].float()
            want = h - h.sum(dim=1, keepdim=True) / d - xr * ((h * xr).sum(dim=1, keepdim=True) / d)
            assert torch.equal(dx[r], want.to(t))
            want_w += (dr * xr).sum(dim=0)
            want_b += dr.sum(dim=0)
        assert torch.equal(dw[e], want_w) and torch.equal(db[e], want_b)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_products_of_many_rows(dtype):
    """More tiles than a launch has blocks, by eight columns."""
    g = torch.Generator(device="cuda").manual_seed(3)
    N, E, K, O = (1 << 28) + 77, 3, 8, 8
    ends = [3, 1 << 27, 1 << 27, N - 5]
    off = torch.tensor(ends, dtype=torch.int32, device="cuda")
    x, dy, w = (signs(g, *s, dtype=dtype) for s in ((N, K), (N, O), (E, O, K)))
    y = pb.expert_linear(x, w, off, out=torch.full_like(dy, 7.0))
    dx = pb.expert_linear_dx(dy, w, off, out=torch.full_like(x, 7.0))
    dw, db = pb.expert_linear_dw(dy, x, off)
    for z in (y, dx):
        assert bool((z[:3] == 7).all()) and bool((z[N - 5:] == 7).all())
    for e in range(E):
        want, want_b = torch.zeros(O, K, device="cuda"), torch.zeros(O, device="cuda")
        for r in steps(ends[e + 1] - ends[e]):
            r = slice(ends[e] + r.start, ends[e] + r.stop)
            xr, dr, we = x[r].float(), dy[r].float(), w[e].float()
            assert torch.equal(y[r].float(), sum(xr[:, i, None] * we[:, i] for i in range(K)))
            assert torch.equal(dx[r].float(), sum(dr[:, i, None] * we[i] for i in range(O)))
            want += torch.stack([(dr[:, i, None] * xr).sum(dim=0) for i in range(O)])
            want_b += dr.sum(dim=0)
        assert torch.equal(dw[e], want) and torch.equal(db[e], want_b)

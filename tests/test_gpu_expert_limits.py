"""The expert layer's calls at the largest sizes they take: rows and matrices of 2^20 columns,
2048 experts. Values are whole numbers, so that sums are exact in fp32 (below 2^24) and results
are equal, or rounded once."""
import pytest
import torch

import paper_2103_16716_amd as pb

pytestmark = pytest.mark.gpu

WIDEST = 1 << 20
TYPES = [torch.bfloat16, torch.float32]


def whole(g, *shape, dtype):
    return torch.randint(-1, 2, shape, generator=g, device="cuda", dtype=torch.int8).to(dtype)


def product(a, b):
    """a b^T of whole numbers, exact in fp64."""
    return a.double() @ b.double().t().contiguous()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K,O", [(WIDEST, 24), (24, WIDEST)])
def test_widest_products(K, O, dtype):
    g = torch.Generator(device="cuda").manual_seed(K)
    ends = [2, 131, 131, 190]
    N, E = 192, 3
    off = torch.tensor(ends, dtype=torch.int32, device="cuda")
    x, dy, w = (whole(g, *s, dtype=dtype) for s in ((N, K), (N, O), (E, O, K)))
    y = pb.expert_linear(x, w, off, out=torch.full_like(dy, 7.0))
    dx = pb.expert_linear_dx(dy, w, off, out=torch.full_like(x, 7.0))
    dw, db = pb.expert_linear_dw(dy, x, off)
    for e in range(E):
        r = slice(ends[e], ends[e + 1])
        assert torch.equal(y[r], product(x[r], w[e]).to(dtype))
        assert torch.equal(dx[r], product(dy[r], w[e].t()).to(dtype))
        assert torch.equal(dw[e].double(), product(dy[r].t(), x[r].t()))
        assert torch.equal(db[e].double(), dy[r].double().sum(dim=0))
    for z in (y, dx):
        assert bool((z[:2] == 7).all()) and bool((z[190:] == 7).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_widest_moves(dtype):
    g = torch.Generator(device="cuda").manual_seed(3)
    T, k = 5, 3
    slots = torch.randperm(T * k, generator=g, device="cuda").to(torch.int32).view(T, k)
    slots[2, 1] = -1
    some = slots >= 0
    at = slots.clamp(min=0).long()
    x, F = whole(g, T, WIDEST, dtype=dtype), whole(g, T * k, WIDEST, dtype=dtype)
    w = torch.randint(1, 4, (T, k), generator=g, device="cuda").float()
    X = pb.dispatch(x, slots, weights=w)
    Y = pb.combine(F, slots, weights=w, residual=x)
    dF, dw = pb.combine_backward(x, F, slots, w)
    terms = F[at].double() * (w * some).double()[:, :, None]
    assert torch.equal(Y.double(), x.double() + terms.sum(dim=1))
    assert torch.equal(dw.double(), (F[at].double() * x.double()[:, None]).sum(dim=2) * some)
    for got in (X, dF):
        want = w[:, :, None] * x.float()[:, None]
        assert torch.equal(got[at][some].float(), want[some])


def test_most_experts_in_the_largest_tile():
    """2048 experts of uneven rows, every eleventh without any, in tiles of 256 x 256."""
    g = torch.Generator(device="cuda").manual_seed(5)
    E, K, O = 2048, 16, 2056
    n = torch.randint(100, 220, (E,), generator=g, device="cuda")
    n[3::11] = 0
    off = torch.cat([n.new_zeros(1), n.cumsum(0)]).to(torch.int32)
    N = int(off[-1])
    assert pb.expert_linear_tile(pb.BASE_PRODUCT_Y, N, E, K, O, pb.BASE_BF16) == (256, 256, 1)
    e = torch.repeat_interleave(torch.arange(E, device="cuda"), n)
    x, w = (whole(g, *s, dtype=torch.bfloat16) for s in ((N, K), (E, O, K)))
    y = pb.expert_linear(x, w, off)
    for r0 in range(0, N, 1 << 14):   # (K is small: the products of each row with its matrix)
        r = slice(r0, r0 + (1 << 14))
        want = torch.zeros(len(y[r]), O, device="cuda")
        for i in range(K):
            want += x[r, i, None].float() * w[:, :, i][e[r]].float()
        assert torch.equal(y[r].float(), want)

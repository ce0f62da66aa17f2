"""Calls of the expert layer that include/base.h allows and the layer itself does not make:
results that are left out, norms through a sort vector with holes, copies of any bits."""
import numpy as np
import pytest
import torch

import paper_2103_16716_amd as pb
from test_gpu_experts import some_offsets, rng_of

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float32]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def ptr(t):
    return None if t is None else t.data_ptr()


def code(dtype):
    return pb.BASE_BF16 if dtype == torch.bfloat16 else pb.BASE_F32


def stream():
    return torch.cuda.current_stream().cuda_stream


def guarded(n, dtype=torch.float32):
    """A result of n elements between two rows that must stay as they are."""
    buf = torch.full((n + 128,), 7, dtype=dtype, device="cuda")
    return buf, buf[64:64 + n]


def untouched(buf, n):
    return bool((buf[:64] == 7).all()) and bool((buf[64 + n:] == 7).all())


@pytest.mark.parametrize("T,E,k", [(40, 16, 3), (3000, 64, 2), (2000, 600, 9)])
def test_routing_without_scores(T, E, k):
    S = torch.randn(T, E, generator=gen(T), device="cuda")
    want = pb.topk_assign(S, k)
    n = T * k
    ws = torch.empty(pb.topk_workspace_size(T, E, k), dtype=torch.uint8, device="cuda")
    got = {name: guarded(m, torch.int32) for name, m in
           (("assign", n), ("perm", n), ("slots", n), ("offsets", E + 1))}
    st = pb.lib().base_topk_assign(S.data_ptr(), T, E, k, ptr(got["assign"][1]), None,
                                   ptr(got["perm"][1]), ptr(got["slots"][1]),
                                   ptr(got["offsets"][1]), ws.data_ptr(), ws.nbytes, stream())
    assert st == pb.BASE_OK
    for name, (buf, out) in got.items():
        assert torch.equal(out, getattr(want, name).view(-1)) and untouched(buf, out.numel()), name


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,E,K,O", [(100, 3, 264, 200), (5000, 3, 264, 40), (3300, 16, 2040, 1000)])
def test_products_without_db(N, E, K, O, dtype):
    """dW whole, in parts and (bf16) in the large tile."""
    g = gen(N)
    x, dy = (torch.randn(N, n, generator=g, device="cuda").to(dtype) for n in (K, O))
    off = torch.from_numpy(some_offsets(rng_of(N), N, E)).cuda()
    want = pb.expert_linear_dw(dy, x, off)[0]
    n = pb.expert_linear_workspace_size(pb.BASE_PRODUCT_DW, N, E, K, O, code(dtype))
    ws = torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
    buf, dw = guarded(E * O * K)
    st = pb.lib().base_expert_linear_dw(dy.data_ptr(), x.data_ptr(), off.data_ptr(), ptr(dw), None, N,
                                        E, K, O, code(dtype), ws.data_ptr(), ws.nbytes, stream())
    assert st == pb.BASE_OK
    assert torch.equal(dw, want.view(-1)) and untouched(buf, dw.numel())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,E,d", [(200, 5, 1000), (40, 2, 9000)])
def test_norm_without_dbias(N, E, d, dtype):
    g = gen(d)
    x, dy = (torch.randn(N, d, generator=g, device="cuda").to(dtype) for _ in range(2))
    w = torch.randn(E, d, generator=g, device="cuda").to(dtype)
    off = torch.from_numpy(some_offsets(rng_of(N), N, E)).cuda()
    _, mean, rstd = pb.expert_norm(x, w, None, off)
    want = pb.expert_norm_backward(dy, x, w, mean, rstd, off)
    ws = torch.empty(pb.expert_norm_workspace_size(N, E, d), dtype=torch.uint8, device="cuda")
    dx, (buf, dw) = torch.empty_like(x), guarded(E * d)
    st = pb.lib().base_expert_norm_backward(
        dy.data_ptr(), x.data_ptr(), None, N, 1, w.data_ptr(), mean.data_ptr(), rstd.data_ptr(),
        off.data_ptr(), None, dx.data_ptr(), ptr(dw), None, N, E, d, code(dtype), ws.data_ptr(),
        ws.nbytes, stream())
    assert st == pb.BASE_OK
    assert torch.equal(dx, want[0]) and torch.equal(dw, want[1].view(-1)) and untouched(buf, E * d)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("N,x_rows,k,d", [(300, 77, 5, 264), (90, 1000, 2, 2056), (33, 4, 9, 8200),
                                          (5, 1, 3, 8)])
def test_norm_through_a_sort_vector_with_holes(N, x_rows, k, d, shared, dtype):
    """perm entries below 0 or past the rows there are have no source: their rows of y and dx
    stay, and the gradients by the weights are those of the other rows. Sources may repeat and
    be left out. The bits of the same rows laid out by the caller."""
    r = rng_of(N, d)
    perm = r.integers(0, x_rows * k, N).astype(np.int32)
    hole = r.random(N) < 0.3
    perm[hole] = r.choice([-1, -7, x_rows * k, np.iinfo(np.int32).max, np.iinfo(np.int32).min],
                          hole.sum())
    live = torch.from_numpy(~hole).cuda()
    g = gen(N)
    E = 1 if shared else 4
    off = None if shared else torch.from_numpy(some_offsets(r, N, E)).cuda()
    x = torch.randn(x_rows, d, generator=g, device="cuda").to(dtype)
    w, b = (torch.randn(E, d, generator=g, device="cuda").to(dtype) for _ in range(2))
    dy = torch.randn(N, d, generator=g, device="cuda").to(dtype)
    p = torch.from_numpy(perm).cuda()
    where = dict(offsets=off, perm=p, k=k)
    seven = torch.full((N, d), 7.0, dtype=dtype, device="cuda")
    y, mean, rstd = pb.expert_norm(x, w, b, out=seven.clone(), **where)
    dx, dw, db = pb.expert_norm_backward(dy, x, w, mean, rstd, out=seven.clone(), **where)
    laid = x[torch.where(live, p, 0).long() // k]
    zero = torch.where(live[:, None], dy, torch.zeros_like(dy))   # (adds nothing to the sums)
    y1, mean1, rstd1 = pb.expert_norm(laid, w, b, offsets=off)
    dx1, dw1, db1 = pb.expert_norm_backward(zero, laid, w, mean1, rstd1, offsets=off)
    for got, want in ((y, y1), (dx, dx1)):
        assert torch.equal(got[live], want[live]) and bool((got[~live] == 7).all())
    assert torch.equal(mean[live], mean1[live]) and torch.equal(rstd[live], rstd1[live])
    assert torch.equal(dw, dw1) and torch.equal(db, db1)


@pytest.mark.parametrize("dtype", TYPES)
def test_dispatch_copies_any_bits(dtype):
    """Without weights a copy bit for bit: NaN of every kind, infinities, subnormal numbers."""
    T, k, d = 129, 3, 72
    i = torch.int16 if dtype == torch.bfloat16 else torch.int32
    most = torch.iinfo(i).max
    bits = torch.randint(-most - 1, most, (T, d), generator=gen(4), device="cuda", dtype=i)
    bits[0] = torch.iinfo(i).max          # a NaN
    slots = torch.randperm(T * k, generator=gen(5), device="cuda").to(torch.int32).view(T, k)
    out = pb.dispatch(bits.view(dtype), slots)
    assert torch.equal(out.view(i)[slots.long()], bits[:, None].expand(T, k, d))

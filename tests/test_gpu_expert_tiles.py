"""The experts' products in tiles that the sizes of the other tests do not lead to, with the
choice asserted. Bounds as in the other tests of the products."""
import numpy as np
import pytest
import torch

import paper_2103_16716_amd as pb
from test_gpu_experts import STEP, U, near_product, rng_of

PRODUCTS = {"y": pb.BASE_PRODUCT_Y, "dx": pb.BASE_PRODUCT_DX, "dw": pb.BASE_PRODUCT_DW}
DTYPES = {"bf16": (pb.BASE_BF16, torch.bfloat16), "f32": (pb.BASE_F32, torch.float32)}
BEFORE, BEHIND = 5, 3   # rows of no expert

# product, type, rows, experts, K, O, tile
CASES = [
    # dW in tiles that blocks go through in turn, two or three to a block, by XCD (32 tiles an
    # expert and more) and by block; the last of rows and columns not full
    ("dw", "bf16", 3300, 16, 2040, 1000, (256, 256)),
    ("dw", "bf16", 6500, 40, 1000, 1016, (256, 256)),
    ("dw", "bf16", 1500, 5, 1016, 8184, (256, 256)),
    # the larger tile of fp32
    ("y", "f32", 5000, 5, 136, 1640, (64, 128)),
    ("dx", "f32", 5000, 5, 1640, 136, (64, 128)),
    # more experts than a wave finds at a time, and than the threads of a block
    ("y", "bf16", 20000, 100, 72, 2056, (256, 256)),
    ("y", "bf16", 121000, 600, 72, 1032, (256, 256)),
    ("dx", "bf16", 26000, 100, 2056, 72, (256, 256)),
    ("dx", "bf16", 154000, 600, 1032, 72, (256, 256)),
]


def uneven(rng, E, N):
    """Rows of E experts, N in all: every seventh has none, one has a single row."""
    p = rng.random(E) ** 2 + 0.05
    p[3::7] = 0.0
    n = rng.multinomial(N - 1, p / p.sum())
    n[np.flatnonzero(p == 0.0)[0]] = 1
    return n


@pytest.mark.gpu
@pytest.mark.parametrize("product,dtype,N,E,K,O,tile", CASES)
def test_tile(product, dtype, N, E, K, O, tile):
    code, t = DTYPES[dtype]
    M = N + BEFORE + BEHIND
    assert pb.expert_linear_tile(PRODUCTS[product], M, E, K, O, code) == (*tile, 1)
    counts = uneven(rng_of(N, E, K), E, N)
    ends = np.cumsum(np.concatenate([[BEFORE], counts]))
    off = torch.tensor(ends, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(N + K)

    def rows(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(t)

    x, dy = rows(M, K), rows(M, O)
    for outside in (x, dy):
        outside[:BEFORE], outside[N + BEFORE:] = float("nan"), float("inf")
    w = rows(E, O, K, scale=K ** -0.5)
    experts = [(e, slice(int(ends[e]), int(ends[e + 1]))) for e in range(E)]
    if product == "dw":
        got = [pb.expert_linear_dw(dy, x, off) for _ in range(3)]
        dw, db = got[0]
        for e, r in experts:
            near_product(dw[e], dy[r].t().contiguous(), x[r], int(counts[e]), U)
            want, mag = dy[r].double().sum(dim=0), dy[r].double().abs().sum(dim=0)
            assert bool(((db[e].double() - want).abs() <= (int(counts[e]) + 1) * U * mag).all())
        assert all(torch.equal(a, dw) and torch.equal(b, db) for a, b in got[1:])
        return
    step = STEP[dtype]
    bias, res, u = rows(E, O, scale=0.1), rows(M, O), rows(M, K)
    out = torch.full_like(dy if product == "y" else x, 7.0)
    if product == "y":
        plain = pb.expert_linear(x, w, off, out=out.clone())
        got = pb.expert_linear(x, w, off, bias=bias, relu=True, residual=res, out=out.clone())
        again = pb.expert_linear(x, w, off, bias=bias, relu=True, residual=res, out=out.clone())
    else:
        plain = pb.expert_linear_dx(dy, w, off, out=out.clone())
        got = pb.expert_linear_dx(dy, w, off, relu_of=u, out=out.clone())
        again = pb.expert_linear_dx(dy, w, off, relu_of=u, out=out.clone())
    assert torch.equal(got, again)
    for e, r in experts:
        a, b = (x, w[e].t().contiguous()) if product == "y" else (dy, w[e])
        near_product(plain[r], a[r], b, b.shape[0], step)
        if product == "dx":
            assert torch.equal(got[r], torch.where(u[r] > 0, plain[r], torch.zeros_like(plain[r])))
            continue
        a, b, bias_e, res_e = a[r].double(), b.double(), bias[e].double(), res[r].double()
        want = (a @ b + bias_e).clamp(min=0) + res_e
        mag = a.abs() @ b.abs() + bias_e.abs()
        bound = (K + 3) * U * mag + U * (mag + res_e.abs())
        assert bool(((got[r].double() - want).abs() <= bound + step * (want.abs() + bound)).all())
    for y in (plain, got):
        assert bool((y[:BEFORE] == 7).all()) and bool((y[N + BEFORE:] == 7).all())

"""Outputs of the expert layer's calls that overlap an input or each other are refused, on the
host: every pair, at its first and its last bytes. No call here is valid, and none reaches the
GPU."""
import pytest

import paper_2103_16716_amd as pb
from paper_2103_16716_amd import build as pbuild

FIRST, APART = 1 << 27, 1 << 26   # stand-in addresses, never dereferenced
T, E, K, d, O, N = 24, 4, 2, 64, 40, 48
F32 = pb.BASE_F32


@pytest.fixture(scope="module", autouse=True)
def library():
    if pbuild.is_stale():
        pbuild.build()


def calls():
    """name, function, its arguments (buffers by name), buffers (bytes), outputs, pairs that may
    be the same matrix."""
    L = pb.lib()
    ws = {"topk": pb.topk_workspace_size(T, E, K), "norm": pb.expert_norm_workspace_size(N, E, d)}
    route = dict(assign=T * K * 4, scores=T * K * 4, perm=T * K * 4, slots=T * K * 4,
                 offsets=(E + 1) * 4, ws=ws["topk"])
    yield ("topk_assign", L.base_topk_assign,
           ("S", T, E, K, "assign", "scores", "perm", "slots", "offsets", "ws", ws["topk"], None),
           dict(S=T * E * 4, **route), ("assign", "scores", "perm", "slots", "offsets", "ws"), ())
    yield ("sort_by_expert", L.base_sort_by_expert,
           ("assign", T, E, K, "perm", "slots", "offsets", "ws", ws["topk"], None),
           {n: b for n, b in route.items() if n != "scores"}, ("perm", "slots", "offsets", "ws"), ())
    pairs, row = T * K * 4, d * 4
    yield ("dispatch", L.base_dispatch, ("x", "w", "slots", "out", T, K, d, F32, None),
           dict(x=T * row, w=pairs, slots=pairs, out=T * K * row), ("out",), ())
    yield ("combine", L.base_combine, ("F", "w", "slots", "residual", "out", T, K, d, F32, None),
           dict(F=T * K * row, w=pairs, slots=pairs, residual=T * row, out=T * row), ("out",),
           (("out", "residual"),))
    yield ("combine_backward", L.base_combine_backward,
           ("dY", "F", "w", "slots", "dF", "dw", T, K, d, F32, None),
           dict(dY=T * row, F=T * K * row, w=pairs, slots=pairs, dF=T * K * row, dw=pairs),
           ("dF", "dw"), ())
    sizes = dict(x=T * row, perm=N * 4, weight=E * row, bias=E * row, offsets=(E + 1) * 4,
                 y=N * row, mean=N * 4, rstd=N * 4)
    yield ("expert_norm", L.base_expert_norm,
           ("x", "perm", T, K, "weight", "bias", "offsets", "y", "mean", "rstd", N, E, d, 1e-5, F32,
            None), sizes, ("y", "mean", "rstd"), ())
    sizes = dict(dy=N * row, x=T * row, perm=N * 4, weight=E * row, mean=N * 4, rstd=N * 4,
                 offsets=(E + 1) * 4, residual=N * row, dx=N * row, dweight=E * row, dbias=E * row,
                 ws=ws["norm"])
    yield ("expert_norm_backward", L.base_expert_norm_backward,
           ("dy", "x", "perm", T, K, "weight", "mean", "rstd", "offsets", "residual", "dx", "dweight",
            "dbias", N, E, d, F32, "ws", ws["norm"], None), sizes, ("dx", "dweight", "dbias", "ws"),
           (("dx", "dy"), ("dx", "residual")))
    n, k, o = 64, 4096, 512     # (in parts, as the next two)
    wsb = pb.expert_linear_workspace_size(pb.BASE_PRODUCT_Y, n, 1, k, o, F32)
    assert wsb > 0
    sizes = dict(x=n * k * 4, w=o * k * 4, bias=o * 4, residual=n * o * 4, offsets=8, y=n * o * 4,
                 ws=wsb)
    yield ("expert_linear", L.base_expert_linear,
           ("x", "w", "bias", "residual", "offsets", "y", n, 1, k, o, 1, F32, "ws", wsb, None),
           sizes, ("y", "ws"), (("y", "residual"),))
    k, o = o, k
    wsb = pb.expert_linear_workspace_size(pb.BASE_PRODUCT_DX, n, 1, k, o, F32)
    assert wsb > 0
    sizes = dict(dy=n * o * 4, w=o * k * 4, relu_of=n * k * 4, offsets=8, dx=n * k * 4, ws=wsb)
    yield ("expert_linear_dx", L.base_expert_linear_dx,
           ("dy", "w", "relu_of", "offsets", "dx", n, 1, k, o, F32, "ws", wsb, None), sizes,
           ("dx", "ws"), (("dx", "relu_of"),))
    n, k, o = 4096, 64, 64
    wsb = pb.expert_linear_workspace_size(pb.BASE_PRODUCT_DW, n, 1, k, o, F32)
    assert wsb > 0
    yield ("expert_linear_dw", L.base_expert_linear_dw,
           ("dy", "x", "offsets", "dw", "db", n, 1, k, o, F32, "ws", wsb, None),
           dict(dy=n * o * 4, x=n * k * 4, offsets=8, dw=o * k * 4, db=o * 4, ws=wsb),
           ("dw", "db", "ws"), ())


NAMES = ["topk_assign", "sort_by_expert", "dispatch", "combine", "combine_backward", "expert_norm",
         "expert_norm_backward", "expert_linear", "expert_linear_dx", "expert_linear_dw"]


def test_every_call_is_here():
    assert [c[0] for c in calls()] == NAMES
    for _, f, args, sizes, outputs, _ in calls():
        assert {a for a in args if isinstance(a, str)} == set(sizes) >= set(outputs)
        assert len(args) == len(f.argtypes)


@pytest.mark.parametrize("name", NAMES)
def test_overlaps(name):
    _, f, args, sizes, outputs, same = next(c for c in calls() if c[0] == name)
    assert all(b <= APART - 512 for b in sizes.values())
    apart = {n: FIRST + i * APART for i, n in enumerate(sizes)}
    for out in outputs:
        for other in sizes:
            if other == out:
                continue
            # the output's first bytes in the other's last ones, and the other way round (a
            # workspace, and addresses that others must be multiples of, on 256 bytes)
            into = apart[other] + (sizes[other] - 1) // 256 * 256
            before = apart[other] - (sizes[out] - 1) // 256 * 256
            for at in {into, before, apart[other]}:
                if at == apart[other] and ((out, other) in same or (other, out) in same):
                    continue
                where = {**apart, out: at}
                st = f(*[where[a] if isinstance(a, str) else a for a in args])
                assert st == pb.BASE_ERR_INVALID_ARG, (out, other, at - apart[other])

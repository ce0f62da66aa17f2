"""A whole layer with k experts a token on the GPU, element by element against the oracle."""
import textwrap

import pytest
import torch

import paper_2103_16716_amd as pb
from gpu_common import dev
from layer_common import PARAMETERS, layer_bounds
from test_gpu_experts import block, block_inputs, close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k", [1, 2, 4])
@pytest.mark.parametrize("T,E,d,inner", [(96, 6, 64, 256), (333, 5, 136, 520)])
def test_every_gradient(T, E, d, inner, k):
    """The layer in fp32 with padded tokens: its result and the gradient of every element of
    the inputs, the weights and the parameters, within the roundings of its steps."""
    H, S, p, dOut = block_inputs(T=T, E=E, d=d, inner=inner, seed=k)
    got = block(dev(H), dev(S), k, {n: dev(v) for n, v in p.items()}, dev(dOut))
    c, g, bound = layer_bounds(H, S, k, p, dOut)
    close(got["out"], c["out"], bound["out"])
    close(got["dw"], g["w"], bound["w"])
    close(got["dH"], g["H"], bound["H"])
    for name in PARAMETERS:
        close(got[name], g[name], bound[name])


def documented():
    """The program in the documentation of paper_2103_16716_amd.experts."""
    lines = pb.experts.__doc__.splitlines()
    return textwrap.dedent("\n".join(x for x in lines if x.startswith("    ") or not x.strip()))


def test_documented_layer_of_a_padded_batch():
    """Tokens without an expert, and with fewer than k, have finite weights, and no NaN reaches
    the scores' gradient (a softmax over a row of -inf has NaN in it)."""
    k = 2
    H, S, p, dOut = block_inputs(T=150, E=6, d=64, inner=256)
    names = {**vars(pb), "torch": torch, "H": dev(H), "S": dev(S), "dOut": dev(dOut)}
    names.update((n, dev(v)) for n, v in p.items())
    exec(compile(documented(), "experts.__doc__", "exec"), names)
    c, g, bound = layer_bounds(H, S, k, p, dOut)
    assert (c["assign"] < 0).all(axis=1).any() and (c["assign"] >= 0).sum(axis=1).min() == 0
    assert torch.isfinite(names["weights"]).all()
    close(names["out"], c["out"], bound["out"])
    for name in PARAMETERS + ("H", "S"):
        close(names["d" + name], g[name], bound[name])

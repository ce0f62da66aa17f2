"""A whole layer with k experts a token on the GPU, element by element against the oracle."""
import pytest

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

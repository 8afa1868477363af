"""attt_gated_ffn_backward with a NaN among the forward call's g and u: the gradients that the formula
makes NaN are, and no others.  dg = dh u act'(g) takes it from g and from u, du = dh act(g) from g
alone, a row of dx from its dg and du."""
import pytest
import torch

from paper_2607_03441_gb300 import attt, build
from tests.gpu_util import DEV
from tests.test_gpu_gated_ffn import Case

pytestmark = pytest.mark.gpu

SHAPES = [  # L, d, f, r: few rows, whole tiles, K pieces and their sum
    (5, 64, 128, 8), (40, 4104, 4104, 0), (300, 128, 264, 8), (300, 3584, 64, 16),
]


@pytest.fixture(scope="module", autouse=True)
def _library():
    build.build()


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
def test_nan_factors(shape, act):
    c = Case(*shape, act=act)
    L, _, f, _ = shape
    want = attt.attt_gated_ffn_backward(c.dy, *c.W, c.g, c.u, **c.kw)
    at_g, at_u = (torch.zeros(L, f, dtype=torch.bool, device=DEV) for _ in range(2))
    at_g[1, 5] = at_g[2, f - 1] = at_u[2, f - 1] = at_u[L - 1, 7] = True
    nan = float("nan")
    dx, dg, du = attt.attt_gated_ffn_backward(c.dy, *c.W, c.g.masked_fill(at_g, nan), c.u.masked_fill(at_u, nan), **c.kw)
    assert attt.attt_device_status() == 0
    assert torch.equal(torch.isnan(dg), at_g | at_u) and torch.equal(torch.isnan(du), at_g)
    assert torch.equal(dg[~(at_g | at_u)], want[1][~(at_g | at_u)]) and torch.equal(du[~at_g], want[2][~at_g])
    rows = (at_g | at_u).any(1)
    assert torch.isnan(dx[rows]).all() and torch.equal(dx[~rows], want[0][~rows])

"""The gradient of a frozen layer norm: no sums for its weight and bias, and what the
policy-gradient example allocates in a round."""
import pytest
import torch

from examples import policy_update as ex
from paper_2607_03441_gb300 import attt, build
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _library():
    build.build()


@pytest.mark.parametrize("L,d,dtype", [(0, 64, torch.float32), (1, 1, torch.float32), (300, 777, torch.bfloat16),
                                       (2500, 512, torch.bfloat16), (20, 9000, torch.float32)])
def test_without_weights(L, d, dtype):
    g = torch.Generator(device=DEV).manual_seed(L + d)
    x, dy = (torch.randn(L, d, generator=g, device=DEV).to(dtype) for _ in range(2))
    gamma = torch.randn(d, generator=g, device=DEV)
    _, mean, rstd = attt.attt_layer_norm_forward(x, gamma)
    want = attt.attt_layer_norm_backward(dy, x, gamma, mean, rstd)
    launches = attt.attt_kernel_launches()
    dx, dgamma, dbeta = attt.attt_layer_norm_backward(dy, x, gamma, mean, rstd, weights=False)
    assert attt.attt_kernel_launches() - launches == (1 if L else 0)
    assert dgamma is None and dbeta is None and torch.equal(dx, want[0])
    # one of the two, where a tensor for it is given
    own = torch.full((d,), 9.0, device=DEV)
    _, dgamma, dbeta = attt.attt_layer_norm_backward(dy, x, gamma, mean, rstd, dbeta=own, weights=False)
    assert dgamma is None and dbeta is own and torch.equal(own, want[2])


def test_a_round_allocates_only_its_small_results():
    """Per row, not per value of a row."""
    L, d, V, r = 4, 4096, 3000, 8
    g = torch.Generator(device=DEV).manual_seed(1)

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device=DEV) * std).to(torch.bfloat16)

    p = ex.Policy(normal(d, d, std=d ** -0.5), normal(V, d, std=d ** -0.5), normal(d, r), normal(r, d), L)
    x, tokens = normal(L, d), torch.zeros(L, dtype=torch.int32, device=DEV)
    adv = torch.ones(L, device=DEV)
    p.gradients(x, tokens, adv, beta=0.01)
    taken = []
    empty = torch.empty
    try:
        torch.empty = lambda *a, **kw: taken.append(empty(*a, **kw)) or taken[-1]
        p.gradients(x, tokens, adv, beta=0.01)
    finally:
        torch.empty = empty
    assert taken and max(t.numel() for t in taken) <= L

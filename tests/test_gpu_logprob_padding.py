"""Rows of padding in the gradient of log probabilities: without a token (-1) and an
entropy weight they give 0, whatever they hold, and leave the other rows alone."""
import pytest
import torch

from paper_2607_03441_gb300 import attt, build
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _library():
    build.build()


@pytest.mark.parametrize("entropy", [False, True])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), 3e38])
@pytest.mark.parametrize("L,d,V", [(3, 64, 700), (40, 136, 5000), (300, 1608, 3001), (700, 264, 2100)])
def test_padding(L, d, V, value, entropy):
    g = torch.Generator(device=DEV).manual_seed(L)
    h = torch.randn(L, d, generator=g, device=DEV).to(torch.bfloat16)
    W = (torch.randn(V, d, generator=g, device=DEV) * 0.05).to(torch.bfloat16)
    tgt = torch.randint(0, V, (L,), generator=g, device=DEV, dtype=torch.int32)
    a, b = torch.randn(L, generator=g, device=DEV), torch.rand(L, generator=g, device=DEV) if entropy else None
    pad = torch.arange(L, device=DEV) % 3 == 1

    def grad(x, t, bb):
        f = attt.attt_logprob_forward(x, W, t)
        dh = attt.attt_logprob_input_grad(x, W, t, f[2], a, f[1] if entropy else None, bb)
        assert attt.attt_device_status() == 0
        return dh

    want = grad(h, tgt, b)
    assert torch.isfinite(want).all()
    x, t = h.clone(), tgt.clone()
    x[pad], t[pad] = value, -1
    if entropy:
        b = b.masked_fill(pad, 0.0)
    got = grad(x, t, b)
    assert not got[pad].any() and torch.equal(got[~pad], want[~pad])


def test_an_entropy_weight_alone_counts():
    """A row without a token whose entropy counts is no padding."""
    g = torch.Generator(device=DEV).manual_seed(7)
    h = torch.randn(5, 64, generator=g, device=DEV).to(torch.bfloat16)
    W = (torch.randn(900, 64, generator=g, device=DEV) * 0.1).to(torch.bfloat16)
    tgt = torch.full((5,), -1, dtype=torch.int32, device=DEV)
    f = attt.attt_logprob_forward(h, W, tgt)
    b = torch.tensor([0.0, 1.0, -2.0, 0.5, 0.0], device=DEV)
    dh = attt.attt_logprob_input_grad(h, W, tgt, f[2], torch.ones(5, device=DEV), f[1], b).float()
    assert not dh[[0, 4]].any()
    x = h.double().requires_grad_()
    lp = torch.log_softmax(x @ W.double().t(), 1)
    (-(lp.exp() * lp).sum(1) * b.double()).sum().backward()
    # two bf16 for dz, dh rounded once (2^-8 of it), sums of 900 terms in fp32
    assert (dh.double() - x.grad).abs().max() <= 2.0 ** -8 * x.grad.abs().max() + 1e-6

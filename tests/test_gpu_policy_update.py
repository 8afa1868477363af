"""The policy-gradient example: its gradients against fp64 autograd through the same
chain, and what its updates do."""
import numpy as np
import pytest
import torch

from examples import policy_update as ex
from paper_2607_03441_gb300 import attt, build
from tests.gpu_util import DEV, rel_l2

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _library():
    build.build()


class _Round(torch.autograd.Function):
    """Rounding to bf16 whose gradient passes through."""

    @staticmethod
    def forward(ctx, x):
        return x.to(torch.bfloat16).double()

    @staticmethod
    def backward(ctx, g):
        return g


@pytest.mark.parametrize("L,d,V,r", [(1, 64, 1000, 8), (45, 136, 3001, 16), (300, 520, 5000, 40)])
def test_gradients(L, d, V, r):
    """Against autograd of the whole chain in fp64, with s (x A), h and n rounded to bf16
    as the calls store them.  What is left are the roundings of G, dn, dh and the adapter
    products, 2^-8 of each at most: 2^-6 of the norm together."""
    g = torch.Generator(device=DEV).manual_seed(L + d)

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device=DEV) * std).to(torch.bfloat16)

    W0, Wlm, x = normal(d, d, std=d ** -0.5), normal(V, d, std=2 * d ** -0.5), normal(L, d)
    A, B = normal(d, r, std=d ** -0.5), normal(r, d, std=0.3)
    tokens = torch.randint(0, V, (L,), generator=g, device=DEV, dtype=torch.int32)
    adv = torch.randn(L, generator=g, device=DEV)
    p = ex.Policy(W0, Wlm, A, B, L, scale=0.5, inv_temp=1.25)
    dA, dB, logp, entropy = p.gradients(x, tokens, adv, beta=0.05)
    assert attt.attt_device_status() == 0

    A64, B64 = A.double().requires_grad_(), B.double().requires_grad_()
    h = _Round.apply(x.double() @ W0.double() + _Round.apply(0.5 * (x.double() @ A64)) @ B64)
    n = _Round.apply(torch.nn.functional.layer_norm(h, (d,), eps=1e-5))
    lp = torch.log_softmax(n @ Wlm.double().t() * 1.25, dim=1)
    got = lp.gather(1, tokens.long()[:, None])[:, 0]
    H = -(lp.exp() * lp).sum(1)
    (-(adv.double() * got + 0.05 * H).mean()).backward()
    assert rel_l2(dA.cpu(), A64.grad.cpu()) <= 2.0 ** -6
    assert rel_l2(dB.cpu(), B64.grad.cpu()) <= 2.0 ** -6
    # a value of h or n on the other side of a rounding moves a logit by 2^-8 of one term at most
    for a, b in ((logp, got), (entropy, H)):
        assert (a.double() - b.detach()).abs().max().item() <= 2.0 ** -6


def test_updates_move_the_policy():
    """Rewarded tokens become the likelier choice."""
    shares = ex.train(rows=128, width=256, vocab=4096, rank=16, rounds=25, verbose=False)
    assert len(shares) == 25
    assert np.mean(shares[-5:]) > np.mean(shares[:5]) + 0.15


def test_rounds_repeat():
    """The same seed gives the same rounds, bit for bit."""
    a = ex.train(rows=64, width=128, vocab=2048, rank=8, rounds=6, verbose=False)
    b = ex.train(rows=64, width=128, vocab=2048, rank=8, rounds=6, verbose=False)
    assert a == b


def test_an_update_in_a_graph():
    """A captured update does what the calls do one by one, bit for bit."""
    L, d, V, r = 70, 128, 3000, 16
    g = torch.Generator(device=DEV).manual_seed(5)

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device=DEV) * std).to(torch.bfloat16)

    W0, Wlm, x = normal(d, d, std=d ** -0.5), normal(V, d, std=2 * d ** -0.5), normal(L, d)
    A, B = normal(d, r, std=d ** -0.5), normal(r, d, std=0.1)
    tokens = torch.randint(0, V, (L,), generator=g, device=DEV, dtype=torch.int32)
    adv = torch.randn(L, generator=g, device=DEV)
    plain, captured = (ex.Policy(W0, Wlm, A, B, L) for _ in range(2))
    for _ in range(3):
        plain.gradients(x, tokens, adv, beta=0.01)
        plain.step(0.02)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.gradients(x, tokens, adv, beta=0.01)
        captured.step(0.02)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(plain.A32, captured.A32) and torch.equal(plain.B32, captured.B32)
    assert attt.attt_device_status() == 0

"""Pins of oracle/operators.py: torch CPU library routines in fp64, finite
differences, closed forms."""
import numpy as np
import pytest
import torch

from oracle import operators as op


def _rng(seed):
    return np.random.default_rng(seed)


def test_logprobs_match_torch():
    r = _rng(0)
    h, W, tgt = r.normal(size=(9, 16)), r.normal(size=(40, 16)), r.integers(-1, 40, 9)
    lp, H, lse, top, ids = op.logprobs(h, W, tgt, 5, 0.7)
    ref = torch.log_softmax(torch.from_numpy(h @ W.T) * 0.7, -1)
    want = np.where(tgt >= 0, ref.numpy()[np.arange(9), np.maximum(tgt, 0)], 0)
    assert np.allclose(lp, want, atol=1e-12)
    assert np.allclose(H, torch.distributions.Categorical(logits=ref).entropy().numpy(), atol=1e-12)
    v, i = ref.topk(5, -1)
    assert np.allclose(top, v.numpy(), atol=1e-12) and np.array_equal(ids, i.numpy())


def test_logprobs_closed_forms():
    h, W = np.zeros((2, 8)), _rng(1).normal(size=(12, 8))
    lp, H, lse, top, ids = op.logprobs(h, W, [3, -1], 4)
    assert np.allclose(lp, [-np.log(12), 0]) and np.allclose(H, np.log(12)) and np.allclose(lse, np.log(12))
    assert np.array_equal(ids, [[0, 1, 2, 3]] * 2)  # equal logits: the lowest ids


def test_logprobs_grad_differences():
    r = _rng(2)
    h, W, tgt = r.normal(size=(6, 8)), r.normal(size=(20, 8)), np.array([0, 5, -1, 19, 7, -1])
    a, b = r.normal(size=6), r.normal(size=6)

    def f(x):
        lp, H, *_ = op.logprobs(x, W, tgt, 0, 0.8)
        return (a * lp + b * H).sum()

    dh, _ = op.logprobs_grad(h, W, tgt, a, b, 0.8)
    for i in np.ndindex(h.shape):
        e = np.zeros_like(h)
        e[i] = 1e-5
        assert abs((f(h + e) - f(h - e)) / 2e-5 - dh[i]) < 1e-8


@pytest.mark.parametrize("bias", [True, False])
def test_layer_norm_matches_torch(bias):
    r = _rng(3)
    x, g = (torch.from_numpy(r.normal(size=s)).requires_grad_() for s in ((5, 12), (12,)))
    b = torch.from_numpy(r.normal(size=12)).requires_grad_() if bias else None
    y = torch.nn.functional.layer_norm(x, (12,), g, b, 1e-5)
    dy = torch.from_numpy(r.normal(size=(5, 12)))
    y.backward(dy)
    got, mean, rstd = op.layer_norm(x.detach().numpy(), g.detach().numpy(), b.detach().numpy() if bias else None)
    assert np.allclose(got, y.detach().numpy(), atol=1e-12)
    dx, dg, db = op.layer_norm_grad(dy.numpy(), x.detach().numpy(), g.detach().numpy(), mean, rstd)
    assert np.allclose(dx, x.grad.numpy(), atol=1e-12) and np.allclose(dg, g.grad.numpy(), atol=1e-12)
    if bias:
        assert np.allclose(db, b.grad.numpy(), atol=1e-12)


@pytest.mark.parametrize("shape", [(4, 30), (30, 4), (7, 7)])
def test_newton_schulz_is_the_polynomial_of_the_singular_values(shape):
    u = _rng(4).normal(size=shape)
    left, s, right = np.linalg.svd(u, full_matrices=False)
    s = s / (np.sqrt((s * s).sum()) + 1e-7)
    for _ in range(5):
        s = op.NS[0] * s + op.NS[1] * s ** 3 + op.NS[2] * s ** 5
    assert np.allclose(op.newton_schulz(u), (left * s) @ right, atol=1e-10)
    assert 0.6 < s.min() and s.max() < 1.3


def test_muon_step_of_zero_gradient_is_decay():
    p = _rng(5).normal(size=(6, 20))
    q, m = op.muon_step(p, 0 * p, 0 * p, 0.1, weight_decay=0.5)
    assert np.allclose(q, p * 0.95) and not m.any()

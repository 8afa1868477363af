"""attt_lora_muon_step at the ends of fp32: gradients whose |u|_F^2 overflows or is far
below eps^2, and entries that are not finite, on every kernel (ranks up to 5, 16, 32,
64).

u is the gradient (no momentum).  The bounds of the finite cases are those of
test_gpu_muon.py: 3e-5 of the update's norm."""
import numpy as np
import pytest
import torch

from oracle import operators as op
from paper_2607_03441_gb300 import attt, build
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu
MAX = float(np.finfo(np.float32).max)
RANKS = [4, 16, 32, 64]


@pytest.fixture(scope="module", autouse=True)
def _library():
    build.build()


def _signs(seed, shape, c):
    """Entries +-c: every row of the r side has the same square, exactly."""
    return (np.random.default_rng(seed).integers(0, 2, shape) * 2 - 1) * c


def _step(dA, dB, eps=1e-7, lr=0.02):
    """The parameters (from 0) of one projection after a step along its gradients."""
    d = [torch.from_numpy(np.ascontiguousarray(v, dtype=np.float32)).to(DEV) for v in (dA, dB)]
    p, m = ([torch.zeros_like(t) for t in d] for _ in range(2))
    attt.attt_lora_muon_step(p[:1], p[1:], d[:1], d[1:], m[:1], m[1:], lr, momentum=0.0, nesterov=False, eps=eps)
    assert attt.attt_device_status() == 0
    return [t.double().cpu().numpy() for t in p]


def _want(g, eps=1e-7, lr=0.02):
    g = np.asarray(g, dtype=np.float32)
    return op.muon_step(np.zeros(g.shape), g, np.zeros(g.shape), lr, 0.0, False, eps=float(np.float32(eps)))[0]


def _near(got, want):
    assert np.linalg.norm(got - want) <= 3e-5 * np.linalg.norm(want)


@pytest.mark.parametrize("r", RANKS)
def test_a_norm_beyond_fp32_is_nan(r):
    """Every diagonal element of the Gram matrix is finite, their sum is not: NaN as a
    whole, and not an update of 0.  The other matrix does not feel it."""
    n = 2000
    big = _signs(r, (n, r), np.sqrt(0.5 * MAX / n))
    fine = np.random.default_rng(r).normal(size=(r, 700)) * 1e-3
    a, b = _step(big, fine)
    assert np.isnan(a).all()
    _near(b, _want(fine))
    a, b = _step(fine.T, big.T)
    assert np.isnan(b).all()
    _near(a, _want(fine.T))


@pytest.mark.parametrize("r", RANKS)
def test_a_norm_just_within_fp32(r):
    n = 2000
    g = _signs(r, (n, r), np.sqrt(0.9 * MAX / (n * r)))
    a, b = _step(g, g.T)
    _near(a, _want(g))
    _near(b, _want(g.T))


@pytest.mark.parametrize("r", RANKS)
@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
def test_an_entry_that_is_not_finite(r, value):
    g = np.random.default_rng(r).normal(size=(900, r)) * 1e-3
    bad = g.copy()
    bad[411, r - 1] = value
    a, b = _step(bad, g.T)
    assert np.isnan(a).all()
    _near(b, _want(g.T))


@pytest.mark.parametrize("r", RANKS)
@pytest.mark.parametrize("size", [0.1, 1.0, 30.0])
def test_a_gradient_of_the_size_of_the_least_eps(r, size):
    eps = 1e-12
    g = np.random.default_rng(r).normal(size=(1500, r))
    g *= size * eps / np.linalg.norm(g)
    a, b = _step(g, g.T[:, :600], eps=eps)
    _near(a, _want(g, eps))
    _near(b, _want(g.T[:, :600], eps))


@pytest.mark.parametrize("r", RANKS)
def test_a_zero_gradient_at_the_least_eps(r):
    a, b = _step(np.zeros((300, r)), np.zeros((r, 200)), eps=1e-12)
    assert not a.any() and not b.any()


@pytest.mark.parametrize("eps", [9e-13, 1e-30, 1e-45])
def test_an_eps_whose_square_fp32_does_not_hold_is_refused(eps):
    launches = attt.attt_kernel_launches()
    with pytest.raises(attt.AtttError) as e:
        _step(np.zeros((40, 8)), np.zeros((8, 40)), eps=eps)
    assert e.value.code == attt.ATTT_ERR_INVALID_ARG
    assert attt.attt_kernel_launches() == launches

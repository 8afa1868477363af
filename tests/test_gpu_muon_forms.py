"""Forms of attt_lora_muon_step that test_gpu_muon.py leaves out, against the fp64
oracle: columns that pass through a CTA's shared memory at ranks 6 to 64, step counts
and settings on every kernel, and the precision of ranks up to 5.

Bounds as there (3e-5 of the update's norm; a further step may multiply what is off by
3.44) but for ranks up to 5.  Their Gram matrix, P and P X are formed in twice 24 bits, so
that nothing of the condition's square is lost; with u exact (no momentum) what is left
is X's rounding, the step's and the update's: 3 half units of 2^-23 of each element, 2^-21
of the norm with room for the oracle's own."""
import numpy as np
import pytest
import torch

from oracle import operators as op
from paper_2607_03441_gb300 import attt, build
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _library():
    build.build()


def _gradients(seed, din, dout, r, cond):
    g = np.random.default_rng(seed)
    fall = np.exp(np.linspace(0, -np.log(cond), r))
    qa, qb = (np.linalg.qr(g.normal(size=(r, r)))[0] for _ in range(2))
    dA = (g.normal(size=(din, r)) * fall) @ qa * 1e-3
    dB = qb @ (fall[:, None] * g.normal(size=(r, dout))) * 1e-3
    return [v.astype(np.float32) for v in (dA, dB)]


def _check(seed, din, dout, r, cond=100.0, tol=3e-5, p_std=0.0, lr=0.02, **kw):
    g = np.random.default_rng(seed + 1)
    grads = _gradients(seed, din, dout, r, cond)
    ps = [(g.normal(size=v.shape) * p_std).astype(np.float32) for v in grads]
    ms = [3 * v for v in grads]
    dev = [[torch.from_numpy(np.ascontiguousarray(v)).to(DEV) for v in vs] for vs in (ps, grads, ms)]
    half = [torch.zeros_like(p, dtype=torch.bfloat16) for p in dev[0]]
    p, d, m = dev
    attt.attt_lora_muon_step(p[:1], p[1:], d[:1], d[1:], m[:1], m[1:], lr, A16s=half[:1], B16s=half[1:], **kw)
    assert attt.attt_device_status() == 0
    okw = {{"ns_steps": "steps"}.get(k, k): v for k, v in kw.items()}
    for i in range(2):
        want, m2 = op.muon_step(ps[i], grads[i], ms[i], lr, **okw)
        got = p[i].double().cpu().numpy()
        size = np.linalg.norm(want - ps[i] * (1 - lr * kw.get("weight_decay", 0.0)))
        assert np.linalg.norm(got - want) <= tol * size + 2.0 ** -22 * np.linalg.norm(ps[i]), i
        assert (np.abs(m[i].double().cpu().numpy() - m2) <= 2.0 ** -22 * (np.abs(ms[i]) + np.abs(grads[i]))).all()
        assert torch.equal(half[i], p[i].to(torch.bfloat16))


# widths that clusters of 16 do not hold in shared memory: 30,976 columns at r 16, 20,608 at 32,
# 6,912 and 9,088 on the two kernels of r 64
STREAMED = [(40000, 35001, 8), (41000, 40004, 16), (30001, 25000, 24), (30000, 29001, 32), (14336, 20001, 33),
            (27648, 18944, 64)]


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("din,dout,r", STREAMED)
def test_columns_that_do_not_stay(din, dout, r, nesterov):
    _check(r, din, dout, r, nesterov=nesterov)


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6, 7])
@pytest.mark.parametrize("din,dout,r", [(500, 601, 3), (500, 601, 32), (700, 9000, 48), (40000, 35001, 8),
                                        (27648, 18944, 64)])
def test_steps(din, dout, r, steps):
    _check(steps, din, dout, r, tol=3e-5 * max(1.0, 3.44 ** (steps - 5)), ns_steps=steps)


@pytest.mark.parametrize("kw", [{"nesterov": False}, {"momentum": 0.0}, {"weight_decay": 0.1}, {"rms": 1.0},
                                {"eps": 1e-2}])
@pytest.mark.parametrize("din,dout,r", [(400, 256, 4), (400, 256, 16), (401, 255, 64), (100001, 90000, 5),
                                        (31008, 100, 12), (300, 14336, 40)])
def test_settings(din, dout, r, kw):
    _check(7, din, dout, r, p_std=0.02, lr=0.05, **kw)


@pytest.mark.parametrize("cond", [1.0, 100.0, 1e4])
@pytest.mark.parametrize("din,dout,r", [(3584, 512, 4), (5120, 1023, 5), (777, 64, 3), (2001, 8, 2), (100001, 90000, 5)])
def test_few_ranks_lose_nothing(din, dout, r, cond):
    _check(r, din, dout, r, cond, tol=2.0 ** -21, momentum=0.0, nesterov=False)


@pytest.mark.parametrize("steps", [1, 2, 4, 7])
def test_steps_of_few_ranks_lose_nothing(steps):
    _check(steps, 3000, 900, 4, 1e3, tol=2.0 ** -21, momentum=0.0, nesterov=False, ns_steps=steps)


def test_wide_and_narrow_matrices_in_one_call():
    """One wide matrix decides the kernel of all: the others' results stay right."""
    r, sizes = 64, [(3584, 3584), (3584, 512), (3584, 18944), (18944, 3584)]
    grads = [_gradients(i, a, b, r, 100.0) for i, (a, b) in enumerate(sizes)]
    d = [[torch.from_numpy(np.ascontiguousarray(v)).to(DEV) for v in pair] for pair in grads]
    p, m = ([[torch.zeros_like(v) for v in pair] for pair in d] for _ in range(2))
    attt.attt_lora_muon_step(*([pair[i] for pair in x] for x in (p, d, m) for i in range(2)), 0.02)
    assert attt.attt_device_status() == 0
    for got, pair in zip(p, grads):
        for x, g in zip(got, pair):
            want, _ = op.muon_step(np.zeros(g.shape), g, np.zeros(g.shape), 0.02)
            assert np.linalg.norm(x.double().cpu().numpy() - want) <= 3e-5 * np.linalg.norm(want)

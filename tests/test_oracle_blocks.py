"""Pins of oracle/blocks.py: torch CPU library routines and autograd in fp64,
closed forms, and the statistics of the random rounding."""
import math

import numpy as np
import pytest
import torch

from oracle import blocks as bl


def _rng(seed):
    return np.random.default_rng(seed)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_multiplication_by_a_complex_number(interleaved):
    r = _rng(0)
    x, pos, w = r.normal(size=(7, 3, 12)), r.integers(-5, 1000, 7), bl.rope_frequencies(8, 100.0)
    y = bl.rotate(x, pos, w, interleaved, 1.5)
    a, b = (slice(0, 8, 2), slice(1, 8, 2)) if interleaved else (slice(0, 4), slice(4, 8))
    z = (x[..., a] + 1j * x[..., b]) * 1.5 * np.exp(1j * pos[:, None] * w)[:, None]
    assert np.allclose(y[..., a], z.real) and np.allclose(y[..., b], z.imag)
    assert np.array_equal(y[..., 8:], x[..., 8:])
    assert np.allclose(bl.rotate(y, pos, w, interleaved, 1 / 1.5, back=True), x)


def test_frequencies():
    assert np.allclose(bl.rope_frequencies(4, 10000.0), [1, 0.01])
    assert np.allclose(bl.rope_frequencies(4, 10000.0, factor=4.0), [0.25, 0.0025])
    w = bl.rope_frequencies(128, 1e4, 8.0, 8192, 1.0, 32.0)
    plain, turns = bl.rope_frequencies(128, 1e4), 8192 * bl.rope_frequencies(128, 1e4) / (2 * math.pi)
    assert np.array_equal(w[turns > 32], plain[turns > 32]) and np.allclose(w[turns < 1], plain[turns < 1] / 8)
    assert (np.diff(w) < 0).all()


@pytest.mark.parametrize("norm", [False, True])
def test_rope_grad_is_autograd(norm):
    r = _rng(1)
    pos, w = r.integers(0, 99, 5), bl.rope_frequencies(6, 100.0)
    x = torch.from_numpy(r.normal(size=(5, 2, 10))).requires_grad_()
    gamma = torch.from_numpy(r.normal(size=10)).requires_grad_()
    dy = r.normal(size=(5, 2, 10))
    z = torch.nn.functional.rms_norm(x, (10,), gamma, 1e-6) if norm else x * 1
    turn = torch.polar(torch.ones(5, 1, 3).double(), torch.from_numpy(pos[:, None, None] * w))
    y = torch.cat([torch.view_as_real(torch.complex(z[..., :3], z[..., 3:6]) * turn).movedim(-1, -2).flatten(-2),
                   z[..., 6:]], -1)
    got = bl.rope(x.detach().numpy(), pos, w, gamma.detach().numpy() if norm else None)
    assert np.allclose(got, y.detach().numpy())
    y.backward(torch.from_numpy(dy))
    dx, dg = bl.rope_grad(dy, x.detach().numpy(), pos, w, gamma.detach().numpy() if norm else None)
    assert np.allclose(dx, x.grad.numpy())
    assert dg is None if not norm else np.allclose(dg, gamma.grad.numpy())


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("adapted", [(0, 1, 2), (1,), ()])
def test_gated_ffn_is_autograd(act, adapted):
    r = _rng(2)
    x, Wg, Wu, Wd = (torch.from_numpy(r.normal(size=s)) for s in ((4, 6), (6, 9), (6, 9), (9, 6)))
    As = [torch.from_numpy(r.normal(size=(s, 2))) if i in adapted else None for i, s in enumerate((6, 6, 9))]
    Bs = [torch.from_numpy(r.normal(size=(2, s))) if i in adapted else None for i, s in enumerate((9, 9, 6))]
    x.requires_grad_()
    merged = [W + 0.5 * A @ B if A is not None else W for W, A, B in zip((Wg, Wu, Wd), As, Bs)]
    g, u = x @ merged[0], x @ merged[1]
    g.retain_grad(), u.retain_grad()
    fn = torch.nn.functional.silu if act == "silu" else lambda t: torch.nn.functional.gelu(t, approximate="tanh")
    y = (fn(g) * u) @ merged[2]
    host = [None if t is None else t.numpy() for t in As], [None if t is None else t.numpy() for t in Bs]
    args = (Wg.numpy(), Wu.numpy(), Wd.numpy())
    got = bl.gated_ffn(x.detach().numpy(), *args, *host, 0.5, act)
    for a, b in zip(got, (y, fn(g) * u, g, u)):
        assert np.allclose(a, b.detach().numpy())
    dy = r.normal(size=(4, 6))
    y.backward(torch.from_numpy(dy))
    dx, dg, du = bl.gated_ffn_grad(dy, *args, g.detach().numpy(), u.detach().numpy(), *host, 0.5, act)
    for a, b in ((dx, x), (dg, g), (du, u)):
        assert np.allclose(a, b.grad.numpy())


def test_adamw_is_torch_adamw():
    r = _rng(3)
    p = torch.from_numpy(r.normal(size=50)).requires_grad_()
    opt = torch.optim.AdamW([p], lr=0.01, betas=(0.9, 0.99), eps=1e-6, weight_decay=0.1)
    q, m, v = p.detach().numpy().copy(), np.zeros(50), np.zeros(50)
    for t in range(1, 5):
        g = r.normal(size=50)
        p.grad = torch.from_numpy(g)
        opt.step()
        q, m, v, _ = bl.adamw(q, g, m, v, 0.01, 0.9, 0.99, 1e-6, 0.1, t)
    assert np.allclose(q, p.detach().numpy(), atol=1e-6)


@pytest.mark.parametrize("mant", [3, 4])
def test_codes(mant):
    v = bl.code_values(mant)
    assert (np.diff(v) > 0).all() and v[0] == 0 and v[-1] == 2 - 2.0 ** -mant
    # every code is its own rounding, whatever the random part
    x = v.astype(np.float32)
    for part in (0, 2.0 ** (23 - mant) - 1):
        for b in range(0, len(x), 200):  # in blocks that hold the largest code
            y = np.concatenate([x[b:b + 200], x[-1:]])
            codes, s = bl.quantise(y, mant, np.full(len(y), part))
            assert np.float32(s[0]) == 1 and np.array_equal(codes[:-1], np.arange(b, b + len(y) - 1))


def test_rounding_keeps_the_mean():
    """Means over 4,000 seeds lie within 6 of their standard deviations, at most half a step
    over sqrt(4000), of the value."""
    x = np.array([1.0, 0.3, 0.031, 1e-3, 4e-5, 1e-5, 1e-6, 0.0], np.float32) * np.float32(1.875)
    got = []
    for seed in range(4000):
        bits = bl.random_bits(len(x), 3, seed)
        codes, s = bl.quantise(x, 3, (bits & np.uint32(0xFFFF)).astype(np.float64) * 16)
        got.append(bl.code_values(3)[codes] * s[0])
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(x / 1.875, 1e-30))), -14) - 3) * 1.875
    assert (np.abs(np.mean(got, 0) - x) <= 6 * 0.5 * step / math.sqrt(4000) + step * 2.0 ** -16).all()


def test_hash_spreads_neighbours():
    """Bits of neighbouring indices, and the two halves that m and v take, are uncorrelated:
    2^16 pairs, 5 standard deviations of 2^-8."""
    n = 1 << 16
    bits = bl.random_bits(n, 0, 7)
    lo, hi = ((bits & np.uint32(0xFFFF)).astype(np.float64), (bits >> np.uint32(16)).astype(np.float64))
    nxt = (bl.random_bits(n, 0, 8) & np.uint32(0xFFFF)).astype(np.float64)
    other = (bl.random_bits(n, 1, 7) & np.uint32(0xFFFF)).astype(np.float64)
    for a, b in ((lo[1:], lo[:-1]), (lo, hi), (lo, nxt), (lo, other), (hi[1:], hi[:-1])):
        assert abs(np.corrcoef(a, b)[0, 1]) < 5 / 256
    for a in (lo, hi):
        assert abs(a.mean() / 65536 - 0.5) < 5 * math.sqrt(1 / 12 / n)

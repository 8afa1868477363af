"""The 8-bit AdamW step of blocks whose gradients span many powers of two, through the oracle.

Gradients of 1 and of +-q, q <= 2^-18, b1 = 0.9, b2 = 0.999, no decay.  A step of a small value, in lr, is
(|m| / (1 - b1^t)) / (sqrt(v) / sqrt(1 - b2^t)) at most, and
  m: rounding adds less than d = 2^-17 max|m| / 1.875 to what is stored (the distance of codes up to 2^-13 of
     the scale), and max|m| = 1 - b1^t is that of the values of size 1.  As if every step rounded up,
     |m| / (1 - b1^t) <= 9 d + q with d = 2^-17 / 1.875, which stays below 2^-13 / 1.875;
  v: a stored sqrt(v) that is not 0 is one code, 2^-18 max sqrt(v) / 1.9375, at least; max sqrt(v) is
     that of a value of size 1, sqrt(1 - b2^(t-1)) but for a code's rounding, 2^-4 of it, and
     sqrt((1 - b2^(t-1)) / (1 - b2^t)) >= 0.7.
So (9 2^-17 / 1.875 + 2^-18) / (0.9995 0.7 (1 - 2^-4) 2^-18 / 1.9375) = 31.3 at most.  Without the rule that a
sqrt(v) above 0 is never stored as 0 the divisor can be sqrt(1 - b2) q instead."""
import numpy as np
import pytest

from oracle import blocks as bl

HYPER = dict(lr=1e-3, b1=0.9, b2=0.999, eps=1e-12, wd=0.0)
BOUND = 31.3


def gradients(n, ratio, steps):
    """Every other value 1, the others of size `ratio` with random signs."""
    r = np.random.default_rng(int(-np.log2(ratio)))
    big = np.arange(n) % 2 == 0
    for _ in range(steps):
        yield np.where(big, 1.0, ratio * r.choice([-1.0, 1.0], n)).astype(np.float32)


@pytest.mark.parametrize("ratio", [2.0 ** -18, 2.0 ** -20, 2.0 ** -24, 2.0 ** -40])
def test_steps_of_small_values_are_bounded(ratio):
    n = 300
    p, m8, v8 = np.zeros(n, np.float32), np.zeros(n, np.uint8), np.zeros(n, np.uint8)
    ms, vs = np.zeros(2, np.float32), np.zeros(2, np.float32)
    worst = 0.0
    for t, g in enumerate(gradients(n, ratio, 300), 1):
        before = p
        p, m8, v8, ms, vs = bl.adamw8(p, g, m8, v8, ms, vs, **HYPER, t=t, seed=t, tensor=0)
        worst = max(worst, np.abs(p - before).max() / HYPER["lr"])
    assert worst <= BOUND


def test_only_zeros_have_the_code_zero():
    n = 512
    g = np.zeros(n, np.float32)
    g[:256] = 2.0 ** -np.linspace(0, 60, 256)  # the second block stays without gradients
    g[100] = 0
    z8, z = np.zeros(n, np.uint8), np.zeros(2, np.float32)
    _, _, v8, _, vs = bl.adamw8(0 * g, g, z8, z8, z, z, **HYPER, t=1, seed=1, tensor=0)
    assert np.array_equal(v8 > 0, g > 0) and vs[1] == 0

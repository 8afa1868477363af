"""Tables of rotation frequencies for stretched contexts: the ramp that is linear in the pair's index
beside the one that is linear in its turns (host-only calls)."""
import math

import numpy as np
import pytest

from oracle import blocks as bl
from paper_2607_03441_gb300 import attt, build

STRETCH = dict(base=1e6, factor=4.0, context=32768, low=1.0, high=32.0)


@pytest.fixture(scope="module", autouse=True)
def _library():
    build.build()


def _radians(rot, **kw):
    return attt.attt_rope_frequencies(rot, **kw).numpy().view(np.uint64).astype(np.float64) * 2.0 ** -64 * 2 * math.pi


@pytest.mark.parametrize("kw", [STRETCH, STRETCH | dict(base=1e4, context=4096, factor=16.0),
                                STRETCH | dict(base=5e5, context=8192, low=1.0, high=4.0), STRETCH | dict(factor=1.0),
                                STRETCH | dict(context=1e9), STRETCH | dict(context=10)])
@pytest.mark.parametrize("rot", [32, 64, 126, 512])
def test_by_index(rot, kw):
    got, want = _radians(rot, **kw, by_index=True), bl.rope_frequencies(rot, **kw, by_index=True)
    # half a step of the table, 2^-63 turns, and fp64 arithmetic: a ramp's share is off by some 2^-50 of 1, which is
    # up to `factor` times as much of a frequency that is divided by it
    assert (np.abs(got - want) <= 2 * math.pi * 2.0 ** -63 + 2.0 ** -48 * kw["factor"] * want).all()


def test_against_values_by_hand():
    """rot 128, base 10^6: 128 ln(32768 / (64 pi)) / (2 ln 10^6) = 23.59 and 128 ln(32768 / (2 pi)) / (2 ln 10^6) =
    39.65, so pairs up to 23 keep their frequency, those from 40 on have a quarter of it, and pair
    23 + k has 1 - 3 k / 68 of it."""
    w = 1e6 ** (-np.arange(64) / 64)
    share = np.concatenate([np.ones(23), 1 - 3 * np.arange(17) / 68, np.full(24, 0.25)])
    assert np.allclose(_radians(128, **STRETCH, by_index=True), w * share, rtol=1e-13, atol=1e-18)


def test_the_two_ramps_differ():
    """Pair 29 turns 32768 10^(-6 29 / 64) / (2 pi) = 9.97 times: by turns it keeps 8.97 / 31 = 0.289 of itself and a quarter of
    the rest, 0.467, by index 1 - 18 / 68 = 0.735; and so on for the pairs of the ramp."""
    a, b = _radians(128, **STRETCH, by_index=True), _radians(128, **STRETCH)
    assert abs(b[29] / a[29] - 0.467 / 0.735) < 2e-3
    off = 1 - b / a
    assert off.min() > -1e-9 and 0.41 < off.max() < 0.43 and (off > 0.01).sum() == 16


@pytest.mark.parametrize("kw", [dict(context=0.0), dict(low=0.0), dict(base=1.0), dict(low=2.0, high=2.0), dict(context=1.0),
                                dict(context=1e30), dict(rot=3), dict(factor=0.5), dict(context=math.nan)])
def test_refusals(kw):
    with pytest.raises(attt.AtttError) as e:
        attt.attt_rope_frequencies(**({"rot": 128} | STRETCH | kw), by_index=True)
    assert e.value.code == attt.ATTT_ERR_INVALID_ARG

"""The gated feed-forward block with adapters on some of its projections, at sizes that the kernels of
few rows take (up to 8 rows, more where a weight has over 2^24 values) and beside them: one product
in the up's half alone, products of one K range alone, none beside those of the other launch.
Bounds: those of test_gpu_gated_ffn."""
import pytest

from paper_2607_03441_gb300 import attt, build
from tests.test_gpu_gated_ffn import Case, check_backward, check_forward

pytestmark = pytest.mark.gpu

ADAPTED = [(0,), (1,), (2,), (0, 1), (0, 2), (1, 2)]


@pytest.fixture(scope="module", autouse=True)
def _library():
    build.build()


def _both(c):
    check_forward(c, attt.attt_gated_ffn_forward(c.x, *c.W, **c.kw, save=True))
    check_backward(c, attt.attt_gated_ffn_backward(c.dy, *c.W, c.g, c.u, **c.kw))
    assert attt.attt_device_status() == 0


@pytest.mark.parametrize("adapted", ADAPTED)
@pytest.mark.parametrize("r", [16, 5, 64])
def test_small_weights(adapted, r):
    for L, d, f in ((1, 192, 456), (5, 192, 456), (8, 1024, 2048)):
        _both(Case(L, d, f, r, adapted=adapted))


@pytest.mark.parametrize("adapted", ADAPTED)
@pytest.mark.parametrize("r", [16, 5])
def test_wide_weights(adapted, r):
    _both(Case(40, 4104, 4104, r, adapted=adapted))
    _both(Case(9, 904, 18952, r, adapted=adapted))

"""The Muon step is as precise as the same steps in fp32, whatever the spectrum: alike
singular values (whose Gram matrices are near multiples of I), and values over a factor
of 10 and of 100.

Bound: 1.5 times what the plain steps in fp32 are off the 64-bit ones, and 1e-6 (some 16
half units of the last place, what a chain of five steps and eleven products is off at
least)."""
import pytest
import torch

from paper_2607_03441_gb300 import attt, build
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _library():
    build.build()


def _plain(u, eps=1e-7):
    """X after five steps, in u's type, on the side of the fewer rows."""
    x = u / (u.square().sum().sqrt() + eps)
    flip = x.shape[0] > x.shape[1]
    x = x.t() if flip else x
    for _ in range(5):
        q = x @ x.t()
        x = 3.4445 * x + (-4.7750 * q + 2.0315 * (q @ q)) @ x
    return x.t() if flip else x


@pytest.mark.parametrize("spread", [1.0, 10.0, 100.0])
@pytest.mark.parametrize("n", [500, 3000, 6001])
@pytest.mark.parametrize("r", [4, 8, 24, 32, 33, 40, 48, 56, 64])
def test_as_fp32(r, n, spread):
    g = torch.Generator(device=DEV).manual_seed(r)
    fall = torch.exp(torch.linspace(0, -1, r, device=DEV) * torch.log(torch.tensor(spread)))
    mix = torch.linalg.qr(torch.randn(r, r, generator=g, device=DEV))[0]
    u = ((torch.randn(n, r, generator=g, device=DEV) * fall) @ mix * 1e-3).contiguous()
    d = [u, u.t().contiguous()]
    p, m = ([torch.zeros_like(v) for v in d] for _ in range(2))
    attt.attt_lora_muon_step(p[:1], p[1:], d[:1], d[1:], m[:1], m[1:], 1.0, momentum=0.0, nesterov=False, rms=1.0)
    assert attt.attt_device_status() == 0
    want = _plain(u.double())
    size = want.norm().item()
    plain = (_plain(u).double() - want).norm().item() / size
    for x in (p[0], p[1].t()):
        off = (-x.double() / n ** 0.5 - want).norm().item() / size
        assert off <= 1.5 * plain + 1e-6, (off, plain)

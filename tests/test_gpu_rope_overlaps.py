"""Results of the heads' norm and rotation beside what is read in one buffer, and those that share
memory, which are refused."""
import pytest
import torch

from paper_2607_03441_gb300 import attt, build
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _library():
    build.build()


@pytest.mark.parametrize("T", [1, 77, 1300])
def test_results_in_one_buffer(T):
    """q where it lies and k where v was; q and k with their heads in turn."""
    hq, hk, D = 6, 2, 64
    g = torch.Generator(device=DEV).manual_seed(T)
    rows = torch.randn(T, (hq + 2 * hk) * D, generator=g, device=DEV).to(torch.bfloat16)
    q, k, v = (rows[:, a * D:b * D].view(T, b - a, D) for a, b in ((0, hq), (hq, hq + hk), (hq + hk, hq + 2 * hk)))
    pos, freq = torch.arange(T, dtype=torch.int32, device=DEV), attt.attt_rope_frequencies(D, device=DEV)
    gammas = [torch.rand(D, generator=g, device=DEV) + 0.5 for _ in range(2)]
    want = attt.attt_rope_forward([q.clone(), k.clone()], pos, freq, gammas)
    before = k.clone()
    got = attt.attt_rope_forward([q, k], pos, freq, gammas, ys=[q, v])
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(k, before)
    xs = [torch.randn(T, hk, D, generator=g, device=DEV) for _ in range(2)]
    turn = torch.zeros(T, hk, 2, D, device=DEV)
    attt.attt_rope_forward(xs, pos, freq, gammas, ys=[turn[:, :, 0], turn[:, :, 1]])
    want = attt.attt_rope_forward(xs, pos, freq, gammas)
    assert torch.equal(turn[:, :, 0], want[0]) and torch.equal(turn[:, :, 1], want[1])
    assert attt.attt_device_status() == 0


def test_shared_results_are_refused():
    T, H, D = 9, 4, 32
    x, other = (torch.randn(T, H, D, device=DEV) for _ in range(2))
    rows = torch.randn(T, 2 * H * D, device=DEV)
    pos, freq = torch.arange(T, dtype=torch.int32, device=DEV), attt.attt_rope_frequencies(D, device=DEV)
    one, w = torch.empty(T, H, D, device=DEV), [torch.ones(D, device=DEV) for _ in range(2)]
    dg = torch.empty(D, device=DEV)
    over = [rows[:, a:a + H * D].view(T, H, D) for a in (0, H * D - 4)]
    n = attt.attt_kernel_launches()
    for call in (lambda: attt.attt_rope_forward([x, other], pos, freq, ys=[one, one]),
                 lambda: attt.attt_rope_forward([x, other], pos, freq, ys=over),
                 lambda: attt.attt_rope_forward([x, other], pos, freq, ys=[other, x]),
                 lambda: attt.attt_rope_forward([x], pos, freq, ys=[x.view(H, T, D).transpose(0, 1)]),
                 lambda: attt.attt_rope_backward([x, other], [x, other], pos, freq, w, dxs=[one, one]),
                 lambda: attt.attt_rope_backward([x, other], [x, other], pos, freq, w, dgammas=[dg, dg])):
        with pytest.raises(attt.AtttError) as e:
            call()
        assert e.value.code == attt.ATTT_ERR_INVALID_ARG
    assert attt.attt_kernel_launches() == n

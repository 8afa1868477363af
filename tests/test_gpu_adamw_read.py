"""attt_adamw_read_state: one array alone, and arrays that share memory, which are refused."""
import pytest
import torch

from paper_2607_03441_gb300 import attt, build
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _library():
    build.build()


@pytest.mark.parametrize("bits", [32, 8])
def test_read_state_arrays(bits):
    p, g = torch.zeros(700, device=DEV), torch.randn(700, device=DEV)
    dtype = torch.float32 if bits == 32 else torch.uint8
    m, v = (torch.zeros(700, dtype=dtype, device=DEV) for _ in range(2))
    scales = [[torch.zeros(3, device=DEV)] for _ in range(2)] if bits == 8 else [None, None]
    opt = attt.attt_adamw_create([p], [g], [m], [v], *scales)
    attt.attt_adamw_step(opt, 0.1, step=1, seed=1)
    m32, v32 = attt.attt_adamw_read_state(opt)
    buf = torch.zeros(2 * 768, device=DEV)
    attt.attt_adamw_read_state(opt, buf[:768], buf[768:])  # side by side
    assert torch.equal(buf[:768], m32) and torch.equal(buf[768:], v32)
    alone = torch.zeros(768, device=DEV)
    assert attt.attt_adamw_read_state(opt, v32=alone)[0] is None and torch.equal(alone, v32)
    n = attt.attt_kernel_launches()
    for a, b in ((alone, alone), (buf[:768], buf[764:1532]), (buf[4:772], buf[:768])):
        with pytest.raises(attt.AtttError) as e:
            attt.attt_adamw_read_state(opt, a, b)
        assert e.value.code == attt.ATTT_ERR_INVALID_ARG
    assert attt.attt_kernel_launches() == n and attt.attt_device_status() == 0

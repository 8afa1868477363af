"""The AdamW step with moments in 8 bits where the gradients of one block span many powers of two:
codes and scales are the oracle's, and a step's size stays bounded (bound: test_oracle_adamw_range)."""
import numpy as np
import pytest
import torch

from oracle import blocks as bl
from paper_2607_03441_gb300 import attt, build
from tests.gpu_util import DEV
from tests.test_oracle_adamw_range import BOUND, HYPER, gradients

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _library():
    build.build()


def _state(n):
    return ([torch.zeros(n, dtype=torch.uint8, device=DEV) for _ in range(2)],
            [torch.zeros(-(-n // 256), device=DEV) for _ in range(2)])


@pytest.mark.parametrize("ratio", [2.0 ** -18, 2.0 ** -20, 2.0 ** -24, 2.0 ** -40])
def test_steps_of_small_values(ratio):
    n, lr = 300, HYPER["lr"]
    p, g = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    (m, v), (ms, vs) = _state(n)
    opt = attt.attt_adamw_create([p], [g], [m], [v], [ms], [vs])
    host = [t.cpu().numpy() for t in (m, v, ms, vs)]
    worst = 0.0
    for t, grad in enumerate(gradients(n, ratio, 150), 1):
        g.copy_(torch.from_numpy(grad))
        before = p.clone()
        attt.attt_adamw_step(opt, lr, (HYPER["b1"], HYPER["b2"]), HYPER["eps"], HYPER["wd"], t, seed=t)
        _, *host = bl.adamw8(before.cpu().numpy(), grad, *host, **HYPER, t=t, seed=t, tensor=0)
        for got, want in zip((m, v, ms, vs), host):
            assert np.array_equal(got.cpu().numpy(), want), t
        worst = max(worst, (p - before).abs().max().item() / lr)
    assert worst <= BOUND
    assert (v > 0).all()  # every value has had a gradient
    assert attt.attt_device_status() == 0

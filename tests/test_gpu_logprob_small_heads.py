"""attt_logprob_input_grad of few rows through heads so small that the contraction
with them takes whole tiles: dz still counts to two bf16."""
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


def _bf16(a):
    return torch.from_numpy(np.asarray(a, dtype=np.float32)).to(DEV).to(torch.bfloat16)


def _shared(seed, L, d, V):
    """Rows that are near three tokens each, none of them the given one as a rule: some
    entries of dz are large, and what they round by does not average out.  Logits are
    exact in fp32 (h on a grid of 1/8 up to 4, W of 1/256 up to 1/4)."""
    r = np.random.default_rng(seed)
    W = np.clip(np.round(r.normal(size=(V, d)) * 20), -64, 64) / 256
    tgt = r.integers(0, V, L).astype(np.int32)
    h = np.zeros((L, d))
    for j in range(L):
        a, b, c = r.integers(0, V, 3)
        h[j] = np.clip(np.round((W[a] + 0.9 * W[b] + 0.85 * W[c]) * 2560 / np.sqrt(d)), -32, 32) / 8
    return h, W, tgt


@pytest.mark.parametrize("L,d,V", [(1, 64, 1000), (2, 64, 1984), (4, 136, 1000), (3, 520, 1984), (17, 136, 1000),
                                   (64, 72, 1000), (33, 3592, 200), (64, 64, 2048), (65, 136, 1000)])
@pytest.mark.parametrize("inv_temp", [1.0, 1.25])
def test_few_rows_keep_their_block(L, d, V, inv_temp):
    """Up to 64 rows take dz in two bf16 (2^-16 of each value), more in one (2^-8 of it);
    dh beside that is off by its own rounding (2^-8 of it) and by fp32 arithmetic: 1e-5 of
    dz's terms, 2^-13 of the sums', and 2^-20 where the given token's parts cancel."""
    h, W, tgt = _shared(L + V, L, d, V)
    r = np.random.default_rng(L)
    a, b = r.normal(size=L).astype(np.float32), (0.3 * r.normal(size=L)).astype(np.float32)
    args = _bf16(h), _bf16(W), torch.from_numpy(tgt).to(DEV)
    f = attt.attt_logprob_forward(*args, inv_temp=inv_temp)
    dh = attt.attt_logprob_input_grad(*args, f[2], torch.from_numpy(a).to(DEV), f[1], torch.from_numpy(b).to(DEV),
                                      inv_temp)
    assert attt.attt_device_status() == 0
    want, dz = op.logprobs_grad(h, W, tgt, a, b, inv_temp)
    p = np.exp(h @ W.T * inv_temp - op.logprobs(h, W, None, 0, inv_temp)[2][:, None])
    terms = p * (np.abs(a) + np.abs(b) * 10)[:, None] * inv_temp
    kept = 2.0 ** -16 if L <= 64 else 2.0 ** -8
    slack = ((kept + 2.0 ** -13) * np.abs(dz) + 1e-5 * terms) @ np.abs(W) + 2.0 ** -20 * np.abs(a)[:, None]
    err = np.abs(dh.float().cpu().numpy() - want)
    assert (err <= 2.0 ** -8 * (np.abs(want) + slack) + slack + 1e-7).all()

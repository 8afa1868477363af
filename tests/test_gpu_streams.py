"""Tensors that the binding allocates for a call on another stream: a workspace or a
result whose kernels are still to run must not share memory with what the caller's
stream frees before the call or allocates after it.

The library's calls are replaced by ones that note the workspace's address and launch
nothing, so that only the binding's allocations are looked at."""
import ctypes

import pytest
import torch

from paper_2607_03441_gb300 import attt, build
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu


class _Notes:
    """The library, but for its calls on a workspace: (address, bytes) of each."""

    def __init__(self, lib):
        self.lib, self.seen = lib, []

    def __getattr__(self, name):
        fn = getattr(self.lib, name)
        if ctypes.c_size_t not in (fn.argtypes or []):
            return fn
        at = list(fn.argtypes).index(ctypes.c_size_t)

        def call(*args):
            self.seen.append((args[at - 1], args[at]))
            return 0
        return call


def _bf16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16, device=DEV)


def _f32(*shape):
    return torch.zeros(shape, device=DEV)


L, D, V, R = 700, 512, 6000, 16
CALLS = {
    "logprob_forward": lambda s: attt.attt_logprob_forward(_bf16(L, D), _bf16(V, D), topk=8, stream=s),
    "logprob_input_grad": lambda s: attt.attt_logprob_input_grad(
        _bf16(L, D), _bf16(V, D), torch.zeros(L, dtype=torch.int32, device=DEV), _f32(L), _f32(L), stream=s),
    "layer_norm_backward": lambda s: attt.attt_layer_norm_backward(
        _bf16(L, D), _bf16(L, D), _f32(D), _f32(L), _f32(L), stream=s),
    "lora_muon_step": lambda s: attt.attt_lora_muon_step(
        *([_f32(D, R)], [_f32(R, D)]) * 3, 0.02, stream=s),
    "weighted_ce_fwd_bwd": lambda s: attt.attt_weighted_ce_fwd_bwd(
        _bf16(L, D), _bf16(V, D), torch.zeros(L, dtype=torch.int32, device=DEV), _f32(L), stream=s),
    "lora_grad": lambda s: attt.attt_lora_grad(_bf16(L, D), [_bf16(L, D)], [_bf16(D, R)], [_bf16(R, D)], 1.0, stream=s),
    "lora_forward": lambda s: attt.attt_lora_forward(_bf16(L, D), _bf16(D, D), _bf16(D, R), _bf16(R, D), 1.0, stream=s),
    "lora_input_grad": lambda s: attt.attt_lora_input_grad(_bf16(L, D), _bf16(D, D), _bf16(D, R), _bf16(R, D), 1.0,
                                                           stream=s),
    "kl_drift": lambda s: attt.attt_kl_drift(_bf16(L, D), _bf16(L, D), _bf16(V, D), stream=s),
}


@pytest.mark.parametrize("name", CALLS)
def test_memory_of_a_call_on_another_stream(name, monkeypatch):
    build.build()
    notes = _Notes(attt.load_library())
    monkeypatch.setattr(attt, "_lib", notes)
    side = torch.cuda.Stream()
    CALLS[name](None)  # how much the call takes
    _, size = notes.seen[-1]
    assert size > 0
    torch.cuda.synchronize()
    before = torch.empty(size, dtype=torch.uint8, device=DEV)
    freed = before.data_ptr()
    del before
    CALLS[name](side)
    taken, size = notes.seen[-1]
    assert taken + size <= freed or freed + size <= taken  # the caller's stream may still use what it freed
    after = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(3)]
    for t in after:  # the call may still use its workspace
        assert taken + size <= t.data_ptr() or t.data_ptr() + size <= taken


def test_results_of_calls_on_another_stream_and_their_values():
    """A call behind a long wait on its stream, while the caller's stream goes on."""
    build.build()
    g = torch.Generator(device=DEV).manual_seed(1)
    h = torch.randn(300, 256, generator=g, device=DEV).to(torch.bfloat16)
    W = (torch.randn(4000, 256, generator=g, device=DEV) * 0.05).to(torch.bfloat16)
    tgt = torch.randint(0, 4000, (300,), generator=g, device=DEV, dtype=torch.int32)
    want = attt.attt_logprob_forward(h, W, tgt, topk=5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    got = attt.attt_logprob_forward(h, W, tgt, topk=5, stream=side)
    for n in (1 << 16, 1 << 20, 1 << 22, 1 << 24):
        torch.full((n,), float("nan"), device=DEV)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(want, got):
        assert torch.equal(a, b)

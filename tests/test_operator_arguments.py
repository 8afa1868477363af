"""What the C entry points of log probabilities, layer norm and the Muon step refuse
before they touch the device: called with made-up addresses, so that nothing but the
refusal may come of it."""
import ctypes

import pytest

from paper_2607_03441_gb300 import attt, build

P = 1 << 20  # an address that every type may have


@pytest.fixture(scope="module")
def lib():
    build.build()
    return attt.load_library()


SIZES_REFUSED = [(0, 64, 100), (4, 0, 100), (4, 64, 0), (4, 4, 100), (4, 63, 100), (4, 100, 100),
                 ((1 << 30) + 1, 64, 100), (4, 64, (1 << 30) + 1), (4, (1 << 20) + 8, 100), (1 << 62, 1 << 20, 1 << 30),
                 (-1, 64, 100)]


@pytest.mark.parametrize("L,d,V", SIZES_REFUSED)
def test_no_workspace_for_sizes_that_are_refused(lib, L, d, V):
    assert lib.attt_logprob_workspace_bytes(L, d, V, 0) == 0
    assert lib.attt_logprob_grad_workspace_bytes(L, d, V) == 0


@pytest.mark.parametrize("topk,V", [(-1, 100), (21, 100), (5, 4)])
def test_no_workspace_for_alternatives_that_are_refused(lib, topk, V):
    assert lib.attt_logprob_workspace_bytes(4, 64, V, topk) == 0


def test_workspaces_of_sizes_that_are_taken(lib):
    for L, d, V, topk in ((1, 8, 1, 1), (4096, 5120, 152064, 20), (1 << 30, 8, 1, 0), (1, 1 << 20, 1 << 30, 0)):
        assert lib.attt_logprob_workspace_bytes(L, d, V, topk) > 0
        assert lib.attt_logprob_grad_workspace_bytes(L, d, V) > 0
    assert lib.attt_layer_norm_workspace_bytes(0, 1) > 0 and lib.attt_layer_norm_workspace_bytes(9, 1 << 24) > 0


@pytest.mark.parametrize("L,d", [(-1, 8), (8, 0), (8, (1 << 24) + 1), (1 << 31, 8), (1 << 62, 1 << 62)])
def test_no_workspace_for_norms_that_are_refused(lib, L, d):
    assert lib.attt_layer_norm_workspace_bytes(L, d) == 0

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


def _forward(lib, **kw):
    a = dict(h=P, W=P, tgt=P, logp=P, entropy=P, lse=P, top_logp=P, top_id=P) | kw
    return lib.attt_logprob_forward(a["h"], 64, a["W"], a["tgt"], 4, 64, 100, 1.0, 3, a["logp"], a["entropy"], a["lse"],
                                    a["top_logp"], a["top_id"], P, 1 << 40, None)


def _input_grad(lib, **kw):
    a = dict(h=P, W=P, tgt=P, lse=P, entropy=P, glogp=P, gent=P, dh=P) | kw
    return lib.attt_logprob_input_grad(a["h"], 64, a["W"], a["tgt"], a["lse"], a["entropy"], a["glogp"], a["gent"], 4,
                                       64, 100, 1.0, a["dh"], P, 1 << 40, None)


def _norm(lib, dtype, **kw):
    a = dict(x=P, gamma=P, beta=P, y=P, mean=P, rstd=P) | kw
    return lib.attt_layer_norm_forward(a["x"], 64, a["gamma"], a["beta"], 4, 64, 1e-5, dtype, a["y"], 64, a["mean"],
                                       a["rstd"], None)


def _norm_grad(lib, dtype, **kw):
    a = dict(dy=P, x=P, gamma=P, mean=P, rstd=P, dx=P, dgamma=P, dbeta=P) | kw
    return lib.attt_layer_norm_backward(a["dy"], 64, a["x"], 64, a["gamma"], a["mean"], a["rstd"], 4, 64, dtype,
                                        a["dx"], 64, a["dgamma"], a["dbeta"], P, 1 << 40, None)


MUON = ("A32", "B32", "dA", "dB", "mA", "mB", "A16", "B16")


def _muon(lib, **kw):
    """A step of two projections; kw: the second one's address of an array."""
    arrays = {k: (ctypes.c_void_p * 2)(P + (i << 12), kw.get(k, P + (i << 12) + 1024)) for i, k in enumerate(MUON)}
    sizes = (ctypes.c_int64 * 2)(16, 16)
    at = {k: ctypes.addressof(v) for k, v in arrays.items()}
    return lib.attt_lora_muon_step(2, at["A32"], at["B32"], at["dA"], at["dB"], at["mA"], at["mB"],
                                   ctypes.addressof(sizes), ctypes.addressof(sizes), 8, 0.02, 0.95, 1, 0.0, 0.2, 1e-7,
                                   5, at["A16"], at["B16"], P << 4, 1 << 40, None)


@pytest.mark.parametrize("name", ["tgt", "logp", "entropy", "lse", "top_logp", "top_id"])
@pytest.mark.parametrize("off", [1, 2])
def test_logprob_forward_refuses_addresses_its_types_do_not_have(lib, name, off):
    assert _forward(lib, **{name: P + off}) == attt.ATTT_ERR_INVALID_ARG


@pytest.mark.parametrize("name", ["tgt", "lse", "entropy", "glogp", "gent"])
@pytest.mark.parametrize("off", [1, 2])
def test_logprob_input_grad_refuses_addresses_its_types_do_not_have(lib, name, off):
    assert _input_grad(lib, **{name: P + off}) == attt.ATTT_ERR_INVALID_ARG


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("off", [1, 2])
def test_layer_norm_refuses_addresses_its_types_do_not_have(lib, dtype, off):
    for name in ("gamma", "beta", "mean", "rstd"):
        assert _norm(lib, dtype, **{name: P + off}) == attt.ATTT_ERR_INVALID_ARG, name
    for name in ("gamma", "mean", "rstd", "dgamma", "dbeta"):
        assert _norm_grad(lib, dtype, **{name: P + off}) == attt.ATTT_ERR_INVALID_ARG, name
    if off % (4 if dtype else 2):
        for name in ("x", "y"):
            assert _norm(lib, dtype, **{name: P + off}) == attt.ATTT_ERR_INVALID_ARG, name
        for name in ("x", "dy", "dx"):
            assert _norm_grad(lib, dtype, **{name: P + off}) == attt.ATTT_ERR_INVALID_ARG, name


@pytest.mark.parametrize("name", MUON)
@pytest.mark.parametrize("off", [1, 2])
def test_muon_refuses_addresses_its_types_do_not_have(lib, name, off):
    if name.endswith("16") and off == 2:
        return  # a bf16 may lie there
    assert _muon(lib, **{name: P + (9 << 12) + off}) == attt.ATTT_ERR_INVALID_ARG


@pytest.mark.parametrize("name,other", [("A32", "A32"), ("B32", "A32"), ("mA", "mA"), ("mB", "A32"), ("dA", "A32"),
                                        ("dB", "mB"), ("A16", "A16"), ("B16", "A16"), ("A16", "B32")])
def test_muon_refuses_matrices_that_are_alike(lib, name, other):
    """What is written belongs to one matrix alone: the step's clusters run at once."""
    assert _muon(lib, **{name: P + (MUON.index(other) << 12)}) == attt.ATTT_ERR_INVALID_ARG

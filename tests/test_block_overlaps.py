"""Results of the block's calls that share memory with one another or with what is still to be read are
refused, others are not.  Made-up addresses: a call that is taken ends at the missing
device, so this file is for machines without one."""
import ctypes

import pytest
import torch

from paper_2607_03441_gb300 import attt, build

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="addresses that no device may see")
BAD = attt.ATTT_ERR_INVALID_ARG


@pytest.fixture(scope="module")
def lib():
    build.build()
    return attt.load_library()


L, D, F, R = 4, 64, 128, 8
NAMES = ("x", "Wg", "Wu", "Wd", "y", "h", "g", "u", "dx", "dg", "du", "ws", "A0", "A1", "A2", "B0", "B1", "B2")
AT = {n: (k + 1) << 32 for k, n in enumerate(NAMES)}  # (dy is "x": the calls' first argument)


def _ffn(lib, back, **kw):
    t = AT | kw
    a, b = ((ctypes.c_void_p * 3)(*(t[f"{n}{i}"] for i in range(3))) for n in "AB")
    pa, pb = ctypes.addressof(a), ctypes.addressof(b)
    if back:
        return lib.attt_gated_ffn_backward(t["x"], t["Wg"], t["Wu"], t["Wd"], pa, pb, t["g"], t["u"], L, D, F, R, 1.0, 0,
                                           t["dx"], t["dg"], t["du"], t["ws"], 1 << 31, None)
    return lib.attt_gated_ffn_forward(t["x"], t["Wg"], t["Wu"], t["Wd"], pa, pb, L, D, F, R, 1.0, 0, t["y"], t["h"],
                                      t["g"], t["u"], t["ws"], 1 << 31, None)


READ = ("Wg", "Wu", "Wd", "A0", "A1", "A2", "B0", "B1", "B2")


@pytest.mark.parametrize("back,results", [(False, ("y", "h", "g", "u", "ws")), (True, ("dx", "dg", "du", "ws"))])
def test_ffn_results_apart(lib, back, results):
    assert _ffn(lib, back) not in (BAD, attt.ATTT_OK)  # taken, but for the device
    for i, a in enumerate(results):
        for b in results[:i] + READ:
            assert _ffn(lib, back, **{a: AT[b]}) == BAD, (a, b)
    size = {"h": 2 * L * F, "dg": 2 * L * F}
    for a, b in (("h", "g"), ("h", "u"), ("h", "x")) if not back else (("dg", "du"), ("dg", "u"), ("dg", "x")):
        for step in (-size[a] + 16, -16, 16):
            assert _ffn(lib, back, **{a: AT[b] + step}) == BAD, (a, b, step)
        assert _ffn(lib, back, **{a: AT[b] - size[a]}) != BAD


def test_ffn_results_that_may_lie_in_what_was_read(lib):
    assert _ffn(lib, False, y=AT["x"]) != BAD and _ffn(lib, False, y=AT["x"] + 16) != BAD
    assert _ffn(lib, True, dx=AT["x"]) != BAD and _ffn(lib, True, dx=AT["g"] + 32) != BAD and _ffn(lib, True, dx=AT["u"]) != BAD
    assert _ffn(lib, True, dg=AT["g"], du=AT["u"]) != BAD and _ffn(lib, True, dg=AT["g"]) != BAD
    for kw in (dict(dg=AT["u"], du=AT["g"]), dict(dg=AT["g"] + 16), dict(du=AT["g"]), dict(du=AT["u"] - 16),
               dict(dg=AT["g"], dx=AT["g"])):
        assert _ffn(lib, True, **kw) == BAD, kw
    for kw in (dict(h=AT["x"]), dict(g=AT["x"]), dict(ws=AT["x"])):
        assert _ffn(lib, False, **kw) == BAD, kw
    for kw in (dict(dg=AT["x"]), dict(du=AT["x"]), dict(ws=AT["g"]), dict(ws=AT["x"])):
        assert _ffn(lib, True, **kw) == BAD, kw
    # the workspace counts with what it needs, not with what it was given
    need = lib.attt_gated_ffn_workspace_bytes(L, D, F, R)
    assert _ffn(lib, False, h=AT["ws"] + need) != BAD and _ffn(lib, False, h=AT["ws"] + need - 16) == BAD

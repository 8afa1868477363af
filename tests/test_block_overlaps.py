"""Results of the block's calls that share memory with one another or with what is still to be read are
refused, others are not.  Made-up addresses: a call that is taken ends at the missing
device, so this file is for machines without one."""
import ctypes

import numpy as np
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


# --------------------------------------------------------------------------

ES = 4  # bytes of a value: fp32
BASE = 1 << 32


def _rope(lib, T, D, parts, back=False):
    """Code of a call whose parts are dicts of y, x, dy = (address, ld, hs in values), heads, dgamma; a missing
    one lies far from all."""
    recs, far = (attt.RopePart * 2)(), 1 << 44
    for i, p in enumerate(parts):
        r = recs[i]
        r.heads = p["heads"]
        for k in ("x", "y", "dy"):
            at, ld, hs = p.get(k, (far, p["heads"] * D, D))
            far += 1 << 40
            setattr(r, k, at), setattr(r, f"{k}_ld", ld), setattr(r, f"{k}_hs", hs)
        r.gamma = 1 << 20
        r.dgamma = p.get("dgamma", (1 << 21) + (i << 16)) if back else None
    at = ctypes.addressof(recs)
    if back:
        return lib.attt_rope_backward(at, len(parts), 1 << 20, 1 << 20, T, D, D, 1e-6, 0, 1.0, 1, 1 << 30, 1 << 30, None)
    return lib.attt_rope_forward(at, len(parts), 1 << 20, 1 << 20, T, D, D, 1e-6, 0, 1.0, 1, None)


def _bytes(T, heads, D, at, ld, hs):
    v = at + ES * (np.arange(T)[:, None, None] * ld + np.arange(heads)[:, None] * hs + np.arange(D))
    return set(v.ravel().tolist())


def test_rope_results_apart(lib):
    """Two random layouts, of two results or of a result and the other part's or its own operand:
    refused where their values, as sets of addresses, meet."""
    r = np.random.default_rng(0)
    seen = [0, 0]
    for k in range(6000):
        T, D = int(r.integers(1, 7)), 2 * int(r.integers(1, 4))
        # one pitch of tokens or of heads for both, or one each
        common = [int(v) for v in r.integers(1, 60, 2)]
        a, b = {}, {}
        for side in (a, b):
            side["heads"] = h = int(r.integers(1, 6))
            hs = D + int(r.integers(0, 3)) * int(r.integers(0, D + 1))
            ld = max(common[0], (h - 1) * hs + D) if r.random() < 0.5 else (h - 1) * hs + D + int(r.integers(0, 8))
            if r.random() < 0.4:  # tokens within heads
                ld = hs
                hs = max(common[1], (T - 1) * ld + D) if r.random() < 0.5 else (T - 1) * ld + D + int(r.integers(0, 8))
            side["y"] = (BASE + ES * int(r.integers(0, 100)), ld, hs)
        if r.random() < 0.5:  # equal strides, as in one buffer
            b["y"] = (b["y"][0],) + a["y"][1:]
            b["heads"] = min(a["heads"], b["heads"])
        pa, pb = a["y"], b["y"]
        meet = bool(_bytes(T, a["heads"], D, *pa) & _bytes(T, b["heads"], D, *pb))
        form = k % 4
        if form == 0:
            code = _rope(lib, T, D, [a, b], back=bool(k & 4))
        elif form == 1:  # a result in what the other part reads
            code = _rope(lib, T, D, [{"heads": a["heads"], "y": pa}, {"heads": b["heads"], "x": pb}], back=bool(k & 4))
        elif form == 2:
            code = _rope(lib, T, D, [{"heads": a["heads"], "x": pa}, {"heads": b["heads"], "y": pb}])
        else:  # a result in its own operand, at other strides or another place (the same: taken)
            heads = min(a["heads"], b["heads"])
            meet = bool(_bytes(T, heads, D, *pa) & _bytes(T, heads, D, *pb))
            strides = [tuple(0 if n == 1 else s for n, s in zip((T, heads), p[1:])) for p in (pa, pb)]
            meet = meet and not (pa[0] == pb[0] and strides[0] == strides[1])
            code = _rope(lib, T, D, [{"heads": heads, "y": pa, "dy" if k & 4 else "x": pb}], back=bool(k & 4))
        assert (code == BAD) == meet, (k, T, D, a, b, code)
        seen[meet] += 1
    assert min(seen) > 500


def test_rope_layouts_of_models(lib):
    T, D, hq, hk = 8192, 128, 40, 8
    row = (hq + 2 * hk) * D
    q, k, v = BASE, BASE + ES * hq * D, BASE + ES * (hq + hk) * D
    one = [{"heads": hq, "y": (q, row, D), "x": (q, row, D)}, {"heads": hk, "y": (k, row, D), "x": (k, row, D)}]
    assert _rope(lib, T, D, one) != BAD  # in place, in one projection's rows
    one[1]["y"] = one[1]["x"] = (k - ES * 8, row, D)
    assert _rope(lib, T, D, one) == BAD
    one[1]["y"], one[1]["x"] = (v, row, D), (k, row, D)
    assert _rope(lib, T, D, one) != BAD  # k's result where v was
    one[1]["y"] = (q, row, D)
    assert _rope(lib, T, D, one) == BAD
    # heads' tokens together, q's and k's heads in turn; and the heads of a token in turn
    for ld, hs, gap in ((D, 2 * T * D, T * D), (2 * D, 2 * T * D, D), (2 * hk * D, 2 * D, D)):
        pair = [{"heads": hk, "y": (BASE + ES * g, ld, hs)} for g in (0, gap)]
        assert _rope(lib, T, D, pair) != BAD
        pair[1]["y"] = (BASE + ES * (gap + 2), ld, hs)
        assert _rope(lib, T, D, pair) == BAD
    # the same result, or the same gradient of the weight, twice
    twice = [{"heads": 4, "y": (BASE, 4 * D, D)} for _ in range(2)]
    assert _rope(lib, T, D, twice) == BAD and _rope(lib, T, D, twice, back=True) == BAD
    for dg, bad in ((1 << 21, True), ((1 << 21) + 4 * D - 4, True), ((1 << 21) + 4 * D, False)):
        parts = [{"heads": 4}, {"heads": 4, "dgamma": dg}]
        assert (_rope(lib, 4, D, parts, back=True) == BAD) == bad
    # operands whose heads lie on one another: one row for all heads, for all tokens
    assert _rope(lib, T, D, [{"heads": 4, "y": (BASE, 4 * D, D), "x": (BASE, 4 * D, 0)}]) == BAD
    assert _rope(lib, T, D, [{"heads": 4, "y": (BASE + ES * D, 4 * D, D), "x": (BASE, 0, 0)}]) != BAD
    assert _rope(lib, T, D, [{"heads": 4, "y": (BASE + ES * D, 4 * D, D), "x": (BASE, D // 2, 0)}]) == BAD

"""What the C entry points of the heads' norm and rotation, the gated feed-forward block
and AdamW over many tensors refuse before they touch the device: called with made-up
addresses, so that nothing but the refusal may come of it."""
import ctypes

import numpy as np
import pytest

from oracle import blocks as bl
from paper_2607_03441_gb300 import attt, build

P = 1 << 20  # an address that every type may have
BAD, BIG = attt.ATTT_ERR_INVALID_ARG, attt.ATTT_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    build.build()
    return attt.load_library()


# --------------------------------------------------------------------------

def _rope(lib, back=False, nparts=1, T=4, D=64, rot=64, eps=1e-6, mscale=1.0, dtype=0, pos=P, freq=P, ws=P, ws_bytes=1 << 30,
          **kw):
    parts = (attt.RopePart * 2)()
    for p in parts:
        f = dict(x=P, y=P, dy=P, gamma=P, dgamma=P if back else None, x_ld=256, x_hs=64, y_ld=256, y_hs=64, dy_ld=256,
                 dy_hs=64, heads=4) | kw
        for k, v in f.items():
            setattr(p, k, v)
    at = ctypes.addressof(parts)
    if back:
        return lib.attt_rope_backward(at, nparts, pos, freq, T, D, rot, eps, 0, mscale, dtype, ws, ws_bytes, None)
    return lib.attt_rope_forward(at, nparts, pos, freq, T, D, rot, eps, 0, mscale, dtype, None)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("kw,code", [
    (dict(nparts=0), BAD), (dict(nparts=3), BAD), (dict(T=-1), BAD), (dict(T=(1 << 30) + 1), BIG), (dict(D=0), BAD),
    (dict(D=63, rot=0), BAD), (dict(D=514), BIG), (dict(rot=66), BAD), (dict(rot=3), BAD), (dict(rot=-2), BAD),
    (dict(eps=-1.0), BAD), (dict(eps=float("nan")), BAD), (dict(mscale=float("nan")), BAD), (dict(dtype=2), BAD),
    (dict(pos=None), BAD), (dict(freq=None), BAD), (dict(pos=P + 2), BAD), (dict(freq=P + 4), BAD), (dict(heads=0), BAD),
    (dict(heads=65537), BIG), (dict(x=P + 1), BAD), (dict(y=P + 1), BAD), (dict(y=None), BAD), (dict(x=None), BAD),
    (dict(gamma=P + 2), BAD), (dict(x_ld=-1), BAD), (dict(y_hs=63), BAD), (dict(y_ld=255), BAD), (dict(y_ld=0), BAD),
    (dict(x_ld=(1 << 36) + 1), BIG), (dict(dtype=1, y=P + 2), BAD),
])
def test_rope_refuses(lib, back, kw, code):
    assert _rope(lib, back, **kw) == code


def test_rope_backward_refuses(lib):
    assert _rope(lib, True, dy=None) == BAD and _rope(lib, True, dy=P + 1) == BAD
    assert _rope(lib, True, gamma=None) == BAD  # a dgamma without a norm
    assert _rope(lib, True, dgamma=P + 1) == BAD
    for kw in (dict(ws=None), dict(ws=P + 16), dict(ws_bytes=16)):
        assert _rope(lib, True, **kw) == attt.ATTT_ERR_WORKSPACE


def test_rope_workspace(lib):
    for T, D in ((-1, 64), (4, 0), (4, 63), (4, 514), ((1 << 30) + 1, 64)):
        assert lib.attt_rope_workspace_bytes(T, D) == 0
    assert lib.attt_rope_workspace_bytes(0, 2) > 0 and lib.attt_rope_workspace_bytes(1 << 30, 512) > 0


@pytest.mark.parametrize("kw", [dict(), dict(base=5e5), dict(factor=8.0), dict(factor=4.0, context=8192, low=1.0, high=4.0)])
def test_rope_frequencies(kw):
    for rot in (2, 64, 126, 512):
        got = attt.attt_rope_frequencies(rot, **kw).numpy().view(np.uint64)
        want = bl.rope_frequencies(rot, **kw) / (2 * np.pi)
        # of the table's 2^-63 steps half a one, and 2^-51 of the value from its formula in fp64
        assert (np.abs(got.astype(np.float64) / 2.0 ** 64 - want) <= 2.0 ** -63 + 2.0 ** -51 * want).all()


@pytest.mark.parametrize("kw", [dict(rot=0), dict(rot=3), dict(rot=514), dict(base=0.5), dict(base=float("inf")),
                                dict(factor=0.5), dict(factor=float("nan")), dict(context=-1.0),
                                dict(context=100.0, low=2.0, high=2.0), dict(context=100.0, low=-1.0)])
def test_rope_frequencies_refuse(kw):
    with pytest.raises(attt.AtttError) as e:
        attt.attt_rope_frequencies(**({"rot": 64} | kw))
    assert e.value.code == BAD


# --------------------------------------------------------------------------

def _ffn(lib, back=False, L=4, d=64, f=128, r=8, act=0, ws=P, ws_bytes=1 << 40, A=(P, P, P), B=(P, P, P), arrays=True, **kw):
    a, b = (ctypes.c_void_p * 3)(*A), (ctypes.c_void_p * 3)(*B)
    pa, pb = (ctypes.addressof(a), ctypes.addressof(b)) if arrays else (None, None)
    t = {k: P for k in ("x", "Wg", "Wu", "Wd", "y", "h", "g", "u", "dx", "dg", "du")} | kw
    if back:
        return lib.attt_gated_ffn_backward(t["x"], t["Wg"], t["Wu"], t["Wd"], pa, pb, t["g"], t["u"], L, d, f, r, 1.0, act,
                                           t["dx"], t["dg"], t["du"], ws, ws_bytes, None)
    return lib.attt_gated_ffn_forward(t["x"], t["Wg"], t["Wu"], t["Wd"], pa, pb, L, d, f, r, 1.0, act, t["y"], t["h"],
                                      t["g"], t["u"], ws, ws_bytes, None)


SIZES = [(dict(L=-1), BAD), (dict(d=4), BAD), (dict(d=60), BAD), (dict(f=0), BAD), (dict(f=100), BAD), (dict(r=-1), BAD),
         (dict(r=65), BAD), (dict(L=(1 << 30) + 1), BIG), (dict(d=(1 << 24) + 8), BIG), (dict(f=(1 << 24) + 8), BIG),
         (dict(L=1 << 30, f=1 << 24), BIG)]


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("kw,code", SIZES + [
    (dict(act=2), BAD), (dict(act=-1), BAD), (dict(r=0), BAD), (dict(arrays=False), BAD), (dict(A=(P, None, P)), BAD),
    (dict(B=(P, P, None)), BAD), (dict(A=(P + 8, P, P)), BAD), (dict(ws=None), attt.ATTT_ERR_WORKSPACE),
    (dict(ws=P + 128), attt.ATTT_ERR_WORKSPACE), (dict(ws_bytes=4096), attt.ATTT_ERR_WORKSPACE)])
def test_ffn_refuses(lib, back, kw, code):
    assert _ffn(lib, back, **kw) == code


@pytest.mark.parametrize("back,names", [(False, ("x", "Wg", "Wu", "Wd", "y", "h", "g", "u")),
                                        (True, ("x", "Wg", "Wu", "Wd", "g", "u", "dx", "dg", "du"))])
def test_ffn_refuses_addresses(lib, back, names):
    for name in names:
        assert _ffn(lib, back, **{name: P + 8}) == BAD
        if name != "dx":
            assert _ffn(lib, back, **{name: None}) == BAD


@pytest.mark.parametrize("kw,_", SIZES)
def test_no_workspace_for_sizes_that_are_refused(lib, kw, _):
    s = dict(L=4, d=64, f=128, r=8) | kw
    assert lib.attt_gated_ffn_workspace_bytes(s["L"], s["d"], s["f"], s["r"]) == 0


def test_workspaces_of_sizes_that_are_taken(lib):
    for s in ((0, 8, 8, 0), (1, 8, 8, 1), (8192, 5120, 27648, 64), (1 << 20, 1 << 14, 1 << 16, 7)):
        assert lib.attt_gated_ffn_workspace_bytes(*s) > 0


# --------------------------------------------------------------------------

def _create(lib, count=2, bits=32, n=(100, 300), **kw):
    names = ("p", "g", "m", "v", "ms", "vs", "p16")
    a = {k: [P + 65536 * (2 * i + j) for j in range(2)] for i, k in enumerate(names)}
    if bits == 32:
        a["ms"] = a["vs"] = None
    for k, v in kw.items():
        a[k] = v
    arrays = {k: None if v is None else (ctypes.c_void_p * 2)(*v) for k, v in a.items()}
    at = {k: None if v is None else ctypes.addressof(v) for k, v in arrays.items()}
    sizes = (ctypes.c_int64 * 2)(*n)
    h = ctypes.c_void_p()
    code = lib.attt_adamw_create(count, at["p"], at["g"], at["m"], at["v"], at["ms"], at["vs"], at["p16"],
                                 ctypes.addressof(sizes), bits, ctypes.byref(h))
    assert not h.value
    return code


Q = 1 << 30


@pytest.mark.parametrize("kw,code", [
    (dict(count=0), BAD), (dict(bits=16), BAD), (dict(p=None), BAD), (dict(g=None), BAD), (dict(m=None), BAD),
    (dict(v=None), BAD), (dict(n=(-1, 4)), BAD), (dict(n=((1 << 40) + 1, 4)), BIG), (dict(p=(None, Q)), BAD),
    (dict(p=(Q + 2, P)), BAD), (dict(g=(Q + 1, P)), BAD), (dict(m=(Q + 2, P)), BAD), (dict(p16=(Q + 1, P)), BAD),
    (dict(bits=8, ms=None), BAD), (dict(bits=32, ms=(Q, Q + 4096)), BAD), (dict(bits=8, ms=(Q + 2, P)), BAD),
    (dict(p=(Q, Q)), BAD), (dict(p=(Q, Q + 396)), BAD), (dict(m=(Q, P + (1 << 26)), v=(Q + 396, P + (1 << 27))), BAD),
    (dict(p=(Q, Q + 65536), g=(Q + 396, P)), BAD), (dict(bits=8, ms=(Q, Q + 4)), BAD),
])
def test_adamw_create_refuses(lib, kw, code):
    if kw.get("bits") == 8 and kw.get("ms") == (Q, Q + 4):
        kw = kw | dict(n=(300, 300))  # two blocks each: their scales share a value
    assert _create(lib, **kw) == code


def test_adamw_calls_refuse_a_missing_handle(lib):
    assert lib.attt_adamw_step(None, 0.1, 0.9, 0.999, 1e-8, 0.0, 1, 0, None) == BAD
    assert lib.attt_adamw_read_state(None, P, P, None) == BAD
    assert lib.attt_adamw_state_values(None) == 0 and lib.attt_adamw_destroy(None) == attt.ATTT_OK

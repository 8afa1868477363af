"""attt_lora_muon_step against the fp64 oracle.

The update X of a matrix with p = 0 is read off exactly.  The same steps in fp32
numpy (pairs of steps on one Gram matrix) are 0.4e-6 to 5e-6 off in norm for
singular values over a factor of 1 to 10,000; 3e-5 leaves room for other orders of
the sums.  m is one fused product and sum, p another: 2^-22 of their terms."""
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


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(DEV)


def _state(seed, dins, douts, r, cond=100.0, zero_p=True):
    g = np.random.default_rng(seed)
    fall = np.exp(np.linspace(0, -np.log(cond), r))
    s = {k: [] for k in ("A32s", "B32s", "dAs", "dBs", "mAs", "mBs")}
    for din, dout in zip(dins, douts):
        qa, qb = (np.linalg.qr(g.normal(size=(r, r)))[0] for _ in range(2))
        s["A32s"].append(g.normal(size=(din, r)) * (0 if zero_p else 0.02))
        s["B32s"].append(g.normal(size=(r, dout)) * (0 if zero_p else 0.01))
        s["dAs"].append((g.normal(size=(din, r)) * fall) @ qa * 1e-3)
        s["dBs"].append(qb @ (fall[:, None] * g.normal(size=(r, dout))) * 1e-3)
        s["mAs"].append(s["dAs"][-1] * 3)
        s["mBs"].append(s["dBs"][-1] * 2)
    return {k: [v.astype(np.float32) for v in vs] for k, vs in s.items()}


def _step(s, lr, copies=True, **kw):
    d = {k: [_dev(v) for v in vs] for k, vs in s.items()}
    h = {}
    if copies:
        h = {k: [torch.zeros_like(v, dtype=torch.bfloat16) for v in d[k[0] + "32s"]] for k in ("A16s", "B16s")}
    attt.attt_lora_muon_step(*(d[k] for k in ("A32s", "B32s", "dAs", "dBs", "mAs", "mBs")), lr, **kw, **h)
    assert attt.attt_device_status() == 0
    return d, h


def _check(s, lr, tol=3e-5, **kw):
    d, h = _step(s, lr, **kw)
    names = {"ns_steps": "steps"}
    okw = {names.get(k, k): v for k, v in kw.items()}
    for side in "AB":
        for i, (p, g, m) in enumerate(zip(s[side + "32s"], s["d" + side + "s"], s["m" + side + "s"])):
            want, m2 = op.muon_step(p, g, m, lr, **okw)
            got = d[side + "32s"][i].double().cpu().numpy()
            keep = 1 - lr * kw.get("weight_decay", 0.0)
            size = np.linalg.norm(want - p * keep)
            assert np.linalg.norm(got - want) <= tol * size + 2.0 ** -22 * np.linalg.norm(p), (side, i)
            mt = 2.0 ** -22 * (np.abs(m) + np.abs(g))
            assert (np.abs(d["m" + side + "s"][i].double().cpu().numpy() - m2) <= mt).all()
            assert torch.equal(h[side + "16s"][i], d[side + "32s"][i].to(torch.bfloat16))
            assert torch.equal(d["d" + side + "s"][i], _dev(g))


CASES = [  # dins, douts, r
    ([1], [1], 1), ([8], [5], 3), ([512], [512], 8), ([3584, 3584], [3584, 512], 16), ([1000], [1001], 12),
    ([130, 7, 129], [64, 2049, 8], 24), ([4096], [1023], 32), ([640, 72], [33, 5120], 64), ([300], [9000], 63),
    ([14336, 64], [64, 27648], 64), ([100] * 8, [200] * 8, 40),
    # as many columns as a CTA of the tensor-core form holds, and numbers just about it
    ([4344, 4392, 688, 816, 1152, 72], [3016, 2128, 4256, 1536, 728, 1304], 64), ([432 * 4], [440 * 4], 48),
    ([5184, 5280, 5176], [5272, 5185, 5279], 64),
    # ranks up to 5: one Gram matrix for all steps; columns that shared memory does not hold
    ([2856, 9], [3512, 100], 4), ([7, 130], [1, 2049], 2), ([100000], [90001], 5), ([100001], [3], 4),
]


@pytest.mark.parametrize("dins,douts,r", CASES)
def test_update(dins, douts, r):
    _check(_state(r + dins[0], dins, douts, r), 0.02)


@pytest.mark.parametrize("cond", [1.0, 1e4])
@pytest.mark.parametrize("r", [16, 32, 64])
def test_conditions(cond, r):
    _check(_state(r, [2000], [777], r, cond), 0.02)


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 5, 6, 7])
@pytest.mark.parametrize("r", [16, 64])
def test_number_of_steps(steps, r):
    # every further step may multiply what is off by 3.44 while singular values still grow
    _check(_state(steps, [600], [700], r), 0.02, tol=3e-5 * max(1.0, 3.44 ** (steps - 5)), ns_steps=steps)


@pytest.mark.parametrize("kw", [{"nesterov": False}, {"momentum": 0.0}, {"weight_decay": 0.1}, {"rms": 1.0},
                                {"eps": 1e-2}])
def test_settings(kw):
    _check(_state(7, [400], [256], 32, zero_p=False), 0.05, **kw)


def test_zero_gradient():
    """The dA of a B that is zero: no update, and no NaN."""
    s = _state(8, [500], [300], 16, zero_p=False)
    for k in ("dAs", "mAs"):
        s[k][0][:] = 0
    d, _ = _step(s, 0.02)
    assert np.array_equal(d["A32s"][0].cpu().numpy(), s["A32s"][0])
    assert torch.isfinite(d["B32s"][0]).all() and not np.array_equal(d["B32s"][0].cpu().numpy(), s["B32s"][0])


def test_low_rank_gradient():
    s = _state(9, [500], [2000], 32)
    s["dAs"][0][:, 1:], s["mAs"][0][:, 1:] = 0, 0  # rank 1
    s["dBs"][0][5:], s["mBs"][0][5:] = 0, 0
    _check(s, 0.02)


def test_nan_stays_in_its_matrix():
    s = _state(10, [500, 500], [300, 300], 16)
    s["dAs"][1][3, 3] = np.nan
    d, _ = _step(s, 0.02)
    assert torch.isnan(d["A32s"][1]).all()
    assert all(torch.isfinite(t).all() for t in (d["A32s"][0], *d["B32s"]))


def test_without_copies_and_repeats():
    s = _state(11, [3000, 60], [700, 5000], 64)
    a, h = _step(s, 0.02)
    b, none = _step(s, 0.02, copies=False)
    assert not none
    for k in a:
        for x, y in zip(a[k], b[k]):
            assert torch.equal(x, y)


def test_another_stream_and_a_graph():
    s = _state(12, [900], [1100], 32, zero_p=False)
    want, _ = _step(s, 0.02)
    d = {k: [_dev(v) for v in vs] for k, vs in s.items()}
    order = ("A32s", "B32s", "dAs", "dBs", "mAs", "mBs")
    ws = torch.empty(attt.attt_lora_muon_workspace_bytes([900], [1100], 32), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        attt.attt_lora_muon_step(*(d[k] for k in order), 0.02, workspace=ws)
    graph.replay()
    torch.cuda.synchronize()
    for k in order:
        assert torch.equal(d[k][0], want[k][0])


def test_refusals():
    s = _state(13, [40], [50], 8)
    d = {k: [_dev(v) for v in vs] for k, vs in s.items()}
    order = ("A32s", "B32s", "dAs", "dBs", "mAs", "mBs")

    def call(lr=0.02, change=None, **kw):
        v = dict(d, **(change or {}))
        attt.attt_lora_muon_step(*(v[k] for k in order), lr, **kw)

    launches = attt.attt_kernel_launches()
    for change in ({"dAs": [d["dAs"][0][:39]]}, {"mBs": []}, {"B32s": [d["B32s"][0].double()]},
                   {"dBs": [d["dBs"][0].t().contiguous().t()]}, {"A32s": [d["A32s"][0].cpu()]}):
        with pytest.raises(ValueError):
            call(change=change)
    with pytest.raises(ValueError):
        call(A16s=[torch.zeros(40, 8, device=DEV)])
    for kw in ({"momentum": 1.0}, {"momentum": -0.1}, {"weight_decay": -1.0}, {"rms": 0.0}, {"eps": 0.0},
               {"ns_steps": 0}, {"ns_steps": 17}, {"lr": float("nan")}, {"lr": float("inf")}):
        with pytest.raises(attt.AtttError) as e:
            call(**kw)
        assert e.value.code == attt.ATTT_ERR_INVALID_ARG
    with pytest.raises(attt.AtttError) as e:
        call(workspace=torch.empty(256, dtype=torch.uint8, device=DEV))
    assert e.value.code == attt.ATTT_ERR_WORKSPACE
    big = {k: [torch.zeros((40, 65) if k[0] == "A" or k[1] == "A" else (65, 50), device=DEV)] for k in order}
    with pytest.raises(attt.AtttError):
        call(change=big)  # rank 65
    nine = {k: v * 9 for k, v in d.items()}
    with pytest.raises(attt.AtttError):
        call(change=nine)
    assert attt.attt_kernel_launches() == launches and attt.attt_device_status() == 0

"""attt_rope_forward / attt_rope_backward against the fp64 oracle.

Bounds, u = 2^-24: cosine and sine of an exact angle are off by at most 4 u (rounding of
what is left of the angle, the function's own 2 u); turning adds two roundings: 8 u of the
pair's two sizes.  A head's sum of squares goes through at most 16 additions in a lane and
five between lanes: 32 u of it, 16 u of its root, and 4 u in what follows (22 additions are
11 u of the root, its function 2 ulp = 4 u, two products 2 u: 17 of these 20).  dgamma adds tokens
and heads in at most 400 steps (a lane takes at most one of 32 groups' heads of 40,013 / 200 tokens).  Results rounded to bf16 are off by 2^-8 of themselves."""
import numpy as np
import pytest
import torch

from oracle import blocks as bl
from paper_2607_03441_gb300 import attt, build
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _library():
    build.build()


def _host(t):
    return t.double().cpu().numpy()


def _heads(r, T, H, D, dtype, form):
    """Heads of NaN-padded rows: "rows" (tokens hold heads), "wide" (inside wider rows, off
    their vectors), "swapped" (heads hold tokens)."""
    v = torch.from_numpy((r.normal(size=(T, H, D)) * np.exp(r.normal(size=D))).astype(np.float32)).to(DEV).to(dtype)
    if form == "rows":
        return v
    if form == "swapped":
        return v.transpose(0, 1).contiguous().transpose(0, 1)
    buf = torch.full((T, H * D + 11), float("nan"), dtype=dtype, device=DEV)
    out = buf[:, 3:3 + H * D].view(T, H, D)
    out.copy_(v)
    return out


def _rounding(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else U


def _sizes(x, rot, interleaved):
    """For every value of a pair, the sum of the pair's sizes; of others, their own."""
    a, b = bl._members(rot, interleaved)
    x = np.abs(x).copy()
    s = x[..., a] + x[..., b]
    x[..., a] = x[..., b] = s
    return x


CASES = [  # T, heads, D, rot, interleaved, norm, dtype, form
    (1, (1,), 2, 2, False, True, torch.float32, "rows"), (1, (4, 1), 128, 128, False, True, torch.bfloat16, "rows"),
    (3, (5, 2), 64, 64, True, True, torch.bfloat16, "swapped"), (16, (28, 4), 128, 128, False, True, torch.bfloat16, "wide"),
    (37, (3, 3), 80, 40, True, False, torch.float32, "rows"), (21, (7, 1), 90, 46, False, True, torch.float32, "wide"),
    (19, (2, 2), 256, 64, False, True, torch.bfloat16, "rows"), (5, (3,), 512, 512, False, True, torch.float32, "rows"),
    (5, (3, 2), 512, 256, True, True, torch.bfloat16, "swapped"), (4, (2, 1), 510, 510, False, True, torch.bfloat16, "rows"),
    (9, (2, 1), 96, 0, False, True, torch.float32, "rows"), (700, (9, 3), 32, 32, True, True, torch.float32, "rows"),
    (1300, (8, 2), 128, 128, False, True, torch.bfloat16, "rows"), (1201, (6,), 64, 32, False, False, torch.bfloat16, "wide"),
    (2, (300, 1), 16, 16, False, True, torch.bfloat16, "rows"), (333, (1, 5), 48, 16, True, True, torch.float32, "wide"),
    (640, (2, 2), 258, 4, False, True, torch.float32, "rows"),
    # runs of tokens that a block's table does not hold at once
    (40013, (2, 1), 64, 64, False, True, torch.bfloat16, "rows"), (9001, (1,), 512, 512, True, True, torch.float32, "rows"),
    (30011, (1, 1), 34, 34, False, True, torch.float32, "wide"),
]


def _case(T, heads, D, rot, interleaved, norm, dtype, form):
    r = np.random.default_rng(T + D + rot)
    xs = [_heads(r, T, H, D, dtype, form) for H in heads]
    dys = [_heads(r, T, H, D, dtype, "rows" if form == "swapped" else form) for H in heads]
    gammas = [torch.from_numpy((1 + 0.2 * r.normal(size=D)).astype(np.float32)).to(DEV) if norm else None for _ in heads]
    pos = r.integers(-3, 1 << 20, T).astype(np.int32)
    freq = attt.attt_rope_frequencies(rot, 5e5, device=DEV) if rot else torch.empty(0, dtype=torch.int64, device=DEV)
    return xs, dys, gammas, pos, freq, bl.rope_frequencies(rot, 5e5)


@pytest.mark.parametrize("case", CASES)
def test_forward(case):
    T, heads, D, rot, interleaved, norm, dtype, form = case
    xs, _, gammas, pos, freq, w = _case(*case)
    ys = attt.attt_rope_forward(xs, torch.from_numpy(pos).to(DEV), freq, gammas if norm else None, 1e-6, interleaved, 1.25)
    assert attt.attt_device_status() == 0
    for x, y, g in zip(xs, ys, gammas):
        gh = _host(g) if norm else None
        want = bl.rope(_host(x), pos, w, gh, 1e-6, interleaved, 1.25)
        z = bl.rope(_host(x), pos, w[:0], gh, 1e-6)
        tol = (8 + 16 + 4 + 4) * U * 1.25 * _sizes(z, rot, interleaved) + _rounding(dtype) * np.abs(want) + 1e-38
        assert (np.abs(_host(y) - want) <= tol).all()


@pytest.mark.parametrize("case", CASES)
def test_backward(case):
    T, heads, D, rot, interleaved, norm, dtype, form = case
    xs, dys, gammas, pos, freq, w = _case(*case)
    dxs, dgs = attt.attt_rope_backward(dys, xs if norm else None, torch.from_numpy(pos).to(DEV), freq,
                                       gammas if norm else None, 1e-6, interleaved, 0.75)
    assert attt.attt_device_status() == 0
    for x, dy, dx, g, dg in zip(xs, dys, dxs, gammas, dgs):
        gh = _host(g) if norm else None
        want, wdg = bl.rope_grad(_host(dy), _host(x), pos, w, gh, 1e-6, interleaved, 0.75)
        ddz = 8 * U * 0.75 * _sizes(_host(dy), rot, interleaved)
        tol = ddz
        if norm:
            xh_ = _host(x)
            rstd = 1 / np.sqrt((xh_ * xh_).mean(-1, keepdims=True) + 1e-6)
            xh, dz = xh_ * rstd, np.abs(bl.rotate(_host(dy), pos, w, interleaved, 0.75, back=True))
            gg, dgg = dz * np.abs(gh), ddz * np.abs(gh)
            mean = (gg * np.abs(xh)).mean(-1, keepdims=True)
            dmean = (dgg * np.abs(xh)).mean(-1, keepdims=True) + (32 + 20 + 4) * U * mean
            tol = rstd * (dgg + np.abs(xh) * dmean + (20 + 8) * U * (gg + np.abs(xh) * mean))
            dtol = ((ddz + 24 * U * dz) * np.abs(xh)).sum((0, 1)) + 400 * U * (dz * np.abs(xh)).sum((0, 1))
            assert (np.abs(_host(dg) - wdg) <= dtol + 1e-38).all()
        else:
            assert dg is None
        assert (np.abs(_host(dx) - want) <= tol + _rounding(dtype) * np.abs(want) + 1e-38).all()


def test_far_positions_and_ends_of_the_range():
    """Angles of the largest positions of int32 are exact: the oracle's fp64 products are
    off by 2^-53 of up to 2^31 radians, 2^-22, so this one is formed in integers."""
    pos = np.array([0, 1, -1, (1 << 31) - 1, -(1 << 31), 123456789], np.int32)
    freq = attt.attt_rope_frequencies(64, 1e4)
    x = torch.zeros(len(pos), 1, 64, device=DEV)
    x[..., :32] = 1
    y, = attt.attt_rope_forward([x], torch.from_numpy(pos).to(DEV), freq.to(DEV))
    turns = np.array([[(int(p) * (int(f) % (1 << 64))) % (1 << 64) / 2 ** 64 for f in freq.tolist()] for p in pos])
    assert np.abs(_host(y)[:, 0, :32] - np.cos(2 * np.pi * turns)).max() < 4 * U + 1e-15
    assert np.abs(_host(y)[:, 0, 32:] - np.sin(2 * np.pi * turns)).max() < 4 * U + 1e-15


def test_in_place_and_inside_one_projection():
    """q and k in the rows of one projection, turned where they lie; v beside them stays."""
    r = np.random.default_rng(3)
    T, hq, hk, D = 77, 6, 2, 64
    rows = torch.from_numpy(r.normal(size=(T, (hq + 2 * hk) * D)).astype(np.float32)).to(DEV).to(torch.bfloat16)
    before = rows.clone()
    q, k = rows[:, :hq * D].view(T, hq, D), rows[:, hq * D:(hq + hk) * D].view(T, hk, D)
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    freq = attt.attt_rope_frequencies(D, device=DEV)
    gammas = [torch.rand(D, device=DEV) + 0.5 for _ in range(2)]
    want = attt.attt_rope_forward([q.clone(), k.clone()], pos, freq, gammas)
    got = attt.attt_rope_forward([q, k], pos, freq, gammas, ys=[q, k])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(rows[:, (hq + hk) * D:], before[:, (hq + hk) * D:])
    dys = [torch.randn_like(t) for t in want]
    xs = [before[:, :hq * D].view(T, hq, D), before[:, hq * D:(hq + hk) * D].view(T, hk, D)]
    want, dgs = attt.attt_rope_backward(dys, xs, pos, freq, gammas)
    got, dgs2 = attt.attt_rope_backward(dys, xs, pos, freq, gammas, dxs=dys)
    assert all(torch.equal(a, b) for a, b in zip(list(want) + list(dgs), list(got) + list(dgs2)))


def test_gradient_against_differences():
    r = np.random.default_rng(4)
    T, H, D, rot = 6, 3, 24, 16
    x, dy = (torch.from_numpy(r.normal(size=(T, H, D)).astype(np.float32)).to(DEV) for _ in range(2))
    g = torch.from_numpy((1 + 0.1 * r.normal(size=D)).astype(np.float32)).to(DEV)
    pos = np.arange(T, dtype=np.int32) * 7
    w = bl.rope_frequencies(rot)
    (dx,), (dg,) = attt.attt_rope_backward([dy], [x], torch.from_numpy(pos).to(DEV),
                                           attt.attt_rope_frequencies(rot, device=DEV), [g])
    xh, gh, dyh = _host(x), _host(g), _host(dy)
    for grad, which in ((_host(dx), 0), (_host(dg), 1)):
        v = r.normal(size=grad.shape)
        e = 1e-5
        f = [(dyh * bl.rope(xh + s * e * v * (which == 0), pos, w, gh + (s * e * v if which else 0))).sum() for s in (1, -1)]
        # fp32 gradients of 432 terms of size 1: 1e-5 at most; differences 1e-9 of them
        assert abs((f[0] - f[1]) / (2 * e) - (grad * v).sum()) < 2e-5


def test_one_norm_of_two():
    """Queries normed and keys not, and the other way round: as two calls."""
    r = np.random.default_rng(6)
    T, D = 33, 64
    xs = [_heads(r, T, H, D, torch.bfloat16, "rows") for H in (4, 2)]
    dys = [_heads(r, T, H, D, torch.bfloat16, "rows") for H in (4, 2)]
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    freq, g = attt.attt_rope_frequencies(D, device=DEV), torch.rand(D, device=DEV) + 0.5
    for gammas in ([g, None], [None, g]):
        ys = attt.attt_rope_forward(xs, pos, freq, gammas)
        dxs, dgs = attt.attt_rope_backward(dys, [x if gm is not None else None for x, gm in zip(xs, gammas)], pos, freq, gammas)
        for i in range(2):
            one = [gammas[i]] if gammas[i] is not None else None
            y, = attt.attt_rope_forward([xs[i]], pos, freq, one)
            (dx,), (dg,) = attt.attt_rope_backward([dys[i]], [xs[i]], pos, freq, one)
            assert torch.equal(y, ys[i]) and torch.equal(dx, dxs[i]) and (dg is None) == (dgs[i] is None)
            if dg is not None:  # other blocks, another order of the sum: 33 x 4 terms
                assert (dg - dgs[i]).abs().max() <= 132 * U * dgs[i].abs().max() * 4


def test_zero_and_nan_heads():
    T, H, D = 3, 4, 64
    x = torch.randn(T, H, D, device=DEV).to(torch.bfloat16)
    x[0, 1] = 0
    x[1, 2, 5] = float("nan")
    x[2, 3, 6] = float("inf")
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    freq, g = attt.attt_rope_frequencies(D, device=DEV), torch.ones(D, device=DEV)
    y, = attt.attt_rope_forward([x], pos, freq, [g])
    assert not y[0, 1].any() and torch.isnan(y[1, 2]).all() and torch.isnan(y[2, 3, 6])
    live = torch.ones(T, H, dtype=torch.bool)
    live[1, 2] = live[2, 3] = False
    assert torch.isfinite(y[live.to(DEV)]).all()
    (dx,), _ = attt.attt_rope_backward([torch.ones_like(x)], [x], pos, freq, [g])
    assert torch.isfinite(dx[live.to(DEV)]).all() and torch.isnan(dx[1, 2]).all()


def test_no_tokens_and_frozen_norms():
    x = torch.empty(0, 3, 32, device=DEV)
    pos, freq, g = (torch.empty(0, dtype=torch.int32, device=DEV), attt.attt_rope_frequencies(32, device=DEV),
                    torch.ones(32, device=DEV))
    y, = attt.attt_rope_forward([x], pos, freq, [g])
    (dx,), (dg,) = attt.attt_rope_backward([x], [x], pos, freq, [g])
    assert y.shape == dx.shape == x.shape and not dg.any() and attt.attt_device_status() == 0
    x = torch.randn(9, 3, 32, device=DEV)
    pos = torch.arange(9, dtype=torch.int32, device=DEV)
    n = attt.attt_kernel_launches()
    (dx,), dgs = attt.attt_rope_backward([x], [x], pos, freq, [g], weights=False)
    assert dgs == [None] and attt.attt_kernel_launches() == n + 1
    want, (dg,) = attt.attt_rope_backward([x], [x], pos, freq, [g])
    assert torch.equal(dx, want[0]) and attt.attt_kernel_launches() == n + 3


def test_repeats_streams_and_graphs():
    r = np.random.default_rng(5)
    xs, dys, gammas, pos, freq, _ = _case(1300, (8, 2), 128, 128, False, True, torch.bfloat16, "rows")
    pos = torch.from_numpy(pos).to(DEV)

    def call(stream=None):
        ys = attt.attt_rope_forward(xs, pos, freq, gammas, stream=stream)
        dxs, dgs = attt.attt_rope_backward(dys, xs, pos, freq, gammas, stream=stream)
        return list(ys) + list(dxs) + list(dgs)

    first = call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    second = call(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        third = call()
    for t in third:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for a, b, c in zip(first, second, third):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_refusals():
    x, pos = torch.randn(4, 2, 32, device=DEV), torch.arange(4, dtype=torch.int32, device=DEV)
    freq, g = attt.attt_rope_frequencies(32, device=DEV), torch.ones(32, device=DEV)
    fwd, bwd = attt.attt_rope_forward, attt.attt_rope_backward
    n = attt.attt_kernel_launches()
    for call in (lambda: fwd([x.half()], pos, freq), lambda: fwd([x, x, x], pos, freq), lambda: fwd([], pos, freq),
                 lambda: fwd([x], pos.long(), freq), lambda: fwd([x], pos[:3], freq), lambda: fwd([x], pos, freq.int()),
                 lambda: fwd([x], pos, freq, [g[:31]]), lambda: fwd([x], pos, freq, [g, g]),
                 lambda: fwd([x.transpose(1, 2)], pos, freq), lambda: fwd([x[0]], pos, freq),
                 lambda: fwd([x, x[:3]], pos, freq), lambda: fwd([x], pos, freq, ys=[x.bfloat16()]),
                 lambda: fwd([x.cpu()], pos, freq), lambda: bwd([x], None, pos, freq, [g]),
                 lambda: bwd([x], [x], pos, freq, dgammas=[g]), lambda: bwd([x], [x], pos, freq, [g], dgammas=[g[:4]])):
        with pytest.raises(ValueError):
            call()
    over = torch.zeros(5, 32, device=DEV).as_strided((4, 2, 32), (32, 16, 1))
    for call, code in ((lambda: fwd([x], pos, freq, eps=-1.0), attt.ATTT_ERR_INVALID_ARG),
                       (lambda: fwd([x], pos, freq, mscale=float("inf")), attt.ATTT_ERR_INVALID_ARG),
                       (lambda: fwd([x[..., :30].contiguous()], pos, freq), attt.ATTT_ERR_INVALID_ARG),
                       (lambda: fwd([x], pos, freq, ys=[over]), attt.ATTT_ERR_INVALID_ARG),
                       (lambda: bwd([x], [x], pos, freq, [g], workspace=torch.empty(16, dtype=torch.uint8, device=DEV)),
                        attt.ATTT_ERR_WORKSPACE)):
        with pytest.raises(attt.AtttError) as e:
            call()
        assert e.value.code == code
    assert attt.attt_kernel_launches() == n and attt.attt_device_status() == 0

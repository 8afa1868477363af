"""attt_gated_ffn_forward / attt_gated_ffn_backward against the fp64 oracle.

Bounds.  A contraction over K adds K products of bf16 (exact in fp32) on the tensor cores,
16 at a time: each of the K / 16 additions may cut off 2^-22 of the sum of the products' sizes
(the partial sums of K pieces and of the adapters' K blocks among them).  A rank-r product is
rounded to bf16 once, 2^-8 of itself, and so are results.  The activation's exponential is off by
at most 2 + 1.16 |z| units of 2^-23, z within 40 of zero where its share of the result is not
below 2^-50: 6e-6 of it; act' is at most 1.13, act at most |g|."""
import math

import numpy as np
import pytest
import torch

from oracle import blocks as bl
from paper_2607_03441_gb300 import attt, build
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu
R16, EXP = 2.0 ** -8, 6e-6


@pytest.fixture(scope="module", autouse=True)
def _library():
    build.build()


def _host(t):
    return None if t is None else t.double().cpu().numpy()


def _cut(K):
    return (K / 16 + 20) * 2.0 ** -22


class Case:
    def __init__(self, L, d, f, r, act="silu", adapted=(0, 1, 2), seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed + L + d + f + r)

        def bf(*shape, std):
            return (torch.randn(shape, generator=g, device=DEV) * std).to(torch.bfloat16)

        self.L, self.d, self.f, self.act, self.scale = L, d, f, act, 0.75
        self.x, self.dy = bf(L, d, std=1.0), bf(L, d, std=1.0)
        self.W = bf(d, f, std=d ** -0.5), bf(d, f, std=d ** -0.5), bf(f, d, std=f ** -0.5)
        ins, outs = (d, d, f), (f, f, d)
        self.As = [bf(n, r, std=n ** -0.5) if r and i in adapted else None for i, n in enumerate(ins)]
        self.Bs = [bf(r, n, std=r ** -0.5) if r and i in adapted else None for i, n in enumerate(outs)]
        self.g, self.u = bf(L, f, std=1.5), bf(L, f, std=1.0)
        self.kw = dict(As=self.As, Bs=self.Bs, scale=self.scale, act=act)

    def host(self):
        return [_host(w) for w in self.W], [_host(t) for t in self.As], [_host(t) for t in self.Bs]


def _project_tol(x, dx, W, A, B, s):
    """How far x W + s (x A) B is off when x is off by dx (elementwise, fp32 result)."""
    x, W = np.abs(x), np.abs(W)
    tol = _cut(len(W)) * (x @ W) + dx @ W
    if A is not None:
        A, B = np.abs(A), np.abs(B)
        xa = s * (x @ A)
        tol += (s * (dx @ A) + (R16 + _cut(len(A))) * xa) @ B + _cut(64) * (xa @ B)
    return tol


def _check(got, want, tol, name):
    worst = (np.abs(_host(got) - want) - tol).max()
    assert worst <= 0, (name, worst, np.abs(want).max())


def check_forward(c, out):
    (Wg, Wu, Wd), As, Bs = c.host()
    x = _host(c.x)
    y, h, g, u = bl.gated_ffn(x, Wg, Wu, Wd, As, Bs, c.scale, c.act)
    tg, tu = (_project_tol(x, 0 * x, W, As[i], Bs[i], c.scale) for i, W in ((0, Wg), (1, Wu)))
    if out[2] is not None:
        _check(out[2], g, tg + R16 * np.abs(g), "g")
        _check(out[3], u, tu + R16 * np.abs(u), "u")
    a = bl.activation(g, c.act)[0]
    th = 1.13 * tg * (np.abs(u) + tu) + np.abs(a) * tu + EXP * np.abs(g * u) + R16 * np.abs(h)
    _check(out[1], h, th, "h")
    _check(out[0], y, _project_tol(h, th, Wd, As[2], Bs[2], c.scale) + R16 * np.abs(y), "y")


def _t(M):
    return None if M is None else M.T


def check_backward(c, out):
    (Wg, Wu, Wd), As, Bs = c.host()
    dy, g, u = _host(c.dy), _host(c.g), _host(c.u)
    dx, dg, du = bl.gated_ffn_grad(dy, Wg, Wu, Wd, g, u, As, Bs, c.scale, c.act)
    dh = bl.project(dy, Wd.T, _t(Bs[2]), _t(As[2]), c.scale)
    tdh = _project_tol(dy, 0 * dy, Wd.T, _t(Bs[2]), _t(As[2]), c.scale)
    a, slope = bl.activation(g, c.act)
    tg = tdh * np.abs(u * slope) + EXP * np.abs(dh * u) * (1 + np.abs(g)) * (1 + np.abs(g)) + R16 * np.abs(dg)
    tu = tdh * np.abs(a) + EXP * np.abs(dh * g) + R16 * np.abs(du)
    _check(out[1], dg, tg, "dg")
    _check(out[2], du, tu, "du")
    if out[0] is not None:
        tol = sum(_project_tol(v, t, W.T, _t(Bs[i]), _t(As[i]), c.scale)
                  for v, t, W, i in ((dg, tg, Wg, 0), (du, tu, Wu, 1)))
        _check(out[0], dx, tol + R16 * np.abs(dx), "dx")


SHAPES = [  # L, d, f, r
    (1, 8, 8, 0), (1, 8, 8, 1), (1, 64, 64, 64), (2, 72, 200, 3), (7, 128, 1000, 8), (16, 512, 1024, 16),
    (33, 264, 344, 20), (93, 512, 2048, 16), (127, 40, 3000, 12), (128, 1024, 512, 32), (129, 512, 776, 64),
    (255, 136, 136, 4), (257, 520, 1288, 24), (403, 768, 2560, 32), (300, 3584, 64, 16), (40, 64, 6400, 16),
    (700, 320, 5000, 40), (1030, 256, 4104, 0), (2500, 64, 264, 7),
]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
def test_forward(shape, act):
    c = Case(*shape, act=act)
    out = attt.attt_gated_ffn_forward(c.x, *c.W, **c.kw, save=True)
    assert attt.attt_device_status() == 0
    check_forward(c, out)
    lean = attt.attt_gated_ffn_forward(c.x, *c.W, **c.kw)
    assert lean[2] is None and lean[3] is None
    assert torch.equal(lean[0], out[0]) and torch.equal(lean[1], out[1])


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
def test_backward(shape, act):
    c = Case(*shape, act=act)
    out = attt.attt_gated_ffn_backward(c.dy, *c.W, c.g, c.u, **c.kw)
    assert attt.attt_device_status() == 0
    check_backward(c, out)
    lean = attt.attt_gated_ffn_backward(c.dy, *c.W, c.g, c.u, **c.kw, input_grad=False)
    assert lean[0] is None and torch.equal(lean[1], out[1]) and torch.equal(lean[2], out[2])


WIDE = [  # more than 2^24 values of a weight: which kernels take the rows depends on L, r and f's tiles
    (9, 4104, 4104, 16), (17, 2056, 8200, 12), (33, 8200, 2056, 8), (64, 4104, 4104, 16), (65, 4104, 4104, 0),
    (96, 4104, 4104, 16), (97, 4104, 4104, 16), (96, 904, 18952, 15), (8, 904, 18952, 64), (32, 904, 18952, 64),
    (33, 904, 18952, 40), (40, 904, 19592, 0), (64, 904, 19592, 16), (65, 904, 19592, 16), (5, 904, 24584, 64),
    (64, 4104, 4104, 32), (96, 904, 18952, 32), (32, 4104, 4104, 48), (33, 904, 19592, 0),
]


@pytest.mark.parametrize("shape", WIDE)
def test_rows_at_wide_weights(shape):
    c = Case(*shape)
    check_forward(c, attt.attt_gated_ffn_forward(c.x, *c.W, **c.kw, save=True))
    check_backward(c, attt.attt_gated_ffn_backward(c.dy, *c.W, c.g, c.u, **c.kw))
    assert attt.attt_device_status() == 0


@pytest.mark.parametrize("adapted", [(0,), (1,), (2,), (0, 2), (1, 2), (0, 1)])
@pytest.mark.parametrize("r", [16, 5])
def test_some_projections_adapted(adapted, r):
    for L in (9, 300):
        c = Case(L, 192, 456, r, adapted=adapted)
        check_forward(c, attt.attt_gated_ffn_forward(c.x, *c.W, **c.kw, save=True))
        check_backward(c, attt.attt_gated_ffn_backward(c.dy, *c.W, c.g, c.u, **c.kw))
    assert attt.attt_device_status() == 0


@pytest.mark.parametrize("shape", [(1, 3584, 18944, 16), (512, 2048, 8192, 32), (2048, 1024, 4096, 16),
                                   (4352, 512, 2304, 64)])
def test_large(shape):
    c = Case(*shape)
    check_forward(c, attt.attt_gated_ffn_forward(c.x, *c.W, **c.kw, save=True))
    check_backward(c, attt.attt_gated_ffn_backward(c.dy, *c.W, c.g, c.u, **c.kw))
    assert attt.attt_device_status() == 0


def test_many_rows():
    """20,000 rows, more row tiles than the device holds clusters: rows' results do not depend on the others."""
    c = Case(20000, 64, 128, 8)
    out = attt.attt_gated_ffn_forward(c.x, *c.W, **c.kw, save=True)
    back = attt.attt_gated_ffn_backward(c.dy, *c.W, out[2], out[3], **c.kw)
    check_forward(c, out)
    c.g, c.u = out[2], out[3]
    check_backward(c, back)
    assert attt.attt_device_status() == 0


def test_saturated_gates():
    """Gates far from zero: act is 0 or g, act' 0 or 1, and neither is a NaN."""
    L, d, f = 5, 64, 128
    c = Case(L, d, f, 0)
    for act in ("silu", "gelu_tanh"):
        c.act = act
        c.kw["act"] = act
        for big in (50.0, 1e4, 3e38):
            c.g = torch.where(torch.rand(L, f, device=DEV) < 0.5, big, -big).to(torch.bfloat16)
            dx, dg, du = attt.attt_gated_ffn_backward(c.dy, *c.W, c.g, c.u, **c.kw, input_grad=False)
            dh = _host(c.dy) @ _host(c.W[2]).T
            on = _host(c.g) > 0
            assert torch.isfinite(dg).all()
            assert (du[torch.from_numpy(~on).to(DEV)].abs() < 1e-15).all()
            want = np.where(on, dh * _host(c.u), 0)
            tol = _cut(d) * (np.abs(_host(c.dy)) @ np.abs(_host(c.W[2]).T)) * np.abs(_host(c.u)) + R16 * np.abs(want)
            assert (np.abs(_host(dg) - want) <= tol + 1e-15).all()


def test_gradient_against_differences():
    """Along a random direction of x, of sum(dy y) of the oracle at the same rounded weights."""
    c = Case(6, 64, 96, 8)
    y, h, g, u = attt.attt_gated_ffn_forward(c.x, *c.W, **c.kw, save=True)
    dx, dg, du = attt.attt_gated_ffn_backward(c.dy, *c.W, g, u, **c.kw)
    (Wg, Wu, Wd), As, Bs = c.host()
    r = np.random.default_rng(0)
    v, x, dy = r.normal(size=(6, 64)), _host(c.x), _host(c.dy)
    e = 1e-5
    f = [(dy * bl.gated_ffn(x + s * e * v, Wg, Wu, Wd, As, Bs, c.scale)[0]).sum() for s in (1, -1)]
    # dx from g, u, dg, du rounded to bf16 and rounded itself: five roundings of 2^-8 of terms that
    # add up in 384 places with random signs, each of size |dx v|
    assert abs((f[0] - f[1]) / (2 * e) - (_host(dx) * v).sum()) < 5 * R16 * math.sqrt(384) * dx.float().abs().max().item() * 3


def test_rows_behind_the_last_and_outputs_given():
    """Outputs inside larger buffers: nothing behind the last row is written."""
    for L, d, f in ((5, 128, 264), (300, 128, 264)):
        c = Case(L, d, f, 8)
        bufs = [torch.full((L + 3, n), 7.0, dtype=torch.bfloat16, device=DEV) for n in (d, f, f, f, d, f, f)]
        y, h, g, u, dx, dg, du = (b[:L] for b in bufs)
        attt.attt_gated_ffn_forward(c.x, *c.W, **c.kw, y=y, h=h, g=g, u=u)
        attt.attt_gated_ffn_backward(c.dy, *c.W, c.g, c.u, **c.kw, dx=dx, dg=dg, du=du)
        check_forward(c, (y, h, g, u))
        check_backward(c, (dx, dg, du))
        assert all((b[L:] == 7).all() for b in bufs)


def test_a_nan_row_stays_its_own():
    c = Case(200, 128, 264, 8)
    want = attt.attt_gated_ffn_forward(c.x, *c.W, **c.kw, save=True)
    x = c.x.clone()
    x[77, 5] = float("nan")
    got = attt.attt_gated_ffn_forward(x, *c.W, **c.kw, save=True)
    rows = torch.arange(200, device=DEV) != 77
    for a, b in zip(got, want):
        assert torch.isnan(a[77]).all() and torch.equal(a[rows], b[rows])


def test_no_rows():
    c = Case(0, 64, 128, 8)
    n = attt.attt_kernel_launches()
    y, h, g, u = attt.attt_gated_ffn_forward(c.x, *c.W, **c.kw, save=True)
    dx, dg, du = attt.attt_gated_ffn_backward(c.dy, *c.W, g, u, **c.kw)
    assert y.shape == dx.shape == (0, 64) and attt.attt_kernel_launches() == n


def test_repeats_streams_and_graphs():
    """Two streams at once with workspaces of their own, and a graph: the same bits."""
    for shape in ((93, 512, 2048, 16), (600, 256, 1024, 12)):
        c = Case(*shape)

        def call(stream=None):
            out = attt.attt_gated_ffn_forward(c.x, *c.W, **c.kw, save=True, stream=stream)
            return list(out) + list(attt.attt_gated_ffn_backward(c.dy, *c.W, c.g, c.u, **c.kw, stream=stream))

        first = call()
        sides = [torch.cuda.Stream() for _ in range(2)]
        for s in sides:
            s.wait_stream(torch.cuda.current_stream())
        both = [call(s) for s in sides]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            kept = call()
        for t in kept:
            t.zero_()
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        for a, b, e, k in zip(first, *both, kept):
            assert torch.equal(a, b) and torch.equal(a, e) and torch.equal(a, k)
    assert attt.attt_device_status() == 0


@pytest.mark.parametrize("shape", [(3, 264, 1000, 8), (33, 4104, 4104, 16), (61, 904, 18952, 12), (90, 4104, 4104, 16)])
def test_few_rows_apart_on_streams_and_in_graphs(shape):
    """As above for calls of few rows: bits repeat, a NaN row stays its own, nothing behind the last
    row is written."""
    c = Case(*shape)
    L, d, f, _ = shape
    bufs = [torch.full((L + 5, n), 7.0, dtype=torch.bfloat16, device=DEV) for n in (d, f, f, f, d, f, f)]
    outs = [b[:L] for b in bufs]

    def call(x, dy, out, stream=None):
        y, h, g, u, dx, dg, du = out or [None] * 7
        got = attt.attt_gated_ffn_forward(x, *c.W, **c.kw, y=y, h=h, g=g, u=u, save=True, stream=stream)
        return list(got) + list(attt.attt_gated_ffn_backward(dy, *c.W, c.g, c.u, **c.kw, dx=dx, dg=dg, du=du, stream=stream))

    first = call(c.x, c.dy, None)
    check_forward(c, first[:4])
    check_backward(c, first[4:])
    sides = [torch.cuda.Stream() for _ in range(2)]
    for s in sides:
        s.wait_stream(torch.cuda.current_stream())
    both = [call(c.x, c.dy, None, s) for s in sides]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(c.x, c.dy, outs)
    graph.replay()
    graph.replay()
    for a, b, e, k in zip(first, *both, outs):
        assert torch.equal(a, b) and torch.equal(a, e) and torch.equal(a, k)
    assert all((b[L:] == 7).all() for b in bufs)
    x, dy = c.x.clone(), c.dy.clone()
    x[1, 5] = dy[1, 5] = float("nan")
    rows = torch.arange(L, device=DEV) != 1
    for a, b in zip(call(x, dy, None), first):
        assert torch.isnan(a[1]).all() and torch.equal(a[rows], b[rows])
    assert attt.attt_device_status() == 0


def test_refusals():
    c = Case(16, 64, 128, 8)
    fwd, bwd = attt.attt_gated_ffn_forward, attt.attt_gated_ffn_backward
    n = attt.attt_kernel_launches()
    kw = {k: v for k, v in c.kw.items() if k not in ("As", "Bs")}
    for call in (lambda: fwd(c.x.float(), *c.W), lambda: fwd(c.x[:, :56], *c.W), lambda: fwd(c.x, c.W[0], c.W[2], c.W[2]),
                 lambda: fwd(c.x, *c.W, As=c.As, **kw), lambda: fwd(c.x, *c.W, As=c.As[:2], Bs=c.Bs[:2]),
                 lambda: fwd(c.x, *c.W, As=c.As, Bs=[None] + c.Bs[1:]), lambda: fwd(c.x, *c.W, act="relu"),
                 lambda: fwd(c.x, *c.W, As=[None] * 3, Bs=c.Bs), lambda: fwd(c.x, *c.W, h=c.x),
                 lambda: fwd(c.x.cpu(), *c.W), lambda: bwd(c.dy, *c.W, c.g[:3], c.u), lambda: bwd(c.dy, *c.W, c.g, c.u.float()),
                 lambda: fwd(c.x, *(w.t().contiguous().t() for w in c.W))):
        with pytest.raises(ValueError):
            call()
    small = torch.empty(256, dtype=torch.uint8, device=DEV)
    odd = [torch.zeros(s, dtype=torch.bfloat16, device=DEV) for s in ((16, 60), (60, 128), (60, 128), (128, 60))]
    for call, code in ((lambda: fwd(c.x, *c.W, workspace=small, **c.kw), attt.ATTT_ERR_WORKSPACE),
                       (lambda: bwd(c.dy, *c.W, c.g, c.u, workspace=small, **c.kw), attt.ATTT_ERR_WORKSPACE),
                       (lambda: fwd(*odd), attt.ATTT_ERR_INVALID_ARG)):
        with pytest.raises(attt.AtttError) as e:
            call()
        assert e.value.code == code
    big = Case(4, 64, 64, 72)
    with pytest.raises(attt.AtttError):
        fwd(big.x, *big.W, **big.kw)
    assert attt.attt_kernel_launches() == n and attt.attt_device_status() == 0

"""attt_layer_norm_forward / attt_layer_norm_backward against the fp64 oracle.

Bounds, u = 2^-24: a row's sum goes through at most 32 additions in a thread, ten
in shuffles and one per 1,024 threads' worth of longer rows, so it is off by at
most 64 u of the sum of its terms' sizes (rows of up to 21,000 values); what follows
adds a few u.  Results rounded to bf16 (8 bits) are off by 2^-8 of themselves.  A
weight's sum over the rows takes at most 93 additions in a thread (14,000 rows in 152
blocks), 26 across blocks and 16 between groups: 256 u of its terms."""
import numpy as np
import pytest
import torch

from oracle import operators as op
from paper_2607_03441_gb300 import attt, build
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _library():
    build.build()


def _rows(a, dtype, pad=0, at=0):
    """A device tensor of a's values as rows of a buffer `pad` wider, NaN elsewhere."""
    L, d = a.shape
    buf = torch.full((L, d + pad), float("nan"), dtype=dtype, device=DEV)
    buf[:, at:at + d] = torch.from_numpy(np.asarray(a, dtype=np.float32)).to(DEV).to(dtype)
    return buf[:, at:at + d]


def _host(t):
    return t.double().cpu().numpy()


def _inputs(seed, L, d, dtype, pad, at, offset=0.5):
    r = np.random.default_rng(seed)
    x = _rows(r.normal(size=(L, d)) * np.exp(r.normal(size=d)) + offset, dtype, pad, at)
    dy = _rows(r.normal(size=(L, d)) * 1e-3, dtype, pad, at)
    g, b = (torch.from_numpy(v.astype(np.float32)).to(DEV) for v in (1 + 0.1 * r.normal(size=d), r.normal(size=d)))
    return x, dy, g, b


CASES = [  # L, d, dtype, row padding, first column
    (1, 1, torch.float32, 0, 0), (1, 1, torch.bfloat16, 0, 0), (3, 7, torch.bfloat16, 0, 0),
    (5, 8, torch.bfloat16, 0, 0), (2, 33, torch.float32, 3, 1), (1, 5120, torch.bfloat16, 0, 0),
    (16, 4096, torch.float32, 8, 4), (37, 512, torch.bfloat16, 64, 8), (700, 64, torch.bfloat16, 0, 0),
    (2500, 200, torch.float32, 4, 0), (2001, 1000, torch.bfloat16, 8, 0), (1300, 777, torch.bfloat16, 1, 1),
    (1300, 2049, torch.float32, 0, 0), (211, 3577, torch.float32, 7, 0), (1300, 5120, torch.bfloat16, 0, 0),
    (9, 8191, torch.bfloat16, 0, 0), (4, 8200, torch.bfloat16, 0, 0), (1400, 8192, torch.float32, 0, 0),
    (3, 16384, torch.bfloat16, 0, 0), (7, 20992, torch.float32, 0, 0), (3, 20001, torch.bfloat16, 0, 0),
    (14000, 24, torch.float32, 0, 0),
]


@pytest.mark.parametrize("L,d,dtype,pad,at", CASES)
@pytest.mark.parametrize("bias", [True, False])
def test_forward(L, d, dtype, pad, at, bias):
    x, _, g, b = _inputs(L + d, L, d, dtype, pad, at)
    y = _rows(np.zeros((L, d)), dtype, pad, at)
    got = attt.attt_layer_norm_forward(x, g, b if bias else None, eps=1e-5, y=y)
    assert got[0] is y and attt.attt_device_status() == 0
    xh, gh = _host(x), _host(g)
    want, mean, rstd = op.layer_norm(xh, gh, _host(b) if bias else None, 1e-5)
    dm = 64 * U * np.abs(xh).mean(1)
    assert (np.abs(_host(got[1]) - mean) <= dm).all()
    rel = 64 * U + rstd * dm * rstd * dm + 2 * U  # half of var's, from the sum and from the mean
    assert (np.abs(_host(got[2]) - rstd) <= rel * rstd).all()
    unit = np.abs((xh - mean[:, None]) * rstd[:, None])
    tol = np.abs(gh) * (rstd * dm + unit.T * (rel + 4 * U)).T + 4 * U * np.abs(want) + 2 * U * np.abs(gh) * unit
    tol += (2.0 ** -8 if dtype == torch.bfloat16 else U) * np.abs(want) + 1e-30
    assert (np.abs(_host(y) - want) <= tol).all()
    if pad:  # nothing beside the rows was written
        assert torch.isnan(y.as_strided((L, d + pad), (d + pad, 1), y.storage_offset() - at)).sum().item() == L * pad


@pytest.mark.parametrize("L,d,dtype,pad,at", CASES)
def test_backward(L, d, dtype, pad, at):
    x, dy, g, _ = _inputs(L + d, L, d, dtype, pad, at)
    _, mean, rstd = attt.attt_layer_norm_forward(x, g)
    dx = _rows(np.zeros((L, d)), dtype, pad, at)
    got = attt.attt_layer_norm_backward(dy, x, g, mean, rstd, dx=dx)
    assert got[0] is dx and attt.attt_device_status() == 0
    xh_, dyh, gh, m, r = (_host(t) for t in (x, dy, g, mean, rstd))
    want, dg, db = op.layer_norm_grad(dyh, xh_, gh, m, r)
    xh = (xh_ - m[:, None]) * r[:, None]
    gg = dyh * gh
    s1, s2 = np.abs(gg).mean(1)[:, None], np.abs(gg * xh).mean(1)[:, None]
    tol = r[:, None] * ((64 + 8) * U * (s1 + np.abs(xh) * s2) + 8 * U * (np.abs(gg) + np.abs(xh) * s2 + s1))
    # xh itself: fl(x - mean) is off by u of it
    tol += (2.0 ** -8 if dtype == torch.bfloat16 else U) * np.abs(want) + 1e-30
    assert (np.abs(_host(dx) - want) <= tol).all()
    assert (np.abs(_host(got[1]) - dg) <= 256 * U * np.abs(dyh * xh).sum(0) + 1e-30).all()
    assert (np.abs(_host(got[2]) - db) <= 256 * U * np.abs(dyh).sum(0) + 1e-30).all()


def test_gradient_against_differences():
    """Of sum(dy y) in fp64, along random directions of x, gamma and beta."""
    L, d = 40, 96
    x, dy, g, b = _inputs(1, L, d, torch.float32, 0, 0)
    _, mean, rstd = attt.attt_layer_norm_forward(x, g, b)
    dx, dg, db = (_host(t) for t in attt.attt_layer_norm_backward(dy, x, g, mean, rstd))
    xh, dyh, gh, bh = (_host(t) for t in (x, dy, g, b))
    r = np.random.default_rng(0)

    def f(x_, g_, b_):
        return (dyh * op.layer_norm(x_, g_, b_, 1e-5)[0]).sum()

    for grad, args in ((dx, 0), (dg, 1), (db, 2)):
        v = [np.zeros_like(xh), np.zeros_like(gh), np.zeros_like(bh)]
        v[args] = r.normal(size=v[args].shape)
        e = 1e-5
        up, down = (f(*(p + s * e * w for p, w in zip((xh, gh, bh), v))) for s in (1, -1))
        # fp32 gradients, u of terms of 1e-3 over 4,000 values; differences 1e-10 of them
        assert abs((up - down) / (2 * e) - (grad * v[args]).sum()) < 1e-7


def test_large_offset_keeps_the_variance():
    """A mean 1,000 times the spread: the variance is of centred values, so y is off
    by the mean's own rounding (64 u of 1,000 spreads), not by 1,000^2 u."""
    x, _, g, b = _inputs(2, 50, 1536, torch.float32, 0, 0, offset=0.0)
    x = (x / x.std() + 1000).contiguous()
    y, mean, rstd = attt.attt_layer_norm_forward(x, g, b)
    want = op.layer_norm(_host(x), _host(g), _host(b))[0]
    assert np.abs(_host(y) - want).max() <= 64 * U * 1000 * _host(rstd).max() * _host(g).max() + 1e-4


def test_constant_rows_and_nan_rows():
    x = torch.full((4, 520), 3.0, device=DEV)
    x[2, 7] = float("nan")
    x[3, 8] = float("inf")
    g, b = torch.ones(520, device=DEV), torch.full((520,), 0.25, device=DEV)
    y, mean, rstd = attt.attt_layer_norm_forward(x, g, b, eps=1e-5)
    assert (y[:2] == 0.25).all() and (mean[:2] == 3).all()
    assert torch.isnan(y[2:]).all()
    y, _, _ = attt.attt_layer_norm_forward(x[:2], g, b, eps=0.0)  # 0 / 0, as the formula has it
    assert torch.isnan(y).all()


def test_no_rows():
    x = torch.empty(0, 64, dtype=torch.bfloat16, device=DEV)
    g = torch.ones(64, device=DEV)
    y, mean, rstd = attt.attt_layer_norm_forward(x, g)
    assert y.shape == (0, 64) and mean.shape == (0,)
    dx, dg, db = attt.attt_layer_norm_backward(x, x, g, mean, rstd)
    assert not dg.any() and not db.any() and attt.attt_device_status() == 0


def test_repeats_and_streams():
    x, dy, g, b = _inputs(3, 3000, 640, torch.bfloat16, 0, 0)
    first = attt.attt_layer_norm_forward(x, g, b)
    grads = attt.attt_layer_norm_backward(dy, x, g, *first[1:])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = attt.attt_layer_norm_forward(x, g, b, stream=side)
    with torch.cuda.stream(side):
        grads2 = attt.attt_layer_norm_backward(dy, x, g, *again[1:])
    torch.cuda.synchronize()
    for p, q in zip(first + grads, again + grads2):
        assert torch.equal(p, q)


def test_refusals():
    x, dy, g, b = _inputs(4, 6, 40, torch.float32, 0, 0)
    fwd, bwd = attt.attt_layer_norm_forward, attt.attt_layer_norm_backward
    m = torch.ones(6, device=DEV)
    launches = attt.attt_kernel_launches()
    for call in (lambda: fwd(x.half(), g), lambda: fwd(x, g[:39]), lambda: fwd(x, g.double()), lambda: fwd(x, g, b[:3]),
                 lambda: fwd(x.t(), torch.ones(6, device=DEV)), lambda: fwd(x, g, y=dy.bfloat16()),
                 lambda: fwd(x[:1].expand(6, 40), g), lambda: fwd(x.cpu(), g), lambda: bwd(dy.bfloat16(), x, g, m, m),
                 lambda: bwd(dy, x, g, m[:5], m), lambda: bwd(dy, x, g, m, m, dgamma=m)):
        with pytest.raises(ValueError):
            call()
    for call, code in ((lambda: fwd(x, g, eps=-1.0), attt.ATTT_ERR_INVALID_ARG),
                       (lambda: fwd(x, g, eps=float("nan")), attt.ATTT_ERR_INVALID_ARG),
                       (lambda: bwd(dy, x, g, m, m, workspace=torch.empty(256, dtype=torch.uint8, device=DEV)),
                        attt.ATTT_ERR_WORKSPACE)):
        with pytest.raises(attt.AtttError) as e:
            call()
        assert e.value.code == code
    assert attt.attt_kernel_launches() == launches and attt.attt_device_status() == 0

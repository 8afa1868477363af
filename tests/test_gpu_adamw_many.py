"""attt_adamw_step over many tensors: with moments in 32 bits the bits of
attt_lora_adamw_step, with moments in 8 the codes and scales of the oracle, whose fp32
operations are the documented ones in their order, and parameters whose update m / denom goes
through an approximate reciprocal: 2 u of its own, five roundings before and after, 2^-21 of
the update, and two roundings of p (u = 2^-24)."""
import numpy as np
import pytest
import torch

from oracle import blocks as bl
from paper_2607_03441_gb300 import attt, build
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu
HYPER = dict(lr=3e-3, b1=0.9, b2=0.98, eps=1e-7, wd=0.05)
SIZES = [1, 255, 256, 257, 4099, 16 * 3584, 8 * 512, 70000, 3, 1000]


@pytest.fixture(scope="module", autouse=True)
def _library():
    build.build()


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _same(t, a):
    return np.array_equal(t.cpu().numpy().view(np.uint8), np.ascontiguousarray(a).view(np.uint8))


def _step(opt, t, seed=0, **kw):
    h = HYPER | kw
    attt.attt_adamw_step(opt, h["lr"], (h["b1"], h["b2"]), h["eps"], h["wd"], t, seed)


def _tensors(sizes, offset=0, seed=0):
    """p, g, m, v, p16 of each size, `offset` values behind an aligned address."""
    r = np.random.default_rng(seed)
    out = []
    for n in sizes:
        p, g = r.normal(size=n).astype(np.float32), (r.normal(size=n) * np.exp(2 * r.normal())).astype(np.float32)
        bufs = []
        for a in (p, g, 0 * p, 0 * p):
            b = torch.full((n + offset + 1,), 7.0, device=DEV)
            b[offset:offset + n] = _dev(a)
            bufs.append(b[offset:offset + n])
        bufs.append(torch.zeros(n + offset, dtype=torch.bfloat16, device=DEV)[offset:])
        out.append(bufs)
    return [list(t) for t in zip(*out)]


@pytest.mark.parametrize("offset", [0, 1])
def test_32_bits_are_those_of_the_step_of_one_adapter(offset):
    ps, gs, ms, vs, p16s = _tensors(SIZES, offset)
    lr = float(np.float32(HYPER["lr"]))  # as the other call takes it
    ref = [[t.clone() for t in ts] for ts in (ps, gs, ms, vs, p16s)]
    opt = attt.attt_adamw_create(ps, gs, ms, vs, p16s=p16s)
    for t in (1, 2, 1000):
        _step(opt, t, lr=lr)
        for p, g, m, v, p16 in zip(*ref):
            e = torch.zeros(1, 1, device=DEV)  # the call steps an A and a B: B is one value here
            es = [e.clone() for _ in range(4)]
            attt.attt_lora_adamw_step(p.view(-1, 1), es[0], g.view(-1, 1), es[1], m.view(-1, 1), v.view(-1, 1), es[2],
                                      es[3], lr, betas=(HYPER["b1"], HYPER["b2"]), eps=HYPER["eps"],
                                      weight_decay=HYPER["wd"], step=t, A16=p16.view(-1, 1))
        for got, want in zip((ps, ms, vs, p16s), (ref[0], ref[2], ref[3], ref[4])):
            assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert attt.attt_device_status() == 0
    if offset:  # nothing behind or before a tensor was written
        assert all(b._base[0] == 7 and b._base[-1] == 7 for b in ps + ms + vs)


@pytest.mark.parametrize("offset", [0, 1])
def test_8_bits(offset):
    ps, gs, _, _, p16s = _tensors(SIZES, offset, seed=1)
    ms, vs = ([torch.zeros(n + offset, dtype=torch.uint8, device=DEV)[offset:] for n in SIZES] for _ in range(2))
    sms, svs = ([torch.zeros(-(-n // 256), device=DEV) for n in SIZES] for _ in range(2))
    opt = attt.attt_adamw_create(ps, gs, ms, vs, sms, svs, p16s)
    host = [[t.cpu().numpy() for t in ts] for ts in (ps, gs, ms, vs, sms, svs)]
    for t, seed in ((1, 11), (2, (5 << 32) + 12), (3, 2 ** 64 - 1)):
        _step(opt, t, seed)
        for k in range(len(SIZES)):
            p, m8, v8, sm, sv = bl.adamw8(*(h[k] for h in host), **HYPER, t=t, seed=seed, tensor=k)
            before = host[0][k].astype(np.float64)
            host[0][k], host[2][k], host[3][k], host[4][k], host[5][k] = ps[k].cpu().numpy(), m8, v8, sm, sv
            for got, want in zip((ms, vs, sms, svs), (m8, v8, sm, sv)):
                assert _same(got[k], want), (t, k)
            update = np.abs(p - before * (1 - HYPER["lr"] * HYPER["wd"]))
            assert (np.abs(host[0][k].astype(np.float64) - p) <= 2.0 ** -21 * update + 4 * 2.0 ** -24 * np.abs(before)).all()
            assert torch.equal(p16s[k], ps[k].to(torch.bfloat16))
        m32, v32 = attt.attt_adamw_read_state(opt)
        at = 0
        for k, n in enumerate(SIZES):
            m, v = bl.read_state(*(host[i][k] for i in (2, 3, 4, 5)))
            assert _same(m32[at:at + n], m) and _same(v32[at:at + n], v)
            end = at + 256 * (-(-n // 256))
            assert not m32[at + n:end].any() and not v32[at + n:end].any()
            at = end
        assert at == m32.numel() == attt.attt_adamw_state_values(opt)
        for ts in (gs,):  # other gradients for the next step
            for k, g in enumerate(ts):
                g.mul_(-0.7)
                host[1][k] = g.cpu().numpy()
    assert attt.attt_device_status() == 0


def test_8_bits_follow_32():
    """200 steps down a quadratic: the 8-bit step ends where the 32-bit one does.  m's code is off by at most a
    step, 2^-3 of it, sqrt(v)'s by 2^-4, without bias; the sum over some 1 / (1 - b1) = 10 independent
    roundings of m and as many steps as p moves keeps p within 2^-3 of the way gone."""
    n = 5000
    r = np.random.default_rng(2)
    target = _dev(r.normal(size=n).astype(np.float32))
    runs = []
    for bits in (32, 8):
        p, g = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
        if bits == 32:
            opt = attt.attt_adamw_create([p], [g], [torch.zeros(n, device=DEV)], [torch.zeros(n, device=DEV)])
        else:
            m, v = (torch.zeros(n, dtype=torch.uint8, device=DEV) for _ in range(2))
            opt = attt.attt_adamw_create([p], [g], [m], [v], [torch.zeros(20, device=DEV)], [torch.zeros(20, device=DEV)])
        for t in range(1, 201):
            g.copy_(p - target)
            attt.attt_adamw_step(opt, 1e-3, weight_decay=0.0, step=t, seed=t)
        runs.append(p)
    assert (runs[1] - runs[0]).norm() <= runs[0].norm() / 8


def test_moments_fall_without_gradients():
    """b2 = 0.999 takes 1/2000 of sqrt(v) a step, far less than a code's step of 2^-5 or more: after 1,000
    steps v's mean has fallen as b2^1000 says, within a tenth (5,120 values, each rounded at random
    by up to a step of 1/16 and some 20 times on its way)."""
    n = 5120
    p, g = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    g.uniform_(0.5, 1.0)
    m, v = (torch.zeros(n, dtype=torch.uint8, device=DEV) for _ in range(2))
    opt = attt.attt_adamw_create([p], [g], [m], [v], [torch.zeros(20, device=DEV)], [torch.zeros(20, device=DEV)])
    attt.attt_adamw_step(opt, 0.0, step=1, seed=1)
    start = attt.attt_adamw_read_state(opt)[1].mean().item()
    g.zero_()
    for t in range(2, 1002):
        attt.attt_adamw_step(opt, 0.0, step=t, seed=t)
    m32, v32 = attt.attt_adamw_read_state(opt)
    assert 0.9 < v32.mean().item() / (start * 0.999 ** 1000) < 1.1
    assert not m32.any()  # 0.9^1000


def test_blocks_of_zeros_small_values_and_nans():
    n = 256 * 6
    for bits in (32, 8):
        p, g = torch.ones(n, device=DEV), torch.zeros(n, device=DEV)
        g[256:512] = 1e-36
        g[513] = float("nan")
        g[768:1024] = 1.0
        g[1025] = float("inf")
        g[1280:] = 1e-3
        dt = torch.float32 if bits == 32 else torch.uint8
        m, v = torch.zeros(n, dtype=dt, device=DEV), torch.zeros(n, dtype=dt, device=DEV)
        s = [[torch.zeros(6, device=DEV)] for _ in range(2)] if bits == 8 else [None, None]
        opt = attt.attt_adamw_create([p], [g], [m], [v], *s)
        attt.attt_adamw_step(opt, 0.1, weight_decay=0.0, step=1, seed=3)
        assert (p[:256] == 1).all() and torch.isfinite(p[:512]).all() and torch.isnan(p[513])
        assert torch.isfinite(p[514:1024]).all() and torch.isfinite(p[1280:]).all()
        m32, v32 = attt.attt_adamw_read_state(opt)
        bad = torch.isnan(m32).view(6, 256).sum(1).tolist()
        if bits == 8:
            assert bad == [0, 0, 256, 0, 256, 0] and not m32[:512].any() and not v32[:512].any()
            assert (m32[768:1024] > 0).all()
        else:
            assert bad == [0, 0, 1, 0, 0, 0] and torch.isinf(m32[1025])


def test_same_seed_repeats_and_another_differs():
    got = []
    for seed in (1, 1, 2):
        ps, gs, _, _, _ = _tensors([70000])
        m, v = (torch.zeros(70000, dtype=torch.uint8, device=DEV) for _ in range(2))
        opt = attt.attt_adamw_create(ps, gs, [m], [v], [torch.zeros(274, device=DEV)], [torch.zeros(274, device=DEV)])
        _step(opt, 1, seed)
        got.append((ps[0], m, v))
    assert all(torch.equal(a, b) for a, b in zip(got[0], got[1]))
    assert torch.equal(got[0][0], got[2][0]) and not torch.equal(got[0][1], got[2][1])
    assert not torch.equal(got[0][2], got[2][2])


def test_graph_stream_and_many_tensors():
    sizes = [64 + 8 * (k % 50) for k in range(900)] + [0]
    ps, gs, ms, vs, p16s = _tensors(sizes, seed=4)
    qs, _, ns, ws, _ = _tensors(sizes, seed=4)
    opt, ref = attt.attt_adamw_create(ps, gs, ms, vs, p16s=p16s), attt.attt_adamw_create(qs, gs, ns, ws)
    _step(ref, 5)
    _step(ref, 5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    attt.attt_adamw_step(opt, HYPER["lr"], (HYPER["b1"], HYPER["b2"]), HYPER["eps"], HYPER["wd"], 5, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    n = attt.attt_kernel_launches()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _step(opt, 5)
    assert attt.attt_kernel_launches() == n + 1
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(ps + ms + vs, qs + ns + ws):
        assert torch.equal(a, b)


def test_some_bf16_copies_and_matrices():
    """Tensors of two dimensions, with and without a bf16 copy, one without values."""
    ps = [torch.randn(s, device=DEV) for s in ((16, 40), (0, 5), (300,))]
    gs, ms, vs = ([torch.randn_like(p) if k == 0 else torch.zeros_like(p) for p in ps] for k in range(3))
    p16s = [torch.zeros(16, 40, dtype=torch.bfloat16, device=DEV), None, None]
    ref = [p.clone() for p in ps]
    one = attt.attt_adamw_create(ps, gs, ms, vs, p16s=p16s)
    _step(one, 1)
    _step(attt.attt_adamw_create(ref, gs, [torch.zeros_like(p) for p in ps], [torch.zeros_like(p) for p in ps]), 1)
    assert all(torch.equal(a, b) for a, b in zip(ps, ref)) and torch.equal(p16s[0], ps[0].to(torch.bfloat16))
    assert attt.attt_adamw_state_values(one) == 256 * (3 + 0 + 2)


def test_values_without_gradients_stay_in_8_bits():
    """No moments, no gradient, no decay: p keeps its bits, whatever eps."""
    p, g = torch.randn(700, device=DEV), torch.zeros(700, device=DEV)
    before = p.clone()
    m, v = (torch.zeros(700, dtype=torch.uint8, device=DEV) for _ in range(2))
    opt = attt.attt_adamw_create([p], [g], [m], [v], [torch.zeros(3, device=DEV)], [torch.zeros(3, device=DEV)])
    for eps in (1e-30, 1e-8, 1.0):
        attt.attt_adamw_step(opt, 0.1, eps=eps, weight_decay=0.0, step=1, seed=1)
    assert torch.equal(p, before) and not m.any() and not v.any()
    with pytest.raises(attt.AtttError):
        attt.attt_adamw_step(opt, 0.1, eps=1e-31)


def test_refusals():
    f = lambda n: torch.zeros(n, device=DEV)  # noqa: E731
    b = lambda n: torch.zeros(n, dtype=torch.uint8, device=DEV)  # noqa: E731
    create = attt.attt_adamw_create
    one = f(600)
    n = attt.attt_kernel_launches()
    for call in (lambda: create([], [], [], []), lambda: create([f(4)], [f(5)], [f(4)], [f(4)]),
                 lambda: create([f(4)], [f(4).bfloat16()], [f(4)], [f(4)]), lambda: create([f(4)], [f(4)], [b(4)], [b(4)]),
                 lambda: create([f(4)], [f(4)], [f(4)], [f(4)], [f(1)], [f(1)]),
                 lambda: create([f(257)], [f(257)], [b(257)], [b(257)], [f(1)], [f(2)]),
                 lambda: create([f(4), f(4)], [f(4)], [f(4)], [f(4)]), lambda: create([f(8)[::2]], [f(4)], [f(4)], [f(4)]),
                 lambda: create([f(4)], [f(4)], [f(4)], [f(4)], p16s=[f(4)])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: create([one[:300]], [f(300)], [one[:300]], [f(300)]),          # p is m
                 lambda: create([one[:300]], [f(300)], [one[299:599]], [f(300)]),       # they share a value
                 lambda: create([one[:300], one[200:600]], [f(300), f(400)], [f(300), f(400)], [f(300), f(400)]),
                 lambda: create([one[:300]], [one[100:400]], [f(300)], [f(300)])):      # the gradient lies in p
        with pytest.raises(attt.AtttError) as e:
            call()
        assert e.value.code == attt.ATTT_ERR_INVALID_ARG
    opt = create([f(4)], [f(4)], [f(4)], [f(4)])
    for kw in (dict(step=0), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=0.0), dict(eps=1e-60),
               dict(weight_decay=-1.0), dict(weight_decay=float("nan"))):
        with pytest.raises(attt.AtttError) as e:
            attt.attt_adamw_step(opt, 0.1, **kw)
        assert e.value.code == attt.ATTT_ERR_INVALID_ARG
    with pytest.raises(attt.AtttError):
        attt.attt_adamw_step(opt, float("inf"))
    attt.attt_fault_inject("alloc")
    with pytest.raises(attt.AtttError) as e:
        create([f(4)], [f(4)], [f(4)], [f(4)])
    assert e.value.code == attt.ATTT_ERR_CUDA
    opt.close()
    with pytest.raises(attt.AtttError):
        attt.attt_adamw_step(opt, 0.1)
    assert attt.attt_kernel_launches() == n and attt.attt_device_status() == 0

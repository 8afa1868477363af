"""attt_logprob_forward / attt_logprob_input_grad against the fp64 oracle.

Inputs lie on grids (hidden states multiples of 1/8 up to 4, heads of 1/256 up to
1/4), so that every logit is exact in fp32 in any order of its sum and the ids
of the alternatives have to agree exactly.  What is left is fp32 arithmetic on the
logits: terms of a sum of exponentials carry 2^-22 each from ex2 and its
argument (up to 64 in log2 units: 2^-24 of it), so values of size s are held
to 1e-5 (1 + s), the entropies' moments included."""
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


def _bf16(a):
    return torch.from_numpy(np.asarray(a, dtype=np.float32)).to(DEV).to(torch.bfloat16)


def _inputs(seed, L, d, V, peaked=True):
    r = np.random.default_rng(seed)
    h = np.clip(np.round(r.normal(size=(L, d)) * 8), -32, 32) / 8
    W = np.clip(np.round(r.normal(size=(V, d)) * 20), -64, 64) / 256
    tgt = r.integers(0, V, L).astype(np.int32)
    if peaked:  # some rows know their token
        for j in range(0, L, 3):
            h[j] = np.clip(np.round(W[tgt[j]] * 8 * 40), -32, 32) / 8
    tgt[1::5] = -1
    return h, W, tgt


def _run(h, W, tgt, topk, inv_temp, **kw):
    out = attt.attt_logprob_forward(_bf16(h), _bf16(W), torch.from_numpy(tgt).to(DEV), topk=topk, inv_temp=inv_temp,
                                    **kw)
    assert attt.attt_device_status() == 0
    return [t.cpu().numpy() for t in out]


def _close(got, want, what):
    err = np.abs(got - want) / (1 + np.abs(want))
    assert err.max(initial=0.0) <= 1e-5, (what, err.max())


CASES = [  # L, d, V, topk, inv_temp
    (1, 8, 1, 1, 1.0), (1, 64, 7, 7, 1.0), (2, 72, 63, 0, 0.5), (3, 64, 64, 5, 1.0), (31, 136, 65, 20, 2.0),
    (1, 512, 8192, 5, 1.0), (16, 512, 8191, 20, 1 / 0.7), (129, 128, 1000, 8, 1.0), (127, 1600, 257, 9, 1.0),
    (257, 64, 255, 1, 1.0), (300, 520, 5001, 12, 0.25), (513, 128, 2049, 20, 1.0), (1000, 64, 300, 3, 1.25),
    # runs of tiles that end inside a row of tiles, begin inside one, or go over to the next
    (700, 72, 15000, 5, 1.0), (2400, 264, 2100, 20, 0.5), (5000, 64, 700, 1, 1.0), (1111, 1608, 6000, 0, 1.0),
]


@pytest.mark.parametrize("L,d,V,topk,inv_temp", CASES)
def test_forward(L, d, V, topk, inv_temp):
    h, W, tgt = _inputs(L + V, L, d, V)
    inv_temp = float(np.float32(inv_temp))
    got = _run(h, W, tgt, topk, inv_temp)
    want = op.logprobs(h, W, tgt, topk, inv_temp)
    for g, w, what in zip(got, want, ("logp", "entropy", "lse", "top_logp")):
        _close(g, w, what)
    assert np.array_equal(got[4], want[4])


@pytest.mark.parametrize("order", ["falling", "rising", "equal", "pairs"])
def test_alternatives_in_any_order_of_the_vocabulary(order):
    """Logits that fall or rise along the vocabulary, that are all equal, or equal
    in pairs far apart: ties go to the lowest id."""
    V, d, L = 3000, 64, 70
    rank = {"falling": -np.arange(V), "rising": np.arange(V), "equal": np.zeros(V),
            "pairs": -(np.arange(V) % 1500)}[order]
    W = np.zeros((V, d))
    W[:, 0], W[:, 1] = np.floor(rank / 64), rank % 64  # exact in bf16, z = 64 W_0 + W_1
    h = np.zeros((L, d))
    h[:, 0], h[:, 1] = 64, 1
    h[40:] /= 64
    tgt = np.full(L, 5, dtype=np.int32)
    got = _run(h, W, tgt, 20, 1.0)
    want = op.logprobs(h, W, tgt, 20)
    assert np.array_equal(got[4], want[4])
    for g, w, what in zip(got[:4], want, ("logp", "entropy", "lse", "top_logp")):
        _close(g, w, what)


@pytest.mark.parametrize("L,topk", [(1300, 20), (2100, 8), (1700, 1)])
def test_equal_logits_over_many_rows(L, topk):
    """Every logit of a row occurs 40 times: the lowest ids come first, wherever the runs
    of tiles begin and end."""
    V, d = 12000, 64
    W = np.zeros((V, d))
    W[:, 0], W[:, 1] = np.floor(-(np.arange(V) % 300) / 64), -(np.arange(V) % 300) % 64
    h = np.zeros((L, d))
    h[:, 0], h[:, 1] = 1, 1 / 64
    h[::2] *= -1  # the least ones become the largest
    tgt = np.full(L, 5, dtype=np.int32)
    got = _run(h, W, tgt, topk, 1.0)
    want = op.logprobs(h[:2], W, tgt[:2], topk)
    assert np.array_equal(got[4], want[4][np.arange(L) % 2])
    for g, w, what in zip(got[:4], want, ("logp", "entropy", "lse", "top_logp")):
        _close(g, w[np.arange(L) % 2], what)


def test_rows_of_wider_tensors_and_given_outputs():
    h, W, tgt = _inputs(5, 37, 96, 700)
    wide = torch.full((37, 200), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[:, 8:104] = _bf16(h)
    out = {"logp": torch.full((37,), 9.0, device=DEV), "entropy": torch.full((37,), 9.0, device=DEV)}
    got = attt.attt_logprob_forward(wide[:, 8:104], _bf16(W), torch.from_numpy(tgt).to(DEV), topk=4, **out)
    assert got[0] is out["logp"] and got[1] is out["entropy"]
    want = op.logprobs(h, W, tgt, 4)
    for g, w, what in zip(got, want, ("logp", "entropy", "lse", "top_logp")):
        _close(g.cpu().numpy(), w, what)
    assert np.array_equal(got[4].cpu().numpy(), want[4])


def test_row_blocks():
    """A call of more rows than one block takes equals the calls on its parts."""
    L, d, V = 90000, 8, 9000
    g = torch.Generator(device=DEV).manual_seed(3)
    h = (torch.randn(L, d, generator=g, device=DEV) * 8).round().clamp(-32, 32).div(8).to(torch.bfloat16)
    W = (torch.randn(V, d, generator=g, device=DEV) * 20).round().clamp(-64, 64).div(256).to(torch.bfloat16)
    tgt = torch.randint(-1, V, (L,), generator=g, device=DEV, dtype=torch.int32)
    assert attt.attt_logprob_workspace_bytes(L, d, V, 20) < 900 << 20
    whole = attt.attt_logprob_forward(h, W, tgt, topk=20)
    for a, b in ((0, 300), (30000, 30500), (60300, 60600), (89500, 90000)):
        part = attt.attt_logprob_forward(h[a:b], W, tgt[a:b].contiguous(), topk=20)
        assert torch.equal(part[4], whole[4][a:b])
        for x, y in zip(part[:4], whole[:4]):
            assert torch.allclose(x, y[a:b], rtol=1e-5, atol=1e-5)


def test_no_given_tokens_and_single_outputs():
    h, W, tgt = _inputs(6, 20, 64, 500)
    lp, ent, lse, top, ids = attt.attt_logprob_forward(_bf16(h), _bf16(W))
    assert lp is None and top.shape == (20, 0) and ids.shape == (20, 0)
    want = op.logprobs(h, W)
    _close(ent.cpu().numpy(), want[1], "entropy")
    _close(lse.cpu().numpy(), want[2], "lse")


def test_infinite_and_nan_logits():
    """-inf logits take no part (all but one: entropy 0); NaN and +inf make their row
    NaN without touching the others; the alternatives leave NaN and -inf out."""
    d, V = 64, 600
    h, W = np.zeros((4, d)), np.zeros((V, d))
    h[:, 0] = 1
    W[:, 0] = np.arange(V) % 7
    W[300, 0] = -np.inf  # finite h: z = -inf + 0 in every row
    h[1, 1] = np.nan
    h[2, 0] = -1       # z_300 = +inf in row 2
    h[3, 0] = 2
    got = _run(h, W, np.array([1, 2, 3, 300], dtype=np.int32), 8, 1.0)
    z = np.where(np.arange(V) == 300, -np.inf, np.arange(V) % 7.0)
    for j, f in ((0, 1.0), (3, 2.0)):
        zt = z * f
        lse = np.log(np.exp(zt).sum())
        p = np.exp(zt - lse)
        H = -(p[p > 0] * (zt - lse)[p > 0]).sum()
        _close(got[2][j], lse, "lse")
        _close(got[1][j], H, "entropy")
        assert np.array_equal(got[4][j], np.argsort(-z, kind="stable")[:8])
    _close(got[0][0], z[1] - got[2][0], "logp")
    assert got[0][3] == -np.inf
    assert np.isnan(got[0][1]) and np.isnan(got[1][1]) and np.isnan(got[2][1]) and (got[4][1] == -1).all()
    assert np.isnan(got[1][2]) and not np.isfinite(got[2][2])
    assert got[4][2][0] == 300


@pytest.mark.parametrize("L", [1, 20, 40, 700])
@pytest.mark.parametrize("gap", [9.0, 14.0, 30.0])
def test_rows_that_are_nearly_sure(L, gap):
    """One token far above all others, which differ: 1 - p, down to 1e-10, and what follows
    from it keep their 24 bits.  Terms carry 2^-22 from ex2 and its argument (up to 64
    in log2 units: 2^-24 of it, 4e-6), sums of them no more: 1e-5 of each value."""
    d, V = 64, 5000
    r = np.random.default_rng(int(gap))
    h, W = np.zeros((L, d)), np.zeros((V, d))
    h[:, 0] = 1
    W[:, 0] = r.integers(0, 64, V) / 32
    sure = r.integers(0, V, L).astype(np.int32)
    for j in range(L):  # a column of h of its own for every 16th row
        h[j, 1 + j % 16] = 1
        sure[j] = sure[j % 16]
        W[sure[j], 1 + j % 16] = gap
    want = op.logprobs(h, W, sure, 3)
    got = _run(h, W, sure, 3, 1.0)
    for g, w, what in zip(got[:4], want, ("logp", "entropy", "lse", "top_logp")):
        assert (np.abs(g - w) <= 1e-5 * np.abs(w)).all(), (what, np.abs((g - w) / w).max())


def test_one_finite_logit():
    W = np.zeros((300, 8))
    W[:, 0] = -np.inf
    W[77, 0] = 1
    got = _run(np.eye(2, 8)[[0, 0]], W, np.array([77, 0], dtype=np.int32), 3, 1.0)
    assert got[0][0] == 0 and got[0][1] == -np.inf and (got[1] == 0).all() and np.allclose(got[2], 1)
    assert np.array_equal(got[4], [[77, -1, -1]] * 2) and got[3][0][0] == 0 and (got[3][:, 1:] == -np.inf).all()


GRAD = [  # L, d, V, inv_temp, with entropy
    (1, 8, 1, 1.0, True), (1, 64, 7, 1.0, False), (3, 72, 65, 0.5, True), (17, 136, 1000, 1.25, True),
    (129, 512, 8191, 1.0, True), (257, 64, 300, 2.0, False), (300, 1608, 5001, 1.0, True),
]


def _grads(seed, L):
    r = np.random.default_rng(seed)
    return r.normal(size=L).astype(np.float32), (0.3 * r.normal(size=L)).astype(np.float32)


@pytest.mark.parametrize("L,d,V,inv_temp,ent", GRAD)
def test_gradient(L, d, V, inv_temp, ent):
    """Against the formula, and against differences of the fp64 objective.  Each dz is
    rounded once to bf16 (8 bits: 2^-8 of it at most), dh too; dz itself carries at most 1e-5 of
    its terms from fp32, the sums over the vocabulary 2^-13 of theirs."""
    h, W, tgt = _inputs(L + V + 1, L, d, V)
    a, b = _grads(L, L)
    f = attt.attt_logprob_forward(_bf16(h), _bf16(W), torch.from_numpy(tgt).to(DEV), inv_temp=inv_temp)
    kw = {"entropy": f[1], "gent": torch.from_numpy(b).to(DEV)} if ent else {}
    dh = attt.attt_logprob_input_grad(_bf16(h), _bf16(W), torch.from_numpy(tgt).to(DEV), f[2],
                                      torch.from_numpy(a).to(DEV), inv_temp=inv_temp, **kw)
    assert attt.attt_device_status() == 0 and dh.dtype == torch.bfloat16
    got = dh.float().cpu().numpy()
    want, dz = op.logprobs_grad(h, W, tgt, a, b if ent else None, inv_temp)
    p = np.exp(h @ W.T * inv_temp - op.logprobs(h, W, None, 0, inv_temp)[2][:, None])
    terms = p * (np.abs(a) + np.abs(b) * 10)[:, None] * inv_temp
    slack = ((2.0 ** -8 + 2.0 ** -13) * np.abs(dz) + 1e-5 * terms) @ np.abs(W)
    tol = slack + 2.0 ** -8 * (np.abs(want) + slack) + 1e-7
    # the given token's own term cancels against p there: its parts' rounding, not the difference's
    assert (np.abs(got - want) <= tol + 2.0 ** -20 * np.abs(a)[:, None]).all()

    def J(x):
        lp, H, *_ = op.logprobs(x, W, tgt, 0, inv_temp)
        return (a * lp).sum() + ((b * H).sum() if ent else 0.0)

    u = np.random.default_rng(9).normal(size=h.shape)
    e = 1e-5
    slope = (J(h + e * u) - J(h - e * u)) / (2 * e)
    # central differences: e^2 of the third derivative and 1e-16 |J| / e, both below 1e-6 of the terms
    bound = (tol * np.abs(u)).sum() + 1e-6 * (np.abs(a).sum() + np.abs(b).sum()) * np.sqrt(d)
    assert abs((got * u).sum() - slope) <= bound


@pytest.mark.parametrize("L,d,V,inv_temp", [(1, 64, 4000, 1.25), (3, 1032, 9100, 1.0), (33, 520, 2001, 2.0),
                                            (64, 136, 5000, 1.0)])
def test_gradient_of_few_rows_keeps_the_block(L, d, V, inv_temp):
    """Up to 64 rows take their dz in two bf16 (2^-16 of each value): dh is off by its own
    rounding (2^-8 of it) and by fp32 arithmetic alone."""
    h, W, tgt = _inputs(L + V, L, d, V)
    a, b = _grads(L, L)
    f = attt.attt_logprob_forward(_bf16(h), _bf16(W), torch.from_numpy(tgt).to(DEV), inv_temp=inv_temp)
    dh = attt.attt_logprob_input_grad(_bf16(h), _bf16(W), torch.from_numpy(tgt).to(DEV), f[2],
                                      torch.from_numpy(a).to(DEV), f[1], torch.from_numpy(b).to(DEV), inv_temp)
    want, dz = op.logprobs_grad(h, W, tgt, a, b, inv_temp)
    p = np.exp(h @ W.T * inv_temp - op.logprobs(h, W, None, 0, inv_temp)[2][:, None])
    terms = p * (np.abs(a) + np.abs(b) * 10)[:, None] * inv_temp
    slack = ((2.0 ** -16 + 2.0 ** -13) * np.abs(dz) + 1e-5 * terms) @ np.abs(W) + 2.0 ** -20 * np.abs(a)[:, None]
    err = np.abs(dh.float().cpu().numpy() - want)
    assert (err <= 2.0 ** -8 * (np.abs(want) + slack) + slack + 1e-7).all()


@pytest.mark.parametrize("L,d,V", [(1, 64, 4000), (40, 1032, 4100), (300, 520, 12000)])
def test_gradient_of_the_given_token_is_not_rounded(L, d, V):
    """Weights halfway between two bf16 values: the given token's own term counts in
    full, and dh is off by its own rounding (2^-8 of it) and by that of the other terms
    (2^-8 of |a| / V |W|, and 1e-5 of their values) alone."""
    h, W, tgt = _inputs(8, L, d, V, peaked=False)
    h[:] = 0
    tgt[:] = np.arange(L) * 7 % V
    a = np.where(np.arange(L) % 2 == 0, 1 + 2.0 ** -8, -1 - 3 * 2.0 ** -8).astype(np.float32)
    f = attt.attt_logprob_forward(_bf16(h), _bf16(W), torch.from_numpy(tgt).to(DEV))
    dh = attt.attt_logprob_input_grad(_bf16(h), _bf16(W), torch.from_numpy(tgt).to(DEV), f[2],
                                      torch.from_numpy(a).to(DEV))
    want, _ = op.logprobs_grad(h, W, tgt, a, None, 1.0)
    rest = np.abs(a)[:, None] / V * np.abs(W).sum(0)[None] * (2.0 ** -8 + 1e-5)
    err = np.abs(dh.float().cpu().numpy() - want)
    # 2^-17: the loss of the given token's term is itself an fp32 difference
    assert (err <= 2.0 ** -8 * (np.abs(want) + rest) + rest + 2.0 ** -17 * np.abs(a[:, None] * W[tgt])).all()


def test_gradient_rows_without_a_token_or_weight():
    h, W, tgt = _inputs(11, 40, 64, 900)
    a, b = _grads(2, 40)
    tgt[:] = -1
    f = attt.attt_logprob_forward(_bf16(h), _bf16(W), torch.from_numpy(tgt).to(DEV))
    dh = attt.attt_logprob_input_grad(_bf16(h), _bf16(W), torch.from_numpy(tgt).to(DEV), f[2],
                                      torch.full((40,), float("nan"), device=DEV))
    assert not dh.float().abs().max().item()


def test_gradient_row_blocks():
    """More rows than one block of the gradient (2 GB) holds."""
    L, d, V = 9000, 16, 131072
    g = torch.Generator(device=DEV).manual_seed(4)
    h = (torch.randn(L, d, generator=g, device=DEV) * 8).round().clamp(-32, 32).div(8).to(torch.bfloat16)
    W = (torch.randn(V, d, generator=g, device=DEV) * 20).round().clamp(-64, 64).div(256).to(torch.bfloat16)
    tgt = torch.randint(-1, V, (L,), generator=g, device=DEV, dtype=torch.int32)
    a = torch.randn(L, generator=g, device=DEV)
    assert attt.attt_logprob_grad_workspace_bytes(L, d, V) < 2300 << 20
    lse = attt.attt_logprob_forward(h, W, tgt)[2]
    whole = attt.attt_logprob_input_grad(h, W, tgt, lse, a).float()
    for lo, hi in ((0, 200), (4400, 4700), (8800, 9000)):
        part = attt.attt_logprob_input_grad(h[lo:hi], W, tgt[lo:hi].contiguous(), lse[lo:hi].contiguous(),
                                            a[lo:hi].contiguous()).float()
        assert (part - whole[lo:hi]).norm() <= 2.0 ** -8 * part.norm()  # sums in another order, rounded to bf16


def test_repeats_and_streams():
    """The same bits each time, on the current stream and on another."""
    h, W, tgt = _inputs(12, 333, 128, 4000)
    hd, Wd, td = _bf16(h), _bf16(W), torch.from_numpy(tgt).to(DEV)
    a = torch.from_numpy(_grads(3, 333)[0]).to(DEV)
    first = attt.attt_logprob_forward(hd, Wd, td, topk=12)
    dh = attt.attt_logprob_input_grad(hd, Wd, td, first[2], a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = attt.attt_logprob_forward(hd, Wd, td, topk=12)
        dh2 = attt.attt_logprob_input_grad(hd, Wd, td, again[2], a)
    third = attt.attt_logprob_forward(hd, Wd, td, topk=12, stream=side)
    torch.cuda.synchronize()
    for x, y, z in zip(first, again, third):
        assert torch.equal(x, y) and torch.equal(x, z)
    assert torch.equal(dh, dh2)


def test_token_out_of_range():
    h, W, tgt = _inputs(13, 10, 64, 100)
    tgt[:] = 5
    tgt[2], tgt[7] = 100, -2
    lp, ent, lse, _, _ = attt.attt_logprob_forward(_bf16(h), _bf16(W), torch.from_numpy(tgt).to(DEV))
    assert attt.attt_device_status() == attt.ATTT_ERR_TOKEN_RANGE
    bad = np.isin(np.arange(10), (2, 7))
    assert np.array_equal(np.isnan(lp.cpu().numpy()), bad) and torch.isfinite(ent).all()
    dh = attt.attt_logprob_input_grad(_bf16(h), _bf16(W), torch.from_numpy(tgt).to(DEV), lse,
                                      torch.ones(10, device=DEV))
    assert attt.attt_device_status() == attt.ATTT_ERR_TOKEN_RANGE
    assert np.array_equal(torch.isnan(dh).any(1).cpu().numpy(), bad)


def test_refusals():
    h, W, tgt = _inputs(14, 10, 64, 100)
    hd, Wd, td = _bf16(h), _bf16(W), torch.from_numpy(tgt).to(DEV)
    f32 = torch.ones(10, device=DEV)
    fwd, grad = attt.attt_logprob_forward, attt.attt_logprob_input_grad
    for args, kw in (((hd, Wd[:, :32], td), {}), ((hd.float(), Wd, td), {}), ((hd, Wd, td.long()), {}),
                     ((hd, Wd, td[:9]), {}), ((hd.t(), Wd, td), {}), ((hd, Wd, td), {"logp": f32[:9]}),
                     ((hd, Wd, td), {"topk": 3, "top_id": torch.zeros(10, 3, device=DEV)}),
                     ((hd, Wd), {"logp": f32})):
        with pytest.raises(ValueError):
            fwd(*args, **kw)
    launches = attt.attt_kernel_launches()
    odd = torch.zeros(10, 63, dtype=torch.bfloat16, device=DEV)
    for args, kw, code in (((hd, Wd, td), {"topk": 21}, attt.ATTT_ERR_INVALID_ARG),
                           ((hd, Wd[:4], td), {"topk": 5}, attt.ATTT_ERR_INVALID_ARG),
                           ((hd, Wd, td), {"topk": -1}, None),
                           ((hd, Wd, td), {"inv_temp": 0.0}, attt.ATTT_ERR_INVALID_ARG),
                           ((hd, Wd, td), {"inv_temp": float("nan")}, attt.ATTT_ERR_INVALID_ARG),
                           ((hd, Wd, td), {"inv_temp": -1.0}, attt.ATTT_ERR_INVALID_ARG),
                           ((odd, odd, td), {}, attt.ATTT_ERR_INVALID_ARG),
                           ((torch.zeros(10, 71, dtype=torch.bfloat16, device=DEV)[:, :64], Wd, td), {},
                            attt.ATTT_ERR_INVALID_ARG),
                           ((hd, Wd, td), {"workspace": torch.empty(256, dtype=torch.uint8, device=DEV)},
                            attt.ATTT_ERR_WORKSPACE)):
        with pytest.raises((attt.AtttError, RuntimeError)) as e:
            fwd(*args, **kw)
        if code is not None:
            assert e.value.code == code
    with pytest.raises(attt.AtttError) as e:
        grad(hd, Wd, td, f32, f32, gent=f32)  # an entropy term without the entropies
    assert e.value.code == attt.ATTT_ERR_INVALID_ARG
    assert attt.attt_kernel_launches() == launches and attt.attt_device_status() == 0

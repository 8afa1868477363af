"""Log probabilities through heads of over 48 MB, whose runs of tiles go to their rows'
boundaries first, and the gradient on pairs of SMs whose last wave is cut into K pieces:
against formulas in 64 bits on the GPU.

Inputs lie on grids (hidden states multiples of 1/8 up to 4, heads of 1/256 up to 1/4),
so that every logit is exact in fp32 in any order of its sum and the ids of the
alternatives have to agree exactly.  What is left is fp32 arithmetic on the logits, as
in test_gpu_logprob.py: 1e-5 (1 + s) for values of size s."""
import pytest
import torch

from paper_2607_03441_gb300 import attt, build
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu
F64 = torch.float64


@pytest.fixture(scope="module", autouse=True)
def _library():
    build.build()


def _inputs(seed, L, d, V):
    g = torch.Generator(device=DEV).manual_seed(seed)
    h = (torch.randn(L, d, generator=g, device=DEV) * 8).round().clamp(-32, 32) / 8
    W = (torch.randn(V, d, generator=g, device=DEV) * 20).round().clamp(-64, 64) / 256
    tgt = torch.randint(0, V, (L,), generator=g, device=DEV, dtype=torch.int32)
    known = torch.arange(0, L, 3, device=DEV)  # some rows know their token
    h[known] = (W[tgt[known].long()] * 320).round().clamp(-32, 32) / 8
    tgt[1::5] = -1
    return h.to(torch.bfloat16), W.to(torch.bfloat16), tgt


def _formulas(h, W, tgt, topk, inv_temp):
    z = h.to(F64) @ W.to(F64).t()
    lp = z * inv_temp
    lse = lp.logsumexp(1)
    lp -= lse[:, None]
    entropy = -(lp.exp() * lp).sum(1)
    # ids in the order of the logit, the lower first among equal ones
    ids = torch.sort(z, dim=1, descending=True, stable=True)[1][:, :topk]
    logp = torch.where(tgt >= 0, lp.gather(1, tgt.long().clamp(min=0)[:, None])[:, 0], 0.0)
    return logp, entropy, lse, lp.gather(1, ids), ids


def _close(got, want, what):
    err = (got.to(F64) - want).abs() / (1 + want.abs())
    assert not err.numel() or err.max().item() <= 1e-5, (what, err.max())


HEADS = [  # L, d, V, topk, inv_temp: 2 d V over 48 MB, more rows than a row of tiles has
    (300, 2048, 13001, 0, 1.0), (600, 2048, 13001, 1, 1.0), (600, 2048, 13001, 8, 0.5), (1500, 2048, 13001, 20, 1.25),
    (700, 1000, 30001, 8, 1.0), (300, 1024, 26000, 20, 1.0), (2400, 1032, 26000, 5, 1.0), (257, 2048, 13000, 3, 1.0),
    (5000, 2048, 13001, 1, 1.0), (1100, 1000, 30001, 0, 1.0),
]


@pytest.mark.parametrize("L,d,V,topk,inv_temp", HEADS)
def test_forward(L, d, V, topk, inv_temp):
    assert 2 * d * V > 48 << 20 and L > 256
    h, W, tgt = _inputs(L + V, L, d, V)
    got = attt.attt_logprob_forward(h, W, tgt, topk=topk, inv_temp=inv_temp)
    assert attt.attt_device_status() == 0
    want = _formulas(h, W, tgt, topk, inv_temp)
    for g, w, what in zip(got, want, ("logp", "entropy", "lse", "top_logp")):
        _close(g, w, what)
    assert torch.equal(got[4].long(), want[4])


@pytest.mark.parametrize("L,topk", [(520, 20), (700, 8), (1300, 1), (2400, 20)])
def test_equal_logits(L, topk):
    """Every logit of a row occurs 80 times, far apart: the lowest ids come first, wherever
    the runs of tiles begin, split and end."""
    V, d = 26000, 1024
    n = -(torch.arange(V, device=DEV) % 325)
    W = torch.zeros(V, d, device=DEV)
    W[:, 0], W[:, 1] = torch.floor(n / 64), n % 64
    h = torch.zeros(L, d, device=DEV)
    h[:, 0], h[:, 1] = 1, 1 / 64
    h[::2] *= -1  # the least ones become the largest
    h, W, tgt = h.to(torch.bfloat16), W.to(torch.bfloat16), torch.full((L,), 5, dtype=torch.int32, device=DEV)
    got = attt.attt_logprob_forward(h, W, tgt, topk=topk)
    want = [t[torch.arange(L, device=DEV) % 2] for t in _formulas(h[:2], W, tgt[:2], topk, 1.0)]
    assert torch.equal(got[4].long(), want[4])
    for g, w, what in zip(got, want, ("logp", "entropy", "lse", "top_logp")):
        _close(g, w, what)


def test_infinite_and_nan_logits():
    """-inf logits take no part, NaN and +inf make their row NaN or infinite without
    touching the others."""
    V, d, L, topk = 26000, 1024, 520, 8
    W = torch.zeros(V, d, device=DEV)
    W[:, 0] = (torch.arange(V, device=DEV) % 7).float()
    minus = torch.tensor([0, 300, 12999, 25999], device=DEV)
    W[minus, 0] = -torch.inf
    h = torch.zeros(L, d, device=DEV)
    h[:, 0] = 1
    h[1::4, 1] = torch.nan
    h[2::4, 0] = -1  # +inf at `minus`
    tgt = torch.full((L,), 13, dtype=torch.int32, device=DEV)
    tgt[4::8] = 300
    lp, ent, lse, top, ids = attt.attt_logprob_forward(h.to(torch.bfloat16), W.to(torch.bfloat16), tgt, topk=topk)
    z = W[:, 0].to(F64)
    p = torch.softmax(z, 0)
    want = torch.logsumexp(z, 0)
    H = -(p[p > 0] * p[p > 0].log()).sum()
    for rows in (slice(0, None, 4), slice(3, None, 4)):
        _close(lse[rows], want.expand_as(lse[rows]), "lse")
        _close(ent[rows], H.expand_as(ent[rows]), "entropy")
        assert (ids[rows].long() == torch.sort(z, descending=True, stable=True)[1][:topk]).all()
    assert (lp[4::8] == -torch.inf).all()
    _close(lp[0::8], (z[13] - want).expand_as(lp[0::8]), "logp")
    assert torch.isnan(torch.stack([lp, ent, lse])[:, 1::4]).all() and (ids[1::4] == -1).all()
    assert torch.isnan(ent[2::4]).all() and not torch.isfinite(lse[2::4]).any()
    assert (ids[2::4, :4].long() == minus).all()


# L, d, V: whole tiles of CTA pairs, and a last wave cut into 2, 3 and 4 pieces
CUT_TAILS = [(1800, 3304, 16001), (2000, 2824, 5003), (2000, 2600, 3001), (2300, 2304, 3001)]


def _gradient_formula(h, W, tgt, a, b, inv_temp):
    lp = h.to(F64) @ W.to(F64).t() * inv_temp
    lp -= lp.logsumexp(1, keepdim=True)
    p = lp.exp()
    H = -(p * lp).sum(1, keepdim=True)
    a = torch.where(tgt >= 0, a, 0.0).to(F64)[:, None]
    dz = -p * (a + b.to(F64)[:, None] * (lp + H))
    dz.scatter_add_(1, tgt.long().clamp(min=0)[:, None], a)
    dz *= inv_temp
    return dz @ W.to(F64), dz, p


@pytest.mark.parametrize("L,d,V", CUT_TAILS)
@pytest.mark.parametrize("inv_temp", [1.0, 1.25])
def test_gradient_of_cut_tails(L, d, V, inv_temp):
    """Each dz is rounded once to bf16 (2^-8 of it at most), dh too; dz itself carries 1e-5 of
    its terms from fp32, the sums over the vocabulary 2^-13 of theirs, the given
    token's parts, which cancel, 2^-20."""
    h, W, tgt = _inputs(L + d, L, d, V)
    g = torch.Generator(device=DEV).manual_seed(L)
    a, b = torch.randn(L, generator=g, device=DEV), 0.3 * torch.randn(L, generator=g, device=DEV)
    f = attt.attt_logprob_forward(h, W, tgt, inv_temp=inv_temp)
    dh = attt.attt_logprob_input_grad(h, W, tgt, f[2], a, f[1], b, inv_temp)
    assert attt.attt_device_status() == 0
    want, dz, p = _gradient_formula(h, W, tgt, a, b, inv_temp)
    terms = p * (a.abs() + b.abs() * 10).to(F64)[:, None] * inv_temp
    slack = ((2.0 ** -8 + 2.0 ** -13) * dz.abs() + 1e-5 * terms) @ W.to(F64).abs() + 2.0 ** -20 * a.abs().to(F64)[:, None]
    err = (dh.to(F64) - want).abs()
    assert (err <= slack + 2.0 ** -8 * (want.abs() + slack) + 1e-7).all()
    # the roundings are independent: their norm is that of 2^-8 of dz through W, and of dh
    spread = (dz.square() @ W.to(F64).square()).sum().sqrt() + want.norm()
    assert err.norm() <= 2.0 ** -8 * spread
    again = attt.attt_logprob_input_grad(h, W, tgt, f[2], a, f[1], b, inv_temp)
    assert torch.equal(dh, again)


@pytest.mark.parametrize("L,d,V", CUT_TAILS)
def test_given_token_of_cut_tails_is_not_rounded(L, d, V):
    """Weights halfway between two bf16 values: the given token's own term counts in full
    after the pieces' sum, and dh is off by its own rounding (2^-8 of it), by that of the
    other terms (2^-8 of |a| / V |W|, and 1e-5 of their values) and by 2^-17 of the
    given token's, whose loss is itself an fp32 difference."""
    _, W, _ = _inputs(1, 4, d, V)
    h = torch.zeros(L, d, dtype=torch.bfloat16, device=DEV)
    tgt = (torch.arange(L, device=DEV) * 7 % V).to(torch.int32)
    a = torch.where(torch.arange(L, device=DEV) % 2 == 0, 1 + 2.0 ** -8, -1 - 3 * 2.0 ** -8)
    f = attt.attt_logprob_forward(h, W, tgt)
    dh = attt.attt_logprob_input_grad(h, W, tgt, f[2], a)
    want, _, _ = _gradient_formula(h, W, tgt, a, torch.zeros_like(a), 1.0)
    rest = a.abs().to(F64)[:, None] / V * W.to(F64).abs().sum(0) * (2.0 ** -8 + 1e-5)
    err = (dh.to(F64) - want).abs()
    own = (a[:, None] * W[tgt.long()].float()).abs().to(F64)
    assert (err <= 2.0 ** -8 * (want.abs() + rest) + rest + 2.0 ** -17 * own).all()

"""Three sets of operators that a program needs which trains an adapter by
policy gradient on its own text, with their plain forms:

  logp       log probabilities of given tokens through the frozen LM head, with
             the entropy and the most probable alternatives
             (attt_logprob_forward): scoring a text, or one token of each of
             some concurrent episodes;
  logp_grad  their gradient with respect to the hidden states
             (attt_logprob_input_grad);
  norm       the layer norm in front of the LM head (attt_layer_norm_forward);
  norm_grad  its gradient, those of its weight and bias among it
             (attt_layer_norm_backward);
  muon       the adapters' step along orthogonalised momentum
             (attt_lora_muon_step).

Where `own` is false, run() computes them from elementary torch operations in
32 bits.  Ranges (draw): 1 to 4,096 rows through heads of 8,192 to 152,064 rows
(norms: up to 8,192 rows), hidden sizes of 512 to 5,120, odd ones among the
norms', bf16 and fp32, ranks 4 to 64, one to seven projections.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-5                              # layer norm
NS = (3.4445, -4.7750, 2.0315)          # Newton-Schulz polynomial a s + b s^3 + c s^5
NS_STEPS, NS_EPS = 5, 1e-7
LR, MOMENTUM, DECAY, RMS = 0.02, 0.95, 0.01, 0.2


def listed():
    return [
        # one token of one episode: the head is read for a single row
        {"name": "logp_token", "kind": "logp", "L": 1, "d": 3584, "V": 152064, "k": 5, "temp": 1.0},
        # one token of each of 16 concurrent episodes, as many alternatives as a server gives
        {"name": "logp_decode", "kind": "logp", "L": 16, "d": 5120, "V": 152064, "k": 20, "temp": 0.7},
        # the text of a few agent steps scored under the policy that wrote it
        {"name": "logp_text", "kind": "logp", "L": 403, "d": 3584, "V": 152064, "k": 0, "temp": 1.0},
        # an update text with its alternatives
        {"name": "logp_7b", "kind": "logp", "L": 2048, "d": 3584, "V": 152064, "k": 8, "temp": 1.0},
        # policy gradient of one short agent text: the head is read for few rows
        {"name": "logp_grad_short", "kind": "logp_grad", "L": 93, "d": 3584, "V": 152064, "temp": 1.0},
        # policy gradient of a long text through the largest head
        {"name": "logp_grad_32b", "kind": "logp_grad", "L": 4096, "d": 5120, "V": 152064, "temp": 0.8},
        # the final norm of one token of each of 16 episodes: latency
        {"name": "norm_token", "kind": "norm", "L": 16, "d": 5120, "bits": 16, "pad": 0, "bias": True},
        # the final norm of a long text
        {"name": "norm_32b", "kind": "norm", "L": 8192, "d": 5120, "bits": 16, "pad": 0, "bias": True},
        # the gradient of an odd-sized norm, rows inside wider ones, fp32
        {"name": "norm_grad_odd", "kind": "norm_grad", "L": 211, "d": 3577, "bits": 32, "pad": 7, "bias": True},
        # the gradient of the final norm of a long text
        {"name": "norm_grad_32b", "kind": "norm_grad", "L": 8192, "d": 5120, "bits": 16, "pad": 0, "bias": True},
        # the step of q and v of the 7B-class update
        {"name": "muon_7b_qv", "kind": "muon", "dins": "3584,3584", "douts": "3584,512", "r": 16},
        # the step of q, k, v and o of the 32B-class update
        {"name": "muon_32b_qkvo", "kind": "muon", "dins": "5120,5120,5120,5120", "douts": "5120,1024,1024,5120",
         "r": 64},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo=512, hi=5120):
    """A hidden size: any multiple of 8."""
    return 8 * _log_int(rng, lo // 8, hi // 8)


def draw(rng):
    kind = rng.choice(["logp", "logp", "logp_grad", "norm", "norm_grad", "muon"])
    if kind in ("logp", "logp_grad"):
        case = {"kind": kind, "L": _log_int(rng, 1, 4096), "d": _width(rng), "V": _log_int(rng, 8192, 152064),
                "temp": rng.choice([0.6, 0.8, 1.0, 1.3])}
        if kind == "logp":
            case["k"] = rng.choice([0, 1, 3, 5, 8, 12, 20])
        return case
    if kind in ("norm", "norm_grad"):
        d = _log_int(rng, 512, 5120) if rng.random() < 0.4 else _width(rng)
        return {"kind": kind, "L": _log_int(rng, 1, 8192), "d": d, "bits": rng.choice([16, 16, 32]),
                "pad": rng.choice([0, 0, 8, 64, 3]), "bias": rng.random() < 0.7}
    n = rng.randint(1, 7)
    dins, douts = ([_width(rng) for _ in range(n)] for _ in range(2))
    return {"kind": kind, "dins": ",".join(map(str, dins)), "douts": ",".join(map(str, douts)),
            "r": rng.choice([4, 8, 12, 16, 24, 32, 64])}


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

class _Rng:
    """Seeded draws on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(int(seed))

    def normal(self, *shape, std=1.0):
        return torch.randn(shape, generator=self.g, device=DEV) * std

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.g, device=DEV)

    def zipf(self, n, V):
        """Token ids of truncated Zipf(1.1), low ids the frequent ones."""
        cdf = torch.arange(1, V + 1, device=DEV, dtype=torch.float64).pow_(-1.1).cumsum_(0)
        return torch.searchsorted(cdf, self.uniform(n).double() * cdf[-1]).clamp_(max=V - 1).to(torch.int32)


def _grid(x, step):
    """bf16 multiples of `step`.  Hidden states on a grid of 1/32 and heads on one
    of 1/2048 (std 0.02 is 41 of them, as in a head quantised to 8 bits) have
    logits that are exact in fp32 whatever the order of their sums, so that
    the ids of the alternatives, ties among them, do not depend on that order."""
    return x.mul_(1 / step).round_().mul_(step).to(torch.bfloat16)


def _head(rng, V, d):
    W = torch.empty(V, d, dtype=torch.bfloat16, device=DEV)
    for a in range(0, V, 16384):
        W[a:a + 16384] = _grid(rng.normal(min(16384, V - a), d, std=0.02), 1 / 2048)
    return W


def _states(rng, W, tgt):
    """Hidden states of a model that knows some of the text: N(0, 1) plus shares of
    the target's and of another token's head row, so that their logits lie up
    to 16 above the rest (probabilities from 0 to nearly 1)."""
    L, d = tgt.numel(), W.shape[1]
    h = rng.normal(L, d)
    for t in (tgt.long(), rng.zipf(L, W.shape[0]).long()):
        h += rng.uniform(L, 1) * (16 / (0.02 ** 2 * d)) * W[t].float()
    return _grid(h, 1 / 32)


def _rows(x, pad, dtype):
    """x as rows of a wider buffer, `pad` values further apart than they are long."""
    L, d = x.shape
    buf = torch.zeros(L, d + pad, dtype=dtype, device=DEV)
    buf[:, :d] = x
    return buf[:, :d]


def prepare(case, seed):
    rng, s = _Rng(seed), dict(case)
    kind = case["kind"]
    if kind in ("logp", "logp_grad"):
        L, d, V = case["L"], case["d"], case["V"]
        s["W"] = _head(rng, V, d)
        tgt = rng.zipf(L, V)
        s["h"] = _states(rng, s["W"], tgt)
        if kind == "logp_grad":
            # a twentieth of the rows are another speaker's, without a token to learn
            s["tgt"] = torch.where(rng.uniform(L) < 0.05, torch.full_like(tgt, -1), tgt)
            s["glogp"] = rng.normal(L) / L            # advantages over the text's length
            s["gent"] = torch.full((L,), 0.01 / L, device=DEV) * (0.5 + rng.uniform(L))
            z = s["h"].float() @ s["W"].float().t()   # lse and entropy as the forward call left them
            z *= 1 / case["temp"]
            s["lse"] = z.logsumexp(1)
            z -= s["lse"][:, None]
            s["entropy"] = -(z * z.exp()).sum(1)
        else:
            s["tgt"] = tgt
    elif kind in ("norm", "norm_grad"):
        L, d = case["L"], case["d"]
        dtype = torch.bfloat16 if case["bits"] == 16 else torch.float32
        # a residual stream: columns of different spread, some of them far out, and rows off zero
        spread = torch.exp(rng.normal(d)) * (1 + 20 * (rng.uniform(d) < 0.002))
        s["x"] = _rows(rng.normal(L, d) * spread + rng.normal(L, 1), case["pad"], dtype)
        s["gamma"] = 1 + rng.normal(d, std=0.1)
        s["beta"] = rng.normal(d, std=0.1) if case["bias"] else None
        if kind == "norm_grad":
            s["dy"] = _rows(rng.normal(L, d, std=1e-3), case["pad"], dtype)
            x = s["x"].float()
            s["mean"] = x.mean(1)
            s["rstd"] = torch.rsqrt((x - s["mean"][:, None]).square().mean(1) + EPS)
    else:
        r = case["r"]
        for key in ("A32s", "dAs", "mAs", "B32s", "dBs", "mBs"):
            s[key] = []
        # singular values of a gradient fall off: over the rank's directions by a factor of 100
        fall = torch.exp(torch.linspace(0, -math.log(100.0), r, device=DEV))
        for din, dout in _widths(case):
            mix = rng.normal(2, r, r) / math.sqrt(r)
            s["A32s"].append(rng.normal(din, r, std=0.02))
            s["B32s"].append(rng.normal(r, dout, std=0.01))
            s["dAs"].append((rng.normal(din, r) * fall) @ mix[0] * 1e-3)
            s["dBs"].append((mix[1] @ (fall[:, None] * rng.normal(r, dout))) * 1e-3)
            s["mAs"].append(4 * s["dAs"][-1] + rng.normal(din, r, std=1e-4))
            s["mBs"].append(4 * s["dBs"][-1] + rng.normal(r, dout, std=1e-4))
        s["A16s"] = [a.to(torch.bfloat16) for a in s["A32s"]]
        s["B16s"] = [b.to(torch.bfloat16) for b in s["B32s"]]
    return s


def _widths(case):
    return list(zip(*([int(v) for v in case[key].split(",")] for key in ("dins", "douts"))))


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------

def run(s):
    return (_calls if own else _plain)[s["kind"]](s)


def _plain_logp(s):
    z = s["h"].float() @ s["W"].float().t()
    zt = z * (1 / s["temp"])
    top = zt.amax(1, keepdim=True)
    e = (zt - top).exp()
    total = e.sum(1, keepdim=True)
    lse = top + total.log()
    entropy = total.log() - (e * (zt - top)).sum(1, keepdim=True) / total
    logp = zt.gather(1, s["tgt"].long()[:, None]) - lse
    ids = []
    for _ in range(s["k"]):  # the largest logits, the lowest id among equal ones
        ids.append(z.max(1, keepdim=True)[1])
        z.scatter_(1, ids[-1], -math.inf)
    ids = torch.cat(ids, 1) if ids else torch.empty(z.shape[0], 0, dtype=torch.int64, device=z.device)
    return {"logp": logp[:, 0], "entropy": entropy[:, 0], "lse": lse[:, 0], "top_logp": zt.gather(1, ids) - lse,
            "top_id": ids.int()}


def _plain_logp_grad(s):
    W = s["W"].float()
    logp = (s["h"].float() @ W.t()) * (1 / s["temp"]) - s["lse"][:, None]
    given = s["tgt"] >= 0
    a = torch.where(given, s["glogp"], 0.0)[:, None]
    dz = -logp.exp() * (a + s["gent"][:, None] * (logp + s["entropy"][:, None]))
    dz.scatter_add_(1, s["tgt"].long().clamp(min=0)[:, None], a)
    return {"dh": ((dz * (1 / s["temp"])) @ W).to(torch.bfloat16)}


def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    c = x - mean
    rstd = torch.rsqrt((c * c).mean(1, keepdim=True) + EPS)
    y = c * rstd * s["gamma"]
    if s["beta"] is not None:
        y = y + s["beta"]
    return {"y": y.to(s["x"].dtype), "mean": mean[:, 0], "rstd": rstd[:, 0]}


def _plain_norm_grad(s):
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    xh = (s["x"].float() - s["mean"][:, None]) * rstd
    g = dy * s["gamma"]
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return {"dx": dx.to(s["x"].dtype), "dgamma": (dy * xh).sum(0), "dbeta": dy.sum(0) if s["bias"] else None}


def _plain_muon_one(p, g, m, p16):
    """One matrix in place: momentum, Newton-Schulz on the side of the fewer rows, the step."""
    m.mul_(MOMENTUM).add_(g)
    u = g + MOMENTUM * m
    x = u / (u.square().sum().sqrt() + NS_EPS)
    x = x.t() if x.shape[0] > x.shape[1] else x
    for _ in range(NS_STEPS):
        q = x @ x.t()
        x = NS[0] * x + (NS[1] * q + NS[2] * (q @ q)) @ x
    x = x.t() if x.shape != p.shape else x
    p.mul_(1 - LR * DECAY).sub_(LR * RMS * math.sqrt(max(p.shape)) * x)
    p16.copy_(p)


def _plain_muon(s):
    for a, b in (("A32s", "dAs"), ("B32s", "dBs")):
        side = a[0]
        for p, g, m, p16 in zip(s[a], s[b], s["m" + side + "s"], s[side + "16s"]):
            _plain_muon_one(p, g, m, p16)
    return {key: s[key] for key in ("A32s", "B32s", "mAs", "mBs", "A16s", "B16s")}


_plain = {"logp": _plain_logp, "logp_grad": _plain_logp_grad, "norm": _plain_norm, "norm_grad": _plain_norm_grad,
          "muon": _plain_muon}


def _kept(s, key, make):
    """Buffers that a program keeps from call to call: made at the first."""
    if key not in s:
        s[key] = make()
    return s[key]


def _bytes(n):
    return torch.empty(n, dtype=torch.uint8, device=DEV)


def _f32(*shape):
    return torch.empty(shape, dtype=torch.float32, device=DEV)


def _call_logp(s):
    from paper_2607_03441_gb300 import attt
    L, k = s["L"], s["k"]
    ws = _kept(s, "ws", lambda: _bytes(attt.attt_logprob_workspace_bytes(L, s["d"], s["V"], k)))
    out = _kept(s, "out", lambda: {"logp": _f32(L), "entropy": _f32(L), "lse": _f32(L), "top_logp": _f32(L, k),
                                   "top_id": torch.empty(L, k, dtype=torch.int32, device=DEV)})
    attt.attt_logprob_forward(s["h"], s["W"], s["tgt"], topk=k, inv_temp=1 / s["temp"], workspace=ws, **out)
    return out


def _call_logp_grad(s):
    from paper_2607_03441_gb300 import attt
    ws = _kept(s, "ws", lambda: _bytes(attt.attt_logprob_grad_workspace_bytes(s["L"], s["d"], s["V"])))
    dh = _kept(s, "dh", lambda: torch.empty_like(s["h"]))
    attt.attt_logprob_input_grad(s["h"], s["W"], s["tgt"], s["lse"], s["glogp"], entropy=s["entropy"], gent=s["gent"],
                                 inv_temp=1 / s["temp"], dh=dh, workspace=ws)
    return {"dh": dh}


def _call_norm(s):
    from paper_2607_03441_gb300 import attt
    out = _kept(s, "out", lambda: {"y": torch.empty(s["L"], s["d"], dtype=s["x"].dtype, device=DEV),
                                   "mean": _f32(s["L"]), "rstd": _f32(s["L"])})
    attt.attt_layer_norm_forward(s["x"], s["gamma"], s["beta"], eps=EPS, **out)
    return out


def _call_norm_grad(s):
    from paper_2607_03441_gb300 import attt
    ws = _kept(s, "ws", lambda: _bytes(attt.attt_layer_norm_workspace_bytes(s["L"], s["d"])))
    out = _kept(s, "out", lambda: {"dx": torch.empty(s["L"], s["d"], dtype=s["x"].dtype, device=DEV),
                                   "dgamma": _f32(s["d"]), "dbeta": _f32(s["d"]) if s["bias"] else None})
    attt.attt_layer_norm_backward(s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"], workspace=ws, **out)
    return out


def _call_muon(s):
    from paper_2607_03441_gb300 import attt
    ws = _kept(s, "ws", lambda: _bytes(attt.attt_lora_muon_workspace_bytes(*zip(*_widths(s)), s["r"])))
    attt.attt_lora_muon_step(s["A32s"], s["B32s"], s["dAs"], s["dBs"], s["mAs"], s["mBs"], LR, momentum=MOMENTUM,
                             weight_decay=DECAY, rms=RMS, eps=NS_EPS, ns_steps=NS_STEPS, A16s=s["A16s"],
                             B16s=s["B16s"], workspace=ws)
    return {key: s[key] for key in ("A32s", "B32s", "mAs", "mBs", "A16s", "B16s")}


_calls = {"logp": _call_logp, "logp_grad": _call_logp_grad, "norm": _call_norm, "norm_grad": _call_norm_grad,
          "muon": _call_muon}


# --------------------------------------------------------------------------
# floors and 64-bit values
# --------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "logp":
        L, d, V, k = case["L"], case["d"], case["V"], case["k"]
        return {"bytes": 2 * (V * d + L * d) + L * (4 + 12 + 8 * k), "flops": 2 * L * d * V}
    if kind == "logp_grad":  # the logits are not kept, so they are formed again
        L, d, V = case["L"], case["d"], case["V"]
        return {"bytes": 2 * (V * d + 2 * L * d) + 20 * L, "flops": 4 * L * d * V}
    if kind == "norm":
        L, d, e = case["L"], case["d"], case["bits"] // 8
        return {"bytes": 2 * e * L * d + 8 * L + 4 * d * (2 if case["bias"] else 1), "flops": 8 * L * d}
    if kind == "norm_grad":
        L, d, e = case["L"], case["d"], case["bits"] // 8
        return {"bytes": 3 * e * L * d + 8 * L + 4 * d * (3 if case["bias"] else 2), "flops": 14 * L * d}
    r = case["r"]
    n = [w for pair in _widths(case) for w in pair]
    # g, m and p are read, m, p and the bf16 copy written; the Gram matrix, its polynomial (17 products), the product
    return {"bytes": sum(22 * r * w for w in n), "flops": sum(4 * r * r * w + 17 * 2 * r ** 3 for w in n)}


def exact(case, seed):
    s = prepare(case, seed)
    return _exact[case["kind"]](s)


def _logits64(s):
    return torch.matmul(s["h"].double(), s["W"].double().T)


def _exact_logp(s):
    z = _logits64(s)
    logp = torch.log_softmax(z / s["temp"], -1)
    entropy = torch.special.entr(logp.exp()).sum(-1)
    lse = torch.logsumexp(z / s["temp"], -1)
    rows = torch.arange(s["L"], device=DEV)
    order = torch.empty(s["L"], 0, dtype=torch.int64, device=DEV)
    if s["k"]:  # every id whose logit is among the k largest values, in order of value and then of id
        least = torch.topk(z, s["k"], -1)[0][:, -1:]
        order = torch.stack([_first(row, lo, s["k"]) for row, lo in zip(z, least)])
    return {"logp": logp[rows, s["tgt"].long()], "entropy": entropy, "lse": lse, "top_logp": logp.gather(1, order),
            "top_id": order.int()}


def _first(row, least, k):
    at = torch.nonzero(row >= least)[:, 0]  # ascending
    return at[torch.sort(row[at], descending=True, stable=True)[1][:k]]


def _exact_logp_grad(s):
    """d/dz of sum_j a_j logp_j + b_j H_j, the entropy's part from -sum p log p; lse and
    entropy are inputs, as for the call."""
    W = s["W"].double()
    z = torch.matmul(s["h"].double(), W.T) / s["temp"]
    p = torch.exp(z - s["lse"].double().unsqueeze(-1))
    a = s["glogp"].double().masked_fill(s["tgt"] < 0, 0)
    b = s["gent"].double()
    hit = torch.nn.functional.one_hot(s["tgt"].long().clamp_min(0), 1 + int(s["tgt"].max().clamp_min(0)))
    dz = p * (z - s["lse"].double().unsqueeze(-1) + s["entropy"].double().unsqueeze(-1)) * -b.unsqueeze(-1)
    dz -= a.unsqueeze(-1) * p
    dz[:, :hit.shape[1]] += a.unsqueeze(-1) * hit
    return {"dh": torch.matmul(dz, W) / s["temp"]}


def _exact_norm(s):
    x = s["x"].double()
    var, mean = torch.var_mean(x, -1, correction=0)
    rstd = (var + EPS) ** -0.5
    y = torch.einsum("ld,l,d->ld", x - mean.unsqueeze(-1), rstd, s["gamma"].double())
    if s["beta"] is not None:
        y += s["beta"].double()
    return {"y": y, "mean": mean, "rstd": rstd}


def _exact_norm_grad(s):
    """Through the statistics' own derivatives: dy -> (mean, rstd) -> x."""
    x, dy, gamma = (s[key].double() for key in ("x", "dy", "gamma"))
    mean, rstd = s["mean"].double().unsqueeze(-1), s["rstd"].double().unsqueeze(-1)
    c, d = x - mean, x.shape[1]
    g = dy * gamma
    d_rstd = (g * c).sum(-1, keepdim=True)
    d_var = -0.5 * d_rstd * rstd ** 3
    d_mean = -(g.sum(-1, keepdim=True) * rstd)
    return {"dx": g * rstd + 2 / d * d_var * c + d_mean / d, "dgamma": torch.einsum("ld,ld,l->d", dy, c, rstd[:, 0]),
            "dbeta": dy.sum(0) if s["bias"] else None}


def _exact_muon(s):
    """The polynomial on the singular values: u = P S Q^T, o = P f(...f(S / (|S| + eps))) Q^T."""
    out = {}
    for side in "AB":
        ps, ms = [], []
        for p, g, m in zip(s[side + "32s"], s["d" + side + "s"], s["m" + side + "s"]):
            p, g, m = p.double(), g.double(), m.double()
            m = MOMENTUM * m + g
            left, sv, right = torch.linalg.svd(g + MOMENTUM * m, full_matrices=False)
            sv = sv / (torch.linalg.vector_norm(sv) + NS_EPS)
            for _ in range(NS_STEPS):
                sv = NS[0] * sv + NS[1] * sv ** 3 + NS[2] * sv ** 5
            o = torch.matmul(left * sv, right)
            ps.append(p - LR * DECAY * p - LR * RMS * max(p.shape) ** 0.5 * o)
            ms.append(m)
        out.update({side + "32s": ps, "m" + side + "s": ms, side + "16s": ps})
    return out


_exact = {"logp": _exact_logp, "logp_grad": _exact_logp_grad, "norm": _exact_norm, "norm_grad": _exact_norm_grad,
          "muon": _exact_muon}

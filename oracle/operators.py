"""Plain fp64 numpy forms of the policy-gradient operators -- TEST
INFRASTRUCTURE ONLY (as the rest of this package).

bf16 inputs are taken as float arrays of their values.
"""
import math

import numpy as np

# Newton-Schulz polynomial f(s) = a s + b s^3 + c s^5 (K. Jordan et al., "Muon: an
# optimizer for hidden layers in neural networks", 2024)
NS = (3.4445, -4.7750, 2.0315)


def _f64(*arrays):
    return [np.asarray(a, dtype=np.float64) for a in arrays]


def logprobs(h, W, tgt=None, topk=0, inv_temp=1.0):
    """(logp [L] or None, entropy [L], lse [L], top_logp [L, topk], top_id [L, topk])."""
    h, W = _f64(h, W)
    z = h @ W.T
    zt = z * inv_temp
    top = zt.max(1, keepdims=True)
    lse = (top + np.log(np.exp(zt - top).sum(1, keepdims=True)))[:, 0]
    lp = zt - lse[:, None]
    with np.errstate(invalid="ignore"):
        entropy = -np.where(np.exp(lp) > 0, np.exp(lp) * lp, 0.0).sum(1)
    ids = np.argsort(-z, axis=1, kind="stable")[:, :topk]
    top_lp = np.take_along_axis(lp, ids, 1)
    if tgt is None:
        return None, entropy, lse, top_lp, ids
    tgt = np.asarray(tgt)
    logp = np.where(tgt >= 0, lp[np.arange(len(tgt)), np.maximum(tgt, 0)], 0.0)
    return logp, entropy, lse, top_lp, ids


def logprobs_grad(h, W, tgt, glogp, gent=None, inv_temp=1.0):
    """(dh, dz): the gradient of sum_j glogp_j logp_j + gent_j H_j with respect to h
    and to the logits."""
    h, W, glogp = _f64(h, W, glogp)
    tgt = np.asarray(tgt)
    _, H, lse, _, _ = logprobs(h, W, None, 0, inv_temp)
    lp = (h @ W.T) * inv_temp - lse[:, None]
    a = np.where(tgt >= 0, glogp, 0.0)
    b = np.zeros_like(a) if gent is None else np.asarray(gent, dtype=np.float64)
    dz = -np.exp(lp) * (a[:, None] + b[:, None] * (lp + H[:, None]))
    rows = np.nonzero(tgt >= 0)[0]
    dz[rows, tgt[rows]] += a[rows]
    dz *= inv_temp
    return dz @ W, dz


def layer_norm(x, gamma, beta=None, eps=1e-5):
    """(y, mean, rstd)."""
    x, gamma = _f64(x, gamma)
    mean = x.mean(1)
    c = x - mean[:, None]
    rstd = 1.0 / np.sqrt((c * c).mean(1) + eps)
    y = c * rstd[:, None] * gamma
    return (y if beta is None else y + np.asarray(beta, dtype=np.float64)), mean, rstd


def layer_norm_grad(dy, x, gamma, mean, rstd):
    """(dx, dgamma, dbeta) for the statistics given."""
    dy, x, gamma, mean, rstd = _f64(dy, x, gamma, mean, rstd)
    xh = (x - mean[:, None]) * rstd[:, None]
    g = dy * gamma
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def newton_schulz(u, eps=1e-7, steps=5):
    """`steps` Newton-Schulz products on u / (|u|_F + eps)."""
    x, = _f64(u)
    x = x / (np.sqrt((x * x).sum()) + eps)
    flip = x.shape[0] > x.shape[1]
    x = x.T if flip else x
    for _ in range(steps):
        q = x @ x.T
        x = NS[0] * x + (NS[1] * q + NS[2] * (q @ q)) @ x
    return x.T if flip else x


def muon_step(p, g, m, lr, momentum=0.95, nesterov=True, weight_decay=0.0, rms=0.2, eps=1e-7, steps=5):
    """(p, m) after one step."""
    p, g, m = _f64(p, g, m)
    m = momentum * m + g
    u = g + momentum * m if nesterov else m
    o = newton_schulz(u, eps, steps)
    return p * (1 - lr * weight_decay) - lr * rms * math.sqrt(max(p.shape)) * o, m

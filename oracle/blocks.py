"""Plain numpy forms of the operators inside an adapted block -- TEST
INFRASTRUCTURE ONLY (as the rest of this package).  fp64 but for the AdamW step,
which is fp32 operation by operation, as the call is documented.

bf16 inputs are taken as float arrays of their values.
"""
import math

import numpy as np


# --------------------------------------------------------------------------
# norm of the heads and position rotation
# --------------------------------------------------------------------------

def rope_frequencies(rot, base=10000.0, factor=1.0, context=0.0, low=1.0, high=32.0, by_index=False):
    """Radians per position of each pair."""
    w = base ** (-2.0 * np.arange(rot // 2) / rot)
    if factor == 1.0:
        return w
    if context == 0.0:
        return w / factor
    turns = context * w / (2 * math.pi)
    keep = np.clip((turns - low) / (high - low), 0, 1)
    if by_index:  # log(turns) falls by ln(base) / (rot / 2) from pair to pair
        first, last = (np.log(turns[0] / n) / np.log(base) * rot / 2 for n in (high, low))
        keep = np.interp(np.arange(rot // 2), [max(0, math.floor(first)), min(rot - 1, math.ceil(last))], [1, 0])
    return w * keep + w / factor * (1 - keep)


def _members(rot, interleaved):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def rotate(x, pos, w, interleaved=False, mscale=1.0, back=False):
    """x [T, H, D] with its first 2 len(w) values turned (back: the transpose)."""
    x = np.array(x, dtype=np.float64)
    angle = np.asarray(pos, dtype=np.float64)[:, None] * w
    c, s = np.cos(angle)[:, None] * mscale, np.sin(angle)[:, None] * mscale * (-1 if back else 1)
    a, b = _members(2 * len(w), interleaved)
    va, vb = x[..., a].copy(), x[..., b].copy()
    x[..., a], x[..., b] = va * c - vb * s, va * s + vb * c
    return x


def rope(x, pos, w, gamma=None, eps=1e-6, interleaved=False, mscale=1.0):
    x = np.asarray(x, dtype=np.float64)
    if gamma is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(gamma, dtype=np.float64)
    return rotate(x, pos, w, interleaved, mscale)


def rope_grad(dy, x, pos, w, gamma=None, eps=1e-6, interleaved=False, mscale=1.0):
    """(dx, dgamma or None)."""
    dz = rotate(dy, pos, w, interleaved, mscale, back=True)
    if gamma is None:
        return dz, None
    x, gamma = np.asarray(x, dtype=np.float64), np.asarray(gamma, dtype=np.float64)
    rstd = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    xh, g = x * rstd, dz * gamma
    return rstd * (g - xh * (g * xh).mean(-1, keepdims=True)), (dz * xh).sum((0, 1))


# --------------------------------------------------------------------------
# the gated feed-forward block
# --------------------------------------------------------------------------

def activation(g, act):
    """(act(g), act'(g))."""
    g = np.asarray(g, dtype=np.float64)
    if act == "silu":
        p = 1 / (1 + np.exp(-g))
        return g * p, p * (1 + g * (1 - p))
    c = math.sqrt(2 / math.pi)
    t = np.tanh(c * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def project(x, W, A=None, B=None, scale=1.0):
    """x W + s (x A) B."""
    return x @ W if A is None else x @ W + scale * ((x @ A) @ B)


def gated_ffn(x, Wg, Wu, Wd, As=(None,) * 3, Bs=(None,) * 3, scale=1.0, act="silu"):
    """(y, h, g, u)."""
    g, u = project(x, Wg, As[0], Bs[0], scale), project(x, Wu, As[1], Bs[1], scale)
    h = activation(g, act)[0] * u
    return project(h, Wd, As[2], Bs[2], scale), h, g, u


def _t(M):
    return None if M is None else M.T


def gated_ffn_grad(dy, Wg, Wu, Wd, g, u, As=(None,) * 3, Bs=(None,) * 3, scale=1.0, act="silu"):
    """(dx, dg, du)."""
    dh = project(dy, Wd.T, _t(Bs[2]), _t(As[2]), scale)
    a, slope = activation(g, act)
    dg, du = dh * u * slope, dh * a
    dx = project(dg, Wg.T, _t(Bs[0]), _t(As[0]), scale) + project(du, Wu.T, _t(Bs[1]), _t(As[1]), scale)
    return dx, dg, du


# --------------------------------------------------------------------------
# AdamW with moments in 8 bits
# --------------------------------------------------------------------------

BLOCK = 256


def mix(x):
    """The hash of 32-bit numbers that the random bits come from."""
    x = np.asarray(x, dtype=np.uint32)
    x = x ^ (x >> np.uint32(16))
    x = x * np.uint32(0xB504F333)
    x = x ^ (x >> np.uint32(15))
    x = x * np.uint32(0xDDB3D743)
    return x ^ (x >> np.uint32(16))


def random_bits(n, tensor, seed):
    with np.errstate(over="ignore"):
        key = mix(np.uint32(seed & 0xFFFFFFFF) ^ mix(np.uint32(seed >> 32) ^ mix(np.uint32(tensor + 1))))
        return mix(np.arange(n, dtype=np.uint32) + mix(key))


def code_values(mant):
    """The value of each code without a sign."""
    c = np.arange(16 << mant)
    e, low = c >> mant, c & ((1 << mant) - 1)
    return np.where(e > 0, (1 + low / 2.0 ** mant) * 2.0 ** (e - 15.0), low * 2.0 ** (-14 - mant))


def _scale(x, mant):
    """(scale, inverse) of a block of sizes."""
    top = np.float32(np.max(x)) if not np.isnan(x).any() else np.float32(np.nan)
    if not np.isfinite(top):
        return np.float32(np.nan), np.float32(0)
    if top < np.float32(2.0 ** -100):
        return np.float32(0), np.float32(0)
    s = np.float32(top * np.float32(1 / (2 - 2.0 ** -mant)))
    return s, np.float32(np.float32(1) / s)


def quantise(x, mant, rnd, least=0):
    """(codes, scales) of sizes x (fp32 [n]) with 23 - mant random bits each; sizes above 0 get
    the code `least` at least."""
    codes, scales = np.zeros(len(x), np.uint8), []
    values, cut = code_values(mant), 23 - mant
    for b in range(0, len(x), BLOCK):
        v = x[b:b + BLOCK]
        s, inv = _scale(v, mant)
        scales.append(s)
        if inv == 0:
            continue
        a = (v * inv).astype(np.float64)  # fp32 product, exact from here on
        step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(a, 1e-300))), -14) - mant)
        units = np.floor(a / step * 2.0 ** cut) + rnd[b:b + BLOCK]
        up = np.minimum(np.floor(units / 2.0 ** cut) * step, values[-1])
        codes[b:b + BLOCK] = np.maximum(np.searchsorted(values, up), least * (v > 0))
    return codes, np.array(scales, np.float32)


def read_state(m8, v8, ms, vs):
    """(m, v) fp32 of codes and scales."""
    n = len(m8)
    rep = [np.repeat(s, BLOCK)[:n].astype(np.float32) for s in (ms, vs)]
    m = code_values(3)[m8 & 127].astype(np.float32) * rep[0]
    r = code_values(4)[v8].astype(np.float32) * rep[1]
    return np.where(m8 & 128, -m, m).astype(np.float32), (r * r).astype(np.float32)


def adamw(p, g, m, v, lr, b1, b2, eps, wd, t):
    """(p, m, v, sqrt(v)) in fp32, every operation rounded on its own."""
    f = np.float32
    p, g, m, v = (np.asarray(a, dtype=f) for a in (p, g, m, v))
    m = f(b1) * m + f(1 - b1) * g
    v = f(b2) * v + f(1 - b2) * (g * g)
    r = np.sqrt(v)
    denom = r / f(math.sqrt(1 - b2 ** t)) + f(eps)
    return p * f(1 - lr * wd) - (f(lr / (1 - b1 ** t)) * m) / denom, m, v, r


def adamw8(p, g, m8, v8, ms, vs, lr, b1, b2, eps, wd, t, seed, tensor):
    """(p, m8, v8, ms, vs) after a step."""
    p, m, _, r = adamw(p, g, *read_state(m8, v8, ms, vs), lr, b1, b2, eps, wd, t)
    bits = random_bits(len(p), tensor, seed)
    cm, ms = quantise(np.abs(m), 3, (bits & np.uint32(0xFFFF)).astype(np.float64) * 16)
    cv, vs = quantise(r, 4, (bits >> np.uint32(16)).astype(np.float64) * 8, least=1)
    return p, (cm | np.where((m < 0) & (cm > 0), 128, 0)).astype(np.uint8), cv, ms, vs

"""Operators that a program needs which trains adapters inside transformer
blocks, with their plain forms:

  rope       queries and keys between their projections and the attention: the
             norm of every head, where the model has one, and the position
             rotation (attt_rope_forward);
  rope_grad  its gradient, the norms' weights among it (attt_rope_backward);
  ffn        the gated feed-forward block with an adapter on each of its three
             projections (attt_gated_ffn_forward);
  ffn_grad   its gradient with respect to the block's input and to the outputs
             of the gate and up projections, from which the adapters'
             gradients follow (attt_gated_ffn_backward);
  adamw      the AdamW step of all adapters of a model at once, with moments in
             32 bits or in 8 (attt_adamw_create, attt_adamw_step,
             attt_adamw_read_state).

Where `own` is false, run() computes them from elementary torch operations in
32 bits.  Ranges (draw): 1 to 8,192 rows; 1 to 64 heads of 32 to 256 values,
whole or partial rotation in either layout, positions up to 1,048,576; blocks
of 512 to 5,120 by 1,024 to 27,648; ranks 4 to 64; 1 to 512 tensors.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6                                  # norm of a head
BETA1, BETA2, ADAM_EPS, DECAY, LR = 0.9, 0.999, 1e-8, 0.01, 5e-4
BLOCK = 256                                 # values per scale of an 8-bit moment


def listed():
    return [
        # one token of each of 16 concurrent episodes, heads of the 7B-class model: latency
        {"name": "rope_token", "kind": "rope", "T": 16, "hq": 28, "hk": 4, "D": 128, "rot": 128, "inter": False,
         "norm": True, "bits": 16, "pad": 512, "far": 131072, "text": False, "factor": 1.0},
        # a long text, heads of the 32B-class model, q and k inside the rows of one projection
        {"name": "rope_32b", "kind": "rope", "T": 8192, "hq": 40, "hk": 8, "D": 128, "rot": 128, "inter": False,
         "norm": True, "bits": 16, "pad": 1024, "far": 40000, "text": True, "factor": 1.0},
        # part of an odd-sized head turned in pairs of neighbours, fp32, far positions of a stretched context
        {"name": "rope_far", "kind": "rope", "T": 403, "hq": 9, "hk": 3, "D": 80, "rot": 40, "inter": True,
         "norm": False, "bits": 32, "pad": 0, "far": 1048576, "text": True, "factor": 8.0},
        # the gradient through q and k of the 7B-class update
        {"name": "rope_grad_7b", "kind": "rope_grad", "T": 2048, "hq": 28, "hk": 4, "D": 128, "rot": 128,
         "inter": False, "norm": True, "bits": 16, "pad": 512, "far": 40000, "text": True, "factor": 1.0},
        # the gradient at an odd head size, half of it turned
        {"name": "rope_grad_odd", "kind": "rope_grad", "T": 211, "hq": 12, "hk": 2, "D": 90, "rot": 46,
         "inter": False, "norm": True, "bits": 32, "pad": 7, "far": 40000, "text": True, "factor": 4.0},
        # one token of one episode through the block: the weights are read for a single row
        {"name": "ffn_token", "kind": "ffn", "L": 1, "d": 3584, "f": 18944, "r": 0, "act": "silu", "save": False},
        # the text of a few agent steps, seven-projection adapters of the long episode
        {"name": "ffn_text", "kind": "ffn", "L": 403, "d": 4096, "f": 14336, "r": 32, "act": "gelu_tanh",
         "save": False},
        # the 7B-class update, what the gradient needs kept
        {"name": "ffn_7b", "kind": "ffn", "L": 2048, "d": 3584, "f": 18944, "r": 16, "act": "silu", "save": True},
        # the gradient of one short agent text
        {"name": "ffn_grad_short", "kind": "ffn_grad", "L": 93, "d": 3584, "f": 18944, "r": 16, "act": "silu"},
        # the gradient of the 32B-class update, the largest call
        {"name": "ffn_grad_32b", "kind": "ffn_grad", "L": 8192, "d": 5120, "f": 27648, "r": 64, "act": "silu"},
        # the step of q and v of every layer of the 7B-class model
        {"name": "adamw_7b_qv", "kind": "adamw", "layers": 28, "widths": "3584,3584,3584,512", "r": 16, "bits": 32},
        # the step of q, k, v and o of every layer of the 32B-class model, moments in 8 bits, read back for a checkpoint
        {"name": "adamw_32b_8bit", "kind": "adamw", "layers": 64, "widths": "5120,5120,5120,1024,5120,1024,5120,5120",
         "r": 64, "bits": 8},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo=512, hi=5120):
    """Any multiple of 8."""
    return 8 * _log_int(rng, lo // 8, hi // 8)


def draw(rng):
    kind = rng.choice(["rope", "rope", "rope_grad", "ffn", "ffn", "ffn_grad", "adamw", "adamw"])
    if kind in ("rope", "rope_grad"):
        D = rng.choice([64, 80, 96, 128, 128, 256, 2 * rng.randint(16, 128)])
        rot = D if rng.random() < 0.6 else 2 * rng.randint(1, D // 2)
        bits, hq = rng.choice([16, 16, 32]), _log_int(rng, 1, 64)
        hk = rng.randint(1, hq)
        most = 8192 * 48 * 128 * 16 // ((hq + hk) * D * bits)
        return {"kind": kind, "T": _log_int(rng, 1, min(8192, most)), "hq": hq, "hk": hk, "D": D, "rot": rot,
                "inter": rng.random() < 0.4, "norm": rng.random() < 0.7, "bits": bits, "pad": rng.choice([0, 0, D, 8, 3]),
                "far": _log_int(rng, 1, 1 << 20), "text": rng.random() < 0.6, "factor": rng.choice([1.0, 1.0, 4.0, 32.0])}
    if kind in ("ffn", "ffn_grad"):
        case = {"kind": kind, "L": _log_int(rng, 1, 8192), "d": _width(rng), "f": _width(rng, 1024, 27648),
                "r": rng.choice([0, 4, 8, 12, 16, 24, 32, 64]), "act": rng.choice(["silu", "silu", "gelu_tanh"])}
        if kind == "ffn":
            case["save"] = rng.random() < 0.5
        return case
    widths = [_log_int(rng, 64, 5120) for _ in range(rng.choice([1, 2, 4, 7, 8]))]
    r = rng.choice([4, 8, 12, 16, 24, 32, 64])
    return {"kind": kind, "layers": _log_int(rng, 1, 64), "widths": ",".join(map(str, widths)), "r": r,
            "bits": rng.choice([8, 32])}


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

    def bf16(self, rows, cols, std):
        """A matrix of bf16 normals, made in slabs."""
        out = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV)
        for a in range(0, rows, 4096):
            out[a:a + 4096] = self.normal(min(4096, rows - a), cols, std=std)
        return out


def _sizes(case):
    """Values of every adapter matrix of the model: r rows or columns of each width, layer by layer."""
    return [case["r"] * int(w) for w in case["widths"].split(",")] * case["layers"]


def prepare(case, seed):
    rng, s = _Rng(seed), dict(case)
    kind = case["kind"]
    if kind in ("rope", "rope_grad"):
        T, D, hq, hk = case["T"], case["D"], case["hq"], case["hk"]
        dtype = torch.bfloat16 if case["bits"] == 16 else torch.float32
        # one projection's rows: q's heads, k's heads and, as padding, what else it gives (v)
        rows = torch.empty(T, (hq + hk) * D + case["pad"], dtype=dtype, device=DEV)
        rows.copy_(rng.normal(*rows.shape) * torch.exp(rng.normal(rows.shape[1], std=0.5)))
        s["q"] = rows[:, :hq * D].view(T, hq, D)
        s["k"] = rows[:, hq * D:(hq + hk) * D].view(T, hk, D)
        if case["text"]:
            start = int(seed) % 1000 if case["far"] <= T else case["far"] - T
            s["pos"] = torch.arange(start, start + T, dtype=torch.int32, device=DEV)
        else:
            s["pos"] = (rng.uniform(T) * case["far"]).to(torch.int32)
        s["base"] = 1000000.0 if case["norm"] else 10000.0
        s["context"] = 32768 if case["factor"] > 1 else 0
        s["mscale"] = 1.0 if case["factor"] == 1 else 0.1 * math.log(case["factor"]) + 1.0
        s["gq"], s["gk"] = (1 + rng.normal(D, std=0.1) if case["norm"] else None for _ in range(2))
        if kind == "rope_grad":
            s["dq"], s["dk"] = ((rng.normal(T, h, D) * 1e-3).to(dtype) for h in (hq, hk))
    elif kind in ("ffn", "ffn_grad"):
        L, d, f, r = case["L"], case["d"], case["f"], case["r"]
        s["Wg"], s["Wu"], s["Wd"] = rng.bf16(d, f, d ** -0.5), rng.bf16(d, f, d ** -0.5), rng.bf16(f, d, f ** -0.5)
        s["scale"] = 16.0 / r if r else 1.0
        # adapters some steps on from zero: gate, up, down
        s["As"] = [rng.bf16(n, r, 0.02) for n in (d, d, f)] if r else None
        s["Bs"] = [rng.bf16(r, n, 0.01) for n in (f, f, d)] if r else None
        if kind == "ffn":
            s["x"] = rng.bf16(L, d, 1.0)
        else:
            s["dy"] = rng.bf16(L, d, 1e-3)
            s["g"], s["u"] = rng.bf16(L, f, 1.0), rng.bf16(L, f, 1.0)  # as the forward call kept them
    else:
        s["sizes"] = _sizes(case)
        s["blocks"] = [-(-n // BLOCK) for n in s["sizes"]]
        # every tensor starts at a multiple of a block's length in one buffer of the program's
        s["starts"], total = [], 0
        for b in s["blocks"]:
            s["starts"].append(total)
            total += b * BLOCK
        lane = torch.arange(total, device=DEV).view(-1, BLOCK)
        first = torch.tensor(s["starts"], device=DEV).repeat_interleave(torch.tensor(s["blocks"], device=DEV))
        last = torch.tensor([a + n for a, n in zip(s["starts"], s["sizes"])], device=DEV)
        inside = (lane < last.repeat_interleave(torch.tensor(s["blocks"], device=DEV))[:, None]).view(-1)
        del lane, first
        # gradients fall off by rows; some tensors have none yet (the dA of B = 0)
        spread = torch.exp(rng.normal(total // BLOCK, 1)).expand(-1, BLOCK).reshape(-1)
        s["p"] = rng.normal(total, std=0.02).mul_(inside)
        s["g"] = rng.normal(total, std=1e-3).mul_(spread).mul_(inside)
        s["p16"] = s["p"].to(torch.bfloat16)
        if case["bits"] == 32:
            s["m"] = rng.normal(total, std=3e-4).mul_(spread).mul_(inside)
            s["v"] = rng.uniform(total).mul_(2e-6).mul_(spread).mul_(spread).mul_(inside)
        else:
            big = spread.view(-1, BLOCK)[:, 0]
            s["m"] = (torch.minimum(rng.normal(total).abs() * 24 + 72, torch.full((), 127.0, device=DEV)).to(torch.uint8)
                      + 128 * (rng.uniform(total) < 0.5).to(torch.uint8)).mul_(inside)
            s["v"] = torch.minimum(rng.normal(total).abs() * 24 + 180, torch.full((), 255.0, device=DEV)).to(
                torch.uint8).mul_(inside)
            s["ms"], s["vs"] = big * 6e-4, big * 2e-3
        s["step"] = 20
    return s


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------

def run(s):
    return (_calls if own else _plain)[s["kind"]](s)


def _frequencies(s):
    """Radians per position of each pair, 64 bits.  A stretched context leaves pairs alone that
    turn more than 32 times over the original one, divides by the factor those that turn
    less than once, and goes from one to the other between."""
    i = torch.arange(s["rot"] // 2, dtype=torch.float64, device=DEV)
    w = s["base"] ** (-2 * i / s["rot"])
    if s["factor"] > 1:
        keep = ((s["context"] * w / (2 * math.pi) - 1) / (32 - 1)).clamp(0, 1)
        w = w * keep + w / s["factor"] * (1 - keep)
    return w


def _turn(x, cos, sin, rot, inter):
    """Pairs of x's first `rot` values turned by the angle of their token."""
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if inter else (x[..., :rot // 2], x[..., rot // 2:rot])
    cos, sin = cos[:, None], sin[:, None]
    ya, yb = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([ya, yb], -1).flatten(-2) if inter else torch.cat([ya, yb], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _angles(s):
    angle = s["pos"].double()[:, None] * _frequencies(s)
    return (angle.cos() * s["mscale"]).float(), (angle.sin() * s["mscale"]).float()


def _plain_rope(s):
    cos, sin = _angles(s)
    out = {}
    for name in "qk":
        x, gamma = s[name].float(), s["g" + name]
        if gamma is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gamma
        out[name] = _turn(x, cos, sin, s["rot"], s["inter"]).to(s[name].dtype)
    return out


def _plain_rope_grad(s):
    cos, sin = _angles(s)
    out = {}
    for name in "qk":
        gamma = s["g" + name]
        dz = _turn(s["d" + name].float(), cos, -sin, s["rot"], s["inter"])
        out["dg" + name] = None
        if gamma is not None:
            x = s[name].float()
            rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
            xh = x * rstd
            out["dg" + name] = (dz * xh).sum((0, 1))
            g = dz * gamma
            dz = rstd * (g - xh * (g * xh).mean(-1, keepdim=True))
        out["d" + name] = dz.to(s["d" + name].dtype)
    return out


def _project(x, W, s, i, back=False):
    """x W + s (x A) B of projection i, or with the transposes."""
    W = W.float()
    y = x @ (W.t() if back else W)
    if s["As"] is not None:
        A, B = s["As"][i].float(), s["Bs"][i].float()
        y = y + s["scale"] * ((x @ B.t()) @ A.t() if back else (x @ A) @ B)
    return y


def _activation(g, act):
    """The activation and its derivative."""
    if act == "silu":
        p = 1 / (1 + (-g).exp())
        return g * p, p * (1 + g * (1 - p))
    c = math.sqrt(2 / math.pi)
    t = (c * (g + 0.044715 * g * g * g)).tanh()
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def _plain_ffn(s):
    x = s["x"].float()
    g, u = _project(x, s["Wg"], s, 0), _project(x, s["Wu"], s, 1)
    h = _activation(g, s["act"])[0] * u
    out = {"y": _project(h, s["Wd"], s, 2), "h": h}
    if s["save"]:
        out.update(g=g, u=u)
    return {name: t.to(torch.bfloat16) for name, t in out.items()}


def _plain_ffn_grad(s):
    g, u = s["g"].float(), s["u"].float()
    dh = _project(s["dy"].float(), s["Wd"], s, 2, back=True)
    a, slope = _activation(g, s["act"])
    dg, du = dh * u * slope, dh * a
    dx = _project(dg, s["Wg"], s, 0, back=True) + _project(du, s["Wu"], s, 1, back=True)
    return {"dx": dx.to(torch.bfloat16), "dg": dg.to(torch.bfloat16), "du": du.to(torch.bfloat16)}


def _mix(x):
    """A bijection of 32-bit numbers (held in 64) that spreads every bit over all."""
    x = x ^ (x >> 16)
    x = (x * 0xB504F333) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0xDDB3D743) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random_bits(s):
    """32 bits for every value, from the step's number, its tensor's and its own: [blocks, BLOCK]."""
    many = torch.tensor(s["blocks"], device=DEV)
    key = _mix(s["step"] ^ _mix(_mix(torch.arange(1, len(s["blocks"]) + 1, device=DEV))))
    key = _mix(key).repeat_interleave(many)
    first = (torch.tensor(s["starts"], device=DEV)).repeat_interleave(many)
    at = torch.arange(sum(s["blocks"]), device=DEV) * BLOCK - first
    return _mix((at[:, None] + torch.arange(BLOCK, device=DEV) + key[:, None]) & 0xFFFFFFFF)


def _decode(code, mant):
    """The value of codes of four exponent bits and `mant` mantissa bits: 0 to 2 less a step."""
    low = code & ((1 << mant) - 1)
    exp = code >> mant
    big = ((exp + 112) << 23 | low << (23 - mant)).to(torch.int32).view(torch.float32)
    return torch.where(exp > 0, big, low.float() * 2.0 ** (-14 - mant))


def _encode(a, mant, rnd):
    """Codes of values in [0, 2 less a step], rounded up with the probability of what is cut off."""
    cut = 23 - mant
    big = ((a.view(torch.int32).long() + rnd) >> cut) - (112 << mant)
    small = ((a * 2.0 ** 37).long() + rnd) >> cut
    return torch.where(a >= 2.0 ** -14, big, small).clamp(max=(16 << mant) - 1)


def _quantise(x, mant, rnd):
    """(codes, scales, values) of [blocks, BLOCK] sizes; a block without a size of 2^-100 is 0,
    one with a NaN or an infinity NaN."""
    top = x.amax(1, keepdim=True)
    scale = torch.where(top >= 2.0 ** -100, top * (1 / (2 - 2.0 ** -mant)), torch.zeros_like(top))
    a = torch.where(scale > 0, x * (1 / scale), torch.zeros_like(x))
    code = _encode(a, mant, rnd)
    scale = torch.where(top.isfinite(), scale, torch.full_like(scale, math.nan))
    return code, scale[:, 0], _decode(code, mant) * scale


def _plain_adamw(s):
    s["step"] += 1
    g, p = s["g"], s["p"]
    if s["bits"] == 32:
        m, v = s["m"], s["v"]
    else:
        cm, cv = s["m"].view(-1, BLOCK).long(), s["v"].view(-1, BLOCK).long()
        m = (_decode(cm & 127, 3) * s["ms"][:, None] * (1 - 2 * (cm >> 7))).view(-1)
        root = (_decode(cv, 4) * s["vs"][:, None]).view(-1)
        v = root * root
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * g) * (1 - BETA2)
    root = v.sqrt()
    denom = root / math.sqrt(1 - BETA2 ** s["step"]) + ADAM_EPS
    p.copy_(p * (1 - LR * DECAY) - (m * (LR / (1 - BETA1 ** s["step"]))) / denom)
    s["p16"].copy_(p)
    if s["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return {name: s[name] for name in ("p", "p16", "m", "v")}
    bits = _random_bits(s)
    cm, ms, size = _quantise(m.view(-1, BLOCK).abs(), 3, (bits & 0xFFFF) << 4)
    cv, vs, root = _quantise(root.view(-1, BLOCK), 4, (bits >> 16) << 3)
    sign = (m.view(-1, BLOCK) < 0) & (cm > 0)
    s["m"].copy_((cm + 128 * sign.long()).view(-1))
    s["v"].copy_(cv.view(-1))
    s["ms"].copy_(ms)
    s["vs"].copy_(vs)
    return {"p": p, "p16": s["p16"], "m": torch.where(sign, -size, size).view(-1), "v": (root * root).view(-1)}


_plain = {"rope": _plain_rope, "rope_grad": _plain_rope_grad, "ffn": _plain_ffn, "ffn_grad": _plain_ffn_grad,
          "adamw": _plain_adamw}


def _kept(s, key, make):
    """What a program keeps from call to call: made at the first."""
    if key not in s:
        s[key] = make()
    return s[key]


def _bytes(n):
    return torch.empty(n, dtype=torch.uint8, device=DEV)


def _bf16(*shape):
    return torch.empty(shape, dtype=torch.bfloat16, device=DEV)


def _table(s):
    from paper_2607_03441_gb300 import attt
    return attt.attt_rope_frequencies(s["rot"], s["base"], factor=s["factor"], context=s["context"], low=1.0, high=32.0,
                                      device=DEV)


def _call_rope(s):
    from paper_2607_03441_gb300 import attt
    freq = _kept(s, "freq", lambda: _table(s))
    ys = _kept(s, "ys", lambda: [torch.empty(s[n].shape, dtype=s[n].dtype, device=DEV) for n in "qk"])
    attt.attt_rope_forward([s["q"], s["k"]], s["pos"], freq, gammas=[s["gq"], s["gk"]], eps=EPS,
                           interleaved=s["inter"], mscale=s["mscale"], ys=ys)
    return dict(zip("qk", ys))


def _call_rope_grad(s):
    from paper_2607_03441_gb300 import attt
    freq = _kept(s, "freq", lambda: _table(s))
    ws = _kept(s, "ws", lambda: _bytes(attt.attt_rope_workspace_bytes(s["T"], s["D"])))
    dxs = _kept(s, "dxs", lambda: [torch.empty(s[n].shape, dtype=s[n].dtype, device=DEV) for n in "qk"])
    dgs = _kept(s, "dgs", lambda: [torch.empty(s["D"], device=DEV) if s["norm"] else None for _ in "qk"])
    attt.attt_rope_backward([s["dq"], s["dk"]], [s["q"], s["k"]], s["pos"], freq, gammas=[s["gq"], s["gk"]], eps=EPS,
                            interleaved=s["inter"], mscale=s["mscale"], dxs=dxs, dgammas=dgs, workspace=ws)
    return {"dq": dxs[0], "dk": dxs[1], "dgq": dgs[0], "dgk": dgs[1]}


def _call_ffn(s):
    from paper_2607_03441_gb300 import attt
    L, d, f = s["L"], s["d"], s["f"]
    ws = _kept(s, "ws", lambda: _bytes(attt.attt_gated_ffn_workspace_bytes(L, d, f, s["r"])))
    out = _kept(s, "out", lambda: {"y": _bf16(L, d), "h": _bf16(L, f),
                                   **({"g": _bf16(L, f), "u": _bf16(L, f)} if s["save"] else {})})
    attt.attt_gated_ffn_forward(s["x"], s["Wg"], s["Wu"], s["Wd"], As=s["As"], Bs=s["Bs"], scale=s["scale"],
                                act=s["act"], workspace=ws, **out)
    return out


def _call_ffn_grad(s):
    from paper_2607_03441_gb300 import attt
    L, d, f = s["L"], s["d"], s["f"]
    ws = _kept(s, "ws", lambda: _bytes(attt.attt_gated_ffn_workspace_bytes(L, d, f, s["r"])))
    out = _kept(s, "out", lambda: {"dx": _bf16(L, d), "dg": _bf16(L, f), "du": _bf16(L, f)})
    attt.attt_gated_ffn_backward(s["dy"], s["Wg"], s["Wu"], s["Wd"], s["g"], s["u"], As=s["As"], Bs=s["Bs"],
                                 scale=s["scale"], act=s["act"], workspace=ws, **out)
    return out


def _optimizer(s):
    """The handle over the tensors in the program's buffers."""
    from paper_2607_03441_gb300 import attt
    t = {name: [s[name][a:a + n] for a, n in zip(s["starts"], s["sizes"])] for name in ("p", "g", "m", "v", "p16")}
    scales = {}
    if s["bits"] == 8:
        for name in ("ms", "vs"):
            scales[name[0] + "_scales"] = [s[name][a // BLOCK:a // BLOCK + b] for a, b in zip(s["starts"], s["blocks"])]
    return attt.attt_adamw_create(t["p"], t["g"], t["m"], t["v"], p16s=t["p16"], **scales)


def _call_adamw(s):
    from paper_2607_03441_gb300 import attt
    opt = _kept(s, "opt", lambda: _optimizer(s))
    s["step"] += 1
    attt.attt_adamw_step(opt, LR, betas=(BETA1, BETA2), eps=ADAM_EPS, weight_decay=DECAY, step=s["step"],
                         seed=s["step"])
    if s["bits"] == 32:
        return {name: s[name] for name in ("p", "p16", "m", "v")}
    m, v = _kept(s, "values", lambda: (torch.empty_like(s["p"]), torch.empty_like(s["p"])))
    attt.attt_adamw_read_state(opt, m, v)
    return {"p": s["p"], "p16": s["p16"], "m": m, "v": v}


_calls = {"rope": _call_rope, "rope_grad": _call_rope_grad, "ffn": _call_ffn, "ffn_grad": _call_ffn_grad,
          "adamw": _call_adamw}


# --------------------------------------------------------------------------
# floors and 64-bit values
# --------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind in ("rope", "rope_grad"):
        n, e = case["T"] * (case["hq"] + case["hk"]) * case["D"], case["bits"] // 8
        back = kind == "rope_grad"
        # x in, y out; back: dy in, dx out, and with a norm x in; positions, weights
        return {"bytes": n * e * (3 if back and case["norm"] else 2) + 4 * case["T"] + 16 * case["D"],
                "flops": n * (6 + (8 if case["norm"] else 0) * (2 if back else 1))}
    if kind in ("ffn", "ffn_grad"):
        L, d, f, r = case["L"], case["d"], case["f"], case["r"]
        weights = 3 * d * f + 3 * r * (d + f)
        acts = L * (2 * d + (3 if case["save"] else 1) * f) if kind == "ffn" else L * (2 * d + 4 * f)
        return {"bytes": 2 * (weights + acts), "flops": 6 * L * d * f + 6 * L * r * (d + f)}
    n = sum(_sizes(case))
    if case["bits"] == 32:  # p, g, m, v in; p, m, v and the bf16 copy out
        return {"bytes": 30 * n, "flops": 14 * n}
    # p, g, codes and scales in; p, codes, scales, the bf16 copy and the moments' values out
    return {"bytes": 26 * n + 16 * n // BLOCK, "flops": 40 * n}


def exact(case, seed):
    s = prepare(case, seed)
    return _exact[case["kind"]](s)


def _exact_heads(s, name, x):
    """Norm and rotation in 64 bits: pairs as complex numbers."""
    if s["g" + name] is not None:
        x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * s["g" + name].double()
    half = s["rot"] // 2
    i = torch.arange(half, device=DEV).double()
    w = torch.exp(-2 * i / s["rot"] * math.log(s["base"]))
    if s["factor"] > 1:
        turns = s["context"] / (2 * math.pi) * w
        mix = torch.where(turns > 32, 1.0, torch.where(turns < 1, 0.0, (turns - 1) / 31))
        w = torch.lerp(w / s["factor"], w, mix)
    phase = torch.polar(torch.full_like(s["pos"][:, None].double() * w, s["mscale"]), s["pos"][:, None].double() * w)
    head, tail = x[..., :s["rot"]], x[..., s["rot"]:]
    pairs = head.unflatten(-1, (half, 2)) if s["inter"] else head.unflatten(-1, (2, half)).transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * phase[:, None])
    z = z.flatten(-2) if s["inter"] else z.transpose(-1, -2).flatten(-2)
    return torch.cat([z, tail], -1)


def _exact_rope(s):
    return {name: _exact_heads(s, name, s[name].double()) for name in "qk"}


def _exact_rope_grad(s):
    out = {}
    for name in "qk":
        x = s[name].double().requires_grad_()
        wanted = [x]
        if s["norm"]:
            s["g" + name] = s["g" + name].double().requires_grad_()
            wanted.append(s["g" + name])
        got = torch.autograd.grad(_exact_heads(s, name, x), wanted, s["d" + name].double())
        out["d" + name], out["dg" + name] = got[0], got[1] if s["norm"] else None
    return out


def _exact_weight(s, name, i):
    """The projection's weight with its adapter."""
    W = s[name].double()
    return W if s["As"] is None else torch.addmm(W, s["As"][i].double(), s["Bs"][i].double(), alpha=s["scale"])


def _exact_gate(g, u, act):
    return u * (torch.nn.functional.silu(g) if act == "silu" else torch.nn.functional.gelu(g, approximate="tanh"))


def _exact_ffn(s):
    x = s["x"].double()
    g, u = torch.matmul(x, _exact_weight(s, "Wg", 0)), torch.matmul(x, _exact_weight(s, "Wu", 1))
    h = _exact_gate(g, u, s["act"])
    out = {"y": torch.matmul(h, _exact_weight(s, "Wd", 2)), "h": h}
    return {**out, "g": g, "u": u} if s["save"] else out


def _exact_ffn_grad(s):
    dh = torch.einsum("ld,fd->lf", s["dy"].double(), _exact_weight(s, "Wd", 2))
    g, u = s["g"].double().requires_grad_(), s["u"].double().requires_grad_()
    dg, du = torch.autograd.grad(_exact_gate(g, u, s["act"]), (g, u), dh)
    del dh
    dx = torch.einsum("lf,df->ld", dg, _exact_weight(s, "Wg", 0))
    dx += torch.einsum("lf,df->ld", du, _exact_weight(s, "Wu", 1))
    return {"dx": dx, "dg": dg, "du": du}


def _exact_adamw(s):
    t = s["step"] + 1
    p, g = s["p"].double(), s["g"].double()
    m, root = s["m"], s["v"]
    if s["bits"] == 32:
        m, v = m.double(), root.double()
    else:  # codes through tables of all their values
        sizes = [torch.tensor([(c % 2 ** k + 2 ** k * (c >= 2 ** k)) * 2.0 ** (max(c >> k, 1) - 15 - k)
                               for c in range(16 * 2 ** k)], dtype=torch.float64, device=DEV) for k in (3, 4)]
        sizes[0] = torch.cat([sizes[0], -sizes[0]])
        m = (sizes[0][m.long()].view(-1, BLOCK) * s["ms"].double()[:, None]).view(-1)
        v = (sizes[1][root.long()].view(-1, BLOCK) * s["vs"].double()[:, None]).view(-1).square()
    m = torch.lerp(g, m, BETA1)
    v = torch.lerp(g.square(), v, BETA2)
    p = p - LR * DECAY * p - LR * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + ADAM_EPS)
    if s["bits"] == 8:  # which of two neighbours a moment is rounded to turns on its last bit of 32
        m = v = None
    return {"p": p, "p16": p, "m": m, "v": v}


_exact = {"rope": _exact_rope, "rope_grad": _exact_rope_grad, "ffn": _exact_ffn, "ffn_grad": _exact_ffn_grad,
          "adamw": _exact_adamw}

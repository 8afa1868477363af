"""An update of the adapters inside a transformer block, built from the library's calls.

One block of a causal model with adapters on q, k, v, gate, up and down:

    q, k, v = x Wq, x Wk, x Wv (each with its adapter);  q, k normed per head and turned
    a = attention(q, k, v) (torch; its gradient by torch.autograd);  t = x + a Wo
    y = t + ffn(layer_norm(t))

trained to follow a given next row with a squared loss: the projections
(attt_lora_forward, attt_lora_grad), the heads' norms and positions (attt_rope_forward,
attt_rope_backward), the norm in front of the feed-forward block (attt_layer_norm_*),
the block (attt_gated_ffn_forward, attt_gated_ffn_backward) and one AdamW step of all
adapters with moments in 8 bits (attt_adamw_create, attt_adamw_step).

    python examples/block_update.py [--rows L] [--width d] [--heads H] [--inner f] [--rank r] [--rounds N]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2607_03441_gb300 import attt  # noqa: E402

BF16 = torch.bfloat16
NAMES = ("q", "k", "v", "gate", "up", "down")


class Block:
    """Frozen weights and the adapters of one block.  kv heads are a half of the query heads."""

    def __init__(self, d: int, heads: int, f: int, r: int, generator: torch.Generator, scale: float = 1.0, bits: int = 8):
        dev = generator.device
        self.d, self.H, self.D, self.f, self.r, self.scale = d, heads, d // heads, f, r, scale
        self.Hk = max(1, heads // 2)
        kv = self.Hk * self.D

        def normal(*shape, std):
            return torch.randn(shape, generator=generator, device=dev) * std

        sizes = {"q": (d, d), "k": (d, kv), "v": (d, kv), "gate": (d, f), "up": (d, f), "down": (f, d)}
        self.W = {n: normal(*s, std=s[0] ** -0.5).to(BF16) for n, s in sizes.items()}
        self.Wo = normal(d, d, std=d ** -0.5).to(BF16)
        self.gq, self.gk = torch.ones(self.D, device=dev), torch.ones(self.D, device=dev)
        self.gamma = torch.ones(d, device=dev)
        self.freq = attt.attt_rope_frequencies(self.D, device=dev)
        # A from the start, B from zero: the block begins as the frozen one
        self.A32 = {n: normal(s[0], r, std=s[0] ** -0.5) for n, s in sizes.items()}
        self.B32 = {n: torch.zeros(r, s[1], device=dev) for n, s in sizes.items()}
        self.A = {n: t.to(BF16) for n, t in self.A32.items()}
        self.B = {n: t.to(BF16) for n, t in self.B32.items()}
        self.dA = {n: torch.zeros_like(t) for n, t in self.A32.items()}
        self.dB = {n: torch.zeros_like(t) for n, t in self.B32.items()}
        ps, gs, p16s = ([side[n] for n in NAMES for side in pair]
                        for pair in ((self.A32, self.B32), (self.dA, self.dB), (self.A, self.B)))
        if bits == 8:
            ms, vs = ([torch.zeros(p.shape, dtype=torch.uint8, device=dev) for p in ps] for _ in range(2))
            scales = [[torch.zeros(-(-p.numel() // attt.ADAMW_BLOCK), device=dev) for p in ps] for _ in range(2)]
        else:
            ms, vs = ([torch.zeros_like(p) for p in ps] for _ in range(2))
            scales = [None, None]
        self.opt = attt.attt_adamw_create(ps, gs, ms, vs, *scales, p16s=p16s)
        self.steps = 0

    def _project(self, x, n):
        return attt.attt_lora_forward(x, self.W[n], self.A[n], self.B[n], self.scale)

    def forward(self, x: torch.Tensor, pos: torch.Tensor):
        """y (bf16 [L, d]) and what the gradient needs."""
        L = x.shape[0]
        s = {"x": x, "pos": pos}
        s["q"], s["k"], s["v"] = (self._project(x, n).view(L, h, self.D) for n, h in (("q", self.H), ("k", self.Hk),
                                                                                 ("v", self.Hk)))
        s["rq"], s["rk"] = attt.attt_rope_forward([s["q"], s["k"]], pos, self.freq, [self.gq, self.gk])
        with torch.enable_grad():
            s["leaves"] = [t.detach().requires_grad_() for t in (s["rq"], s["rk"], s["v"])]
            q, k, v = (t.float().repeat_interleave(self.H // t.shape[1], 1).transpose(0, 1) for t in s["leaves"])
            scores = (q @ k.transpose(1, 2)) / math.sqrt(self.D)
            later = torch.ones(L, L, dtype=torch.bool, device=x.device).triu(1)
            s["a"] = (scores.masked_fill(later, -math.inf).softmax(-1) @ v).transpose(0, 1).reshape(L, self.d).to(BF16)
        t = (x.float() + (s["a"].detach().float() @ self.Wo.float())).to(BF16)
        s["t"] = t
        s["n"], s["mean"], s["rstd"] = attt.attt_layer_norm_forward(t, self.gamma)
        o, s["h"], s["g"], s["u"] = attt.attt_gated_ffn_forward(
            s["n"], self.W["gate"], self.W["up"], self.W["down"], *self._ffn_adapters(), self.scale, save=True)
        return (t.float() + o.float()).to(BF16), s

    def _ffn_adapters(self):
        return [[side[n] for n in ("gate", "up", "down")] for side in (self.A, self.B)]

    def backward(self, dy: torch.Tensor, s) -> None:
        """The adapters' gradients (dA, dB) from y's (bf16 [L, d])."""
        L = dy.shape[0]
        dn, dg, du = attt.attt_gated_ffn_backward(dy, self.W["gate"], self.W["up"], self.W["down"], s["g"], s["u"],
                                                  *self._ffn_adapters(), self.scale)
        self._adapter_grads(s["n"], ("gate", "up"), [dg, du])
        self._adapter_grads(s["h"], ("down",), [dy])
        dt, _, _ = attt.attt_layer_norm_backward(dn, s["t"], self.gamma, s["mean"], s["rstd"], weights=False)
        dt = dt.float() + dy.float()
        s["a"].backward((dt @ self.Wo.float().t()).to(BF16))
        drq, drk, dv = (t.grad for t in s["leaves"])
        (dq, dk), _ = attt.attt_rope_backward([drq.contiguous(), drk.contiguous()], [s["q"], s["k"]], s["pos"], self.freq,
                                              [self.gq, self.gk], weights=False)
        self._adapter_grads(s["x"], ("q", "k", "v"), [t.reshape(L, -1).contiguous() for t in (dq, dk, dv)])

    def _adapter_grads(self, x, names, dys):
        attt.attt_lora_grad(x, dys, [self.A[n] for n in names], [self.B[n] for n in names], self.scale,
                            dAs=[self.dA[n] for n in names], dBs=[self.dB[n] for n in names])

    def step(self, lr: float) -> None:
        self.steps += 1
        attt.attt_adamw_step(self.opt, lr, weight_decay=0.0, step=self.steps, seed=self.steps)


def train(rows: int = 128, width: int = 256, heads: int = 4, inner: int = 768, rank: int = 8, rounds: int = 40,
          lr: float = 2e-3, seed: int = 0, verbose: bool = True):
    """Returns every round's loss."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    block = Block(width, heads, inner, rank, g)
    x = torch.randn(rows, width, generator=g, device="cuda").to(BF16)
    want = torch.randn(rows, width, generator=g, device="cuda")
    pos = torch.arange(rows, dtype=torch.int32, device="cuda")
    losses = []
    for k in range(rounds):
        y, s = block.forward(x, pos)
        off = y.float() - want
        losses.append(off.square().mean().item())
        block.backward((2 / off.numel() * off).to(BF16), s)
        block.step(lr)
        if verbose:
            print(f"round {k:3d}  loss {losses[-1]:.5f}")
    code = attt.attt_device_status()
    if code != 0:
        raise RuntimeError(attt.attt_status_string(code))
    return losses


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("rows", 128), ("width", 256), ("heads", 4), ("inner", 768), ("rank", 8), ("rounds", 40)):
        p.add_argument(f"--{name}", type=int, default=value)
    train(**vars(p.parse_args()))


if __name__ == "__main__":
    main()

"""A policy-gradient update of an adapter, built from the library's calls.

A policy maps L contexts x to distributions over V tokens:

    h = x W0 + s (x A) B,   n = layer_norm(h),   p = softmax(n Wlm^T / T),

with W0 and the head Wlm frozen and the adapter A, B trained.  Every round picks one
token per context among its most probable alternatives, scores the tokens with a
reward, and takes one step on

    J = -1/L sum_j (advantage_j log p_j(token_j) + beta H(p_j)):

log probabilities, entropies and alternatives (attt_logprob_forward), the gradient
back to n (attt_logprob_input_grad), through the norm (attt_layer_norm_backward) to
the adapter (attt_lora_grad), and the step (attt_lora_muon_step).  The demonstration
rewards even tokens; the share of them rises.

    python examples/policy_update.py [--rows L] [--width d] [--vocab V] [--rank r] [--rounds N]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2607_03441_gb300 import attt  # noqa: E402


class Policy:
    """Frozen weights, a trained adapter, and the buffers an update needs: allocated
    once for L rows, so that a round allocates nothing but its own small results."""

    def __init__(self, W0: torch.Tensor, Wlm: torch.Tensor, A: torch.Tensor, B: torch.Tensor, rows: int,
                 scale: float = 1.0, inv_temp: float = 1.0, topk: int = 20):
        dev = W0.device
        din, d = W0.shape
        V, r = Wlm.shape[0], A.shape[1]
        self.W0, self.Wlm, self.scale, self.inv_temp, self.topk = W0, Wlm, float(scale), float(inv_temp), topk
        self.A32, self.B32 = A.float().contiguous(), B.float().contiguous()
        self.A16, self.B16 = self.A32.to(torch.bfloat16), self.B32.to(torch.bfloat16)
        self.mA, self.mB = torch.zeros_like(self.A32), torch.zeros_like(self.B32)
        self.dA, self.dB = torch.empty_like(self.A32), torch.empty_like(self.B32)
        self.gamma, self.beta = torch.ones(d, device=dev), torch.zeros(d, device=dev)
        need = [attt.attt_lora_forward_workspace_bytes(rows, din, d, r),
                attt.attt_logprob_workspace_bytes(rows, d, V, topk),
                attt.attt_logprob_grad_workspace_bytes(rows, d, V),
                attt.attt_layer_norm_workspace_bytes(rows, d),
                attt.attt_lora_workspace_bytes(rows, din, [d], r),
                attt.attt_lora_muon_workspace_bytes([din], [d], r)]
        self.ws = torch.empty(max(need), dtype=torch.uint8, device=dev)  # the calls follow one another
        self.h, self.n, self.dn, self.dh = (torch.empty(rows, d, dtype=torch.bfloat16, device=dev) for _ in range(4))
        self.mean, self.rstd = torch.empty(rows, device=dev), torch.empty(rows, device=dev)

    def hidden(self, x: torch.Tensor) -> torch.Tensor:
        """n = layer_norm(x W0 + s (x A) B), bf16 [L, d]."""
        attt.attt_lora_forward(x, self.W0, self.A16, self.B16, self.scale, h=self.h, workspace=self.ws)
        attt.attt_layer_norm_forward(self.h, self.gamma, self.beta, y=self.n, mean=self.mean, rstd=self.rstd)
        return self.n

    def alternatives(self, x: torch.Tensor):
        """The most probable tokens of every row and their log probabilities [L, topk]."""
        _, _, _, top_logp, top_id = attt.attt_logprob_forward(self.hidden(x), self.Wlm, topk=self.topk,
                                                              inv_temp=self.inv_temp, workspace=self.ws)
        return top_logp, top_id

    def gradients(self, x: torch.Tensor, tokens: torch.Tensor, advantage: torch.Tensor, beta: float):
        """J's gradients (dA, dB) at the tokens, and (logp, entropy)."""
        L = x.shape[0]
        n = self.hidden(x)
        logp, entropy, lse, _, _ = attt.attt_logprob_forward(n, self.Wlm, tokens, inv_temp=self.inv_temp,
                                                             workspace=self.ws)
        gent = torch.full((L,), -beta / L, device=x.device)
        attt.attt_logprob_input_grad(n, self.Wlm, tokens, lse, advantage * (-1.0 / L), entropy, gent, self.inv_temp,
                                     dh=self.dn, workspace=self.ws)
        attt.attt_layer_norm_backward(self.dn, self.h, self.gamma, self.mean, self.rstd, dx=self.dh,
                                      workspace=self.ws, weights=False)
        attt.attt_lora_grad(x, [self.dh], [self.A16], [self.B16], self.scale, dAs=[self.dA], dBs=[self.dB],
                            workspace=self.ws)
        return self.dA, self.dB, logp, entropy

    def step(self, lr: float) -> None:
        attt.attt_lora_muon_step([self.A32], [self.B32], [self.dA], [self.dB], [self.mA], [self.mB], lr,
                                 A16s=[self.A16], B16s=[self.B16], workspace=self.ws)


def train(rows: int = 256, width: int = 512, vocab: int = 8192, rank: int = 16, rounds: int = 30, lr: float = 0.02,
          beta: float = 0.001, seed: int = 0, verbose: bool = True):
    """Returns the share of even tokens of every round."""
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape, std):
        return torch.randn(shape, generator=g, device=dev) * std

    W0 = normal(width, width, std=width ** -0.5).to(torch.bfloat16)
    Wlm = normal(vocab, width, std=2 * width ** -0.5).to(torch.bfloat16)
    policy = Policy(W0, Wlm, normal(width, rank, std=width ** -0.5), torch.zeros(rank, width, device=dev), rows)
    x = normal(rows, width, std=1.0).to(torch.bfloat16)
    shares = []
    for k in range(rounds):
        top_logp, top_id = policy.alternatives(x)
        pick = torch.multinomial(top_logp.exp(), 1, generator=g)
        tokens = top_id.gather(1, pick)[:, 0].contiguous()
        reward = (tokens % 2 == 0).float()
        _, _, logp, entropy = policy.gradients(x, tokens, reward - reward.mean(), beta)
        policy.step(lr)
        shares.append(reward.mean().item())
        if verbose:
            print(f"round {k:3d}  even tokens {shares[-1]:.3f}  log p {logp.mean().item():8.3f}  "
                  f"entropy {entropy.mean().item():.3f}")
    code = attt.attt_device_status()
    if code != 0:
        raise RuntimeError(attt.attt_status_string(code))
    return shares


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("rows", 256), ("width", 512), ("vocab", 8192), ("rank", 16), ("rounds", 30)):
        p.add_argument(f"--{name}", type=int, default=value)
    train(**vars(p.parse_args()))


if __name__ == "__main__":
    main()

"""The calls of an adapted block run together (examples/block_update.py): the gradients of all
adapters against fp64 autograd of the same block, the step, and a graph.

Bounds: every stage rounds its result to bf16, 2^-8 of it at most and 2^-8 / sqrt(3) in root mean
square; a gradient passes some 12 of them forth and back (projection, turn, attention, sum,
norm, h, y; dn, dg, dt, da, drq, dq), and roundings of different values are independent:
norm-wise sqrt(12) 2^-8 / sqrt(3) = 0.8%, doubled for what a stage amplifies."""
import importlib.util
import math
import os

import pytest
import torch

from paper_2607_03441_gb300 import attt, build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    build.build()
    path = os.path.join(os.path.dirname(__file__), "..", "examples", "block_update.py")
    spec = importlib.util.spec_from_file_location("block_update", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def _block(example, d, heads, f, r, bits=8, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    b = example.Block(d, heads, f, r, g, scale=0.5, bits=bits)
    for n in example.NAMES:  # adapters some steps on
        b.B32[n].normal_(std=0.3 / math.sqrt(r), generator=g)
        b.B[n].copy_(b.B32[n])
    b.gq.add_(0.2 * torch.randn(b.D, generator=g, device="cuda"))
    b.gk.add_(0.2 * torch.randn(b.D, generator=g, device="cuda"))
    return b, g


def _turn(x, pos, freq):
    w = freq.double() / 2.0 ** 64 * 2 * math.pi
    w = torch.where(freq < 0, w + 2 * math.pi, w)
    angle = pos.double()[:, None] * w
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    a, b = x.chunk(2, -1)
    return torch.cat([a * c - b * s, a * s + b * c], -1)


def _reference(b, x, pos, dy, names):
    """y and the adapters' gradients in fp64."""
    A = {n: b.A[n].double().requires_grad_() for n in names}
    B = {n: b.B[n].double().requires_grad_() for n in names}
    x = x.double()
    L = x.shape[0]

    def project(v, n):
        return v @ b.W[n].double() + b.scale * (v @ A[n]) @ B[n]

    q, k, v = (project(x, n).view(L, h, b.D) for n, h in (("q", b.H), ("k", b.Hk), ("v", b.Hk)))
    q, k = (t * torch.rsqrt(t.square().mean(-1, keepdim=True) + 1e-6) * g.double() for t, g in ((q, b.gq), (k, b.gk)))
    q, k = _turn(q, pos, b.freq), _turn(k, pos, b.freq)
    q, k, v = (t.repeat_interleave(b.H // t.shape[1], 1).transpose(0, 1) for t in (q, k, v))
    scores = (q @ k.transpose(1, 2)) / math.sqrt(b.D)
    later = torch.ones(L, L, dtype=torch.bool, device=x.device).triu(1)
    a = (scores.masked_fill(later, -math.inf).softmax(-1) @ v).transpose(0, 1).reshape(L, b.d)
    t = x + a @ b.Wo.double()
    n = torch.nn.functional.layer_norm(t, (b.d,), b.gamma.double(), None, 1e-5)
    y = t + project(torch.nn.functional.silu(project(n, "gate")) * project(n, "up"), "down")
    y.backward(dy.double())
    return y, {m: (A[m].grad, B[m].grad) for m in names}


@pytest.mark.parametrize("L,d,heads,f,r", [(1, 128, 2, 256, 8), (50, 256, 4, 520, 16), (200, 192, 6, 768, 8)])
def test_gradients(example, L, d, heads, f, r):
    b, g = _block(example, d, heads, f, r)
    x, dy = ((torch.randn(L, d, generator=g, device="cuda")).to(torch.bfloat16) for _ in range(2))
    pos = torch.arange(7, 7 + L, dtype=torch.int32, device="cuda")
    y, s = b.forward(x, pos)
    b.backward(dy, s)
    assert attt.attt_device_status() == 0
    want, grads = _reference(b, x, pos, dy, example.NAMES)
    bound = 2 * math.sqrt(12 / 3) * 2.0 ** -8
    assert (y.double() - want).norm() <= bound * want.norm()
    for n, pair in grads.items():
        for got, ref in zip((b.dA[n], b.dB[n]), pair):
            if ref.norm() < 1e-6:  # a single token attends to itself alone: q and k have no gradient
                assert got.norm() < 1e-3 * dy.float().norm()
            else:
                assert (got.double() - ref).norm() <= bound * ref.norm(), n


def test_step_moves_every_adapter_against_its_gradient(example):
    for bits in (8, 32):
        b, g = _block(example, 128, 2, 256, 8, bits)
        x, dy = ((torch.randn(40, 128, generator=g, device="cuda")).to(torch.bfloat16) for _ in range(2))
        pos = torch.arange(40, dtype=torch.int32, device="cuda")
        _, s = b.forward(x, pos)
        b.backward(dy, s)
        before = {n: (b.A32[n].clone(), b.B32[n].clone()) for n in example.NAMES}
        b.step(1e-3)
        for n in example.NAMES:
            for p, q, grad, p16 in zip((b.A32[n], b.B32[n]), before[n], (b.dA[n], b.dB[n]), (b.A[n], b.B[n])):
                # the first step is lr times the gradient's sign (eps 1e-8 aside)
                big = grad.abs() > 1e-4
                assert big.any() and torch.allclose((q - p)[big], 1e-3 * grad[big].sign(), rtol=1e-3, atol=1e-6)
                assert torch.equal(p16, p.to(torch.bfloat16))


def test_feed_forward_and_step_in_a_graph(example):
    """Block, adapter gradients and step, captured once and replayed: as issued one by one."""
    runs = []
    for graphed in (False, True):
        b, g = _block(example, 128, 2, 256, 8, seed=3)
        x, dy = ((torch.randn(60, 128, generator=g, device="cuda")).to(torch.bfloat16) for _ in range(2))

        def update(b=b, x=x, dy=dy):
            W = b.W["gate"], b.W["up"], b.W["down"]
            y, h, gate, up = attt.attt_gated_ffn_forward(x, *W, *b._ffn_adapters(), b.scale, save=True)
            _, dg, du = attt.attt_gated_ffn_backward(dy, *W, gate, up, *b._ffn_adapters(), b.scale)
            b._adapter_grads(x, ("gate", "up"), [dg, du])
            b._adapter_grads(h, ("down",), [dy])
            attt.attt_adamw_step(b.opt, 1e-3, step=1, seed=5)
            return y

        if graphed:
            graph = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                y = update()
            for _ in range(3):
                graph.replay()
        else:
            for _ in range(3):
                y = update()
        torch.cuda.synchronize()
        runs.append([y] + [t for n in example.NAMES for t in (b.A32[n], b.B32[n], b.A[n], b.B[n])])
    assert all(torch.equal(p, q) for p, q in zip(*runs))


def test_example_runs(example):
    losses = example.train(rows=64, rounds=3, verbose=False)
    assert len(losses) == 3 and all(math.isfinite(v) for v in losses)

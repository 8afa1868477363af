"""The gated feed-forward block with results in the memory of what was read: y in x, dx in dy or in g,
dg and du in g and u, as with memory of their own; results that share memory are refused."""
import pytest
import torch

from paper_2607_03441_gb300 import attt, build
from tests.gpu_util import DEV
from tests.test_gpu_gated_ffn import Case

pytestmark = pytest.mark.gpu

SHAPES = [  # L, d, f, r: few rows (one CTA a tile, clusters), whole tiles (pairs), K pieces and their sum
    (5, 64, 128, 8), (40, 4104, 4104, 16), (96, 4104, 4104, 0), (300, 128, 264, 8), (700, 320, 5000, 40), (300, 3584, 64, 16),
    (300, 2048, 2048, 12), (4352, 512, 2304, 64),
]


@pytest.fixture(scope="module", autouse=True)
def _library():
    build.build()


@pytest.mark.parametrize("shape", SHAPES)
def test_in_place(shape):
    c = Case(*shape)
    L, d, f, _ = shape
    y, h, g, u = attt.attt_gated_ffn_forward(c.x, *c.W, **c.kw, save=True)
    x = c.x.clone()
    got = attt.attt_gated_ffn_forward(x, *c.W, **c.kw, save=True, y=x)
    assert all(torch.equal(a, b) for a, b in zip(got, (y, h, g, u)))
    want = attt.attt_gated_ffn_backward(c.dy, *c.W, c.g, c.u, **c.kw)
    dy, gg, uu = c.dy.clone(), c.g.clone(), c.u.clone()
    got = attt.attt_gated_ffn_backward(dy, *c.W, gg, uu, **c.kw, dx=dy, dg=gg, du=uu)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    if f >= d:
        gg = c.g.clone()
        dx = gg.view(-1)[:L * d].view(L, d)
        got = attt.attt_gated_ffn_backward(c.dy, *c.W, gg, c.u, **c.kw, dx=dx)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert attt.attt_device_status() == 0


def test_in_place_in_a_graph():
    c = Case(93, 512, 2048, 16)
    want = attt.attt_gated_ffn_backward(c.dy, *c.W, c.g, c.u, **c.kw)
    dy, g, u = c.dy.clone(), c.g.clone(), c.u.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        dy.copy_(c.dy), g.copy_(c.g), u.copy_(c.u)
        attt.attt_gated_ffn_backward(dy, *c.W, g, u, **c.kw, dx=dy, dg=g, du=u)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((dy, g, u), want))


def test_shared_results_are_refused():
    c = Case(16, 64, 128, 8)
    one = torch.empty(16, 128, dtype=torch.bfloat16, device=DEV)
    n = attt.attt_kernel_launches()
    for call in (lambda: attt.attt_gated_ffn_forward(c.x, *c.W, **c.kw, h=one, g=one),
                 lambda: attt.attt_gated_ffn_forward(c.x, *c.W, **c.kw, g=one, u=one),
                 lambda: attt.attt_gated_ffn_forward(c.x, *c.W, **c.kw, y=one.view(-1)[:1024].view(16, 64), h=one),
                 lambda: attt.attt_gated_ffn_backward(c.dy, *c.W, c.g, c.u, **c.kw, dg=one, du=one),
                 lambda: attt.attt_gated_ffn_backward(c.dy, *c.W, c.g, c.u, **c.kw, dg=c.u, du=c.g)):
        with pytest.raises(attt.AtttError) as e:
            call()
        assert e.value.code == attt.ATTT_ERR_INVALID_ARG
    assert attt.attt_kernel_launches() == n

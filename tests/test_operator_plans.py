"""The shapes of test_gpu_logprob_heads.py run what they are there for on 152 SMs: the
gradient on whole tiles of CTA pairs and a last wave cut into K pieces (from the
library's own headers)."""
import subprocess

from paper_2607_03441_gb300 import build
from tests.test_gpu_logprob_heads import CUT_TAILS

PROGRAM = r"""
#include <cstdio>
#include "gemm_launch.cuh"
using namespace attt;
// L, d, V: whether tiles are CTA pairs', their pieces, row tiles, whole waves, pieces of the last wave's tiles
int main() {
    long long L, d, V;
    while (std::scanf("%lld %lld %lld", &L, &d, &V) == 3) {
        const int64_t kb = cdiv(V, 64), most = 2 * kMaxPieces * cdiv(L, 256) * cdiv(d, 256);
        const int regions = (int)(most < 320 ? most : 320);
        const TilePlan t = plan_tiles(L, d, kb, 152, regions, true, true);
        const int units = t.pair ? 76 : 152, rows = t.pair ? 256 : 128;
        const int tiles = (int)(cdiv(L, rows) * cdiv(d, t.BN));
        std::printf("%d %d %d %d %d\n", t.pair ? 1 : 0, t.pieces, (int)cdiv(L, rows), tiles / units,
                    tail_pieces(tiles, units, (int)kb, t.pair ? 2 : 1, regions));
    }
}
"""


def test_gradients_of_cut_tails(tmp_path):
    src, exe = tmp_path / "plans.cu", tmp_path / "plans"
    src.write_text(PROGRAM)
    subprocess.run([build._nvcc(), *build.ARCH, *build.NVCC_FLAGS, str(src), "-o", str(exe)], check=True)
    text = "\n".join(" ".join(map(str, s)) for s in CUT_TAILS)
    out = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True).stdout
    got = [tuple(map(int, line.split())) for line in out.splitlines()]
    for (L, d, V), (pair, pieces, row_tiles, waves, cut) in zip(CUT_TAILS, got):
        assert pair and pieces == 1 and row_tiles > 1 and waves >= 1 and cut > 1, (L, d, V)
    assert sorted(g[-1] for g in got) == [2, 3, 4, 4]
    assert all(L % 256 for L, _, _ in CUT_TAILS)  # the last row tile is partial

"""What the Muon kernels do after a wait that ran out, on the parts that they share
(csrc/muon.cuh): a CTA whose exchange did not arrive sends nothing more, so that the
others' waits run out too, and no CTA of the cluster writes the weights.

A program of one cluster of two CTAs: one exchange of an 16 x 16 matrix's halves, then
the update.  Where the first CTA has lost an exchange before (its flag is set from the
start), the second's wait is bounded by the library's limit and returns."""
import subprocess

import pytest

from paper_2607_03441_gb300 import build

pytestmark = pytest.mark.gpu

PROGRAM = r"""
#include <cstdio>
#include "muon.cuh"
using namespace attt;

constexpr int RP = 16, LD = RP + 4, kCols = 8;

// X of CTA c is c + 1 everywhere; z's rows [8 c, 8 c + 8) are 10 (c + 1).
__global__ void __launch_bounds__(kMuonThreads, 1) step(const __grid_constant__ MuonArgs a, int lost, float *z_out) {
    __shared__ __align__(8) uint64_t bars[2];
    __shared__ int abort_flag;
    const int rank = (int)cluster_ctarank();
    float *const z = muon_smem(0), *const X = muon_smem(RP * LD);
    for (int e = threadIdx.x; e < RP * LD; e += kMuonThreads) z[e] = e / LD / 8 == rank ? 10.f * (rank + 1) : 0.f;
    for (int e = threadIdx.x; e < kCols * LD; e += kMuonThreads) X[e] = (float)(rank + 1);
    const MuonLink link{smem_u32(bars), 2, rank, &abort_flag, a.status};
    if (threadIdx.x == 0) {
        mbar_init(link.bar0, 1);
        mbar_init(link.bar0 + 8u, 1);
        abort_flag = lost && rank == 0;
        fence_mbar_init();
    }
    cluster_sync();
    link.share<LD>(0, z + 8 * rank * LD, z, 8 * rank, 8 * rank + 8, RP);
    __syncthreads();
    const MuonMat &t = a.mat[0];
    UPDATE
    if (rank == 1 && threadIdx.x == 0) *z_out = z[0];
    cluster_sync();
}

int main(int, char **argv) {
    const int lost = argv[1][0] == '1';
    MuonArgs a{};
    float *p, *z;
    int *status;
    cudaMalloc(&p, 2 * kCols * RP * sizeof(float));
    cudaMalloc(&z, sizeof(float));
    cudaMalloc(&status, sizeof(int));
    cudaMemset(p, 0, 2 * kCols * RP * sizeof(float));
    cudaMemset(status, 0, sizeof(int));
    a.r = RP; a.cluster = 2; a.inv_r = (uint32_t)(((1ull << 32) + RP - 1) / RP); a.keep = 1.f; a.status = status;
    a.mat[0].p = p; a.mat[0].n = 2 * kCols; a.mat[0].per = kCols; a.mat[0].tall = 1; a.mat[0].step = 1.f;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2);
    cfg.blockDim = dim3(kMuonThreads);
    cfg.dynamicSmemBytes = (RP + kCols) * LD * sizeof(float);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, step, a, lost, z) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) return 1;
    float hp[2 * kCols * RP], hz;
    int hs;
    cudaMemcpy(hp, p, sizeof hp, cudaMemcpyDeviceToHost);
    cudaMemcpy(&hz, z, sizeof hz, cudaMemcpyDeviceToHost);
    cudaMemcpy(&hs, status, sizeof hs, cudaMemcpyDeviceToHost);
    for (int c = 0; c < 2; ++c) {  // one value each, all of a CTA's columns alike
        for (int e = 1; e < kCols * RP; ++e)
            if (hp[c * kCols * RP + e] != hp[c * kCols * RP]) return 2;
        std::printf("%g ", hp[c * kCols * RP]);
    }
    std::printf("%g %d\n", hz, hs);
}
"""
UPDATE = "muon_update<RP>(a, t, RP * LD, rank * t.per, kCols, link);"


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    d = tmp_path_factory.mktemp("timeout")
    src, exe = d / "step.cu", d / "step"
    src.write_text(PROGRAM.replace("UPDATE", UPDATE))
    subprocess.run([build._nvcc(), *build.ARCH, *build.NVCC_FLAGS, str(src), "-o", str(exe)], check=True)

    def go(lost):
        out = subprocess.run([str(exe), str(lost)], capture_output=True, text=True, check=True, timeout=120).stdout
        return [float(v) for v in out.split()]
    return go


def test_an_exchange_that_arrives_is_followed_by_the_update(run):
    assert run(0) == [-1.0, -2.0, 10.0, 0.0]


def test_after_a_lost_exchange_nothing_is_sent_and_no_weight_written(run):
    from paper_2607_03441_gb300 import attt
    assert run(1) == [0.0, 0.0, 0.0, float(attt.ATTT_ERR_TIMEOUT)]

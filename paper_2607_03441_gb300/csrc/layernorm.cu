// layernorm.cu -- layer norm over the rows of a matrix, forward and backward,
// with the reduction of the weight's and the bias's gradient.
//
//   y_i = (x_i - mean) rstd gamma_i + beta_i,  rstd = 1 / sqrt(var + eps)
//   with g = dy gamma, xh = (x - mean) rstd:
//   dx = rstd (g - mean(g) - xh mean(g xh)),  dgamma = sum_rows dy xh,  dbeta = sum_rows dy
// A row stays in the registers of its warps between the reductions (mean, then the
// centred variance: no difference of large sums), so x and dy are read and y and
// dx written once; all sums are fp32.  Bound: HBM bytes, below a few hundred rows
// the chain of a launch, a load, two reductions and a store.
// The backward keeps the weight sums of a thread's columns in registers over all
// rows that its block takes; blocks leave one partial row each, and a second kernel
// adds those in a fixed order.
#include <algorithm>

#include "attt_common.cuh"
#include "attt_host.h"

namespace attt {

constexpr int kLnMaxBlocks = 4 * 160;  // partial rows of the weight gradients, at most

__device__ __forceinline__ void ln_load(const float *p, float (&f)[4]) {
    const float4 v = __ldcs(reinterpret_cast<const float4 *>(p));
    f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
}
__device__ __forceinline__ void ln_load(const __nv_bfloat16 *p, float (&f)[8]) {
    const uint4 u = __ldcs(reinterpret_cast<const uint4 *>(p));
    const __nv_bfloat162 *b = reinterpret_cast<const __nv_bfloat162 *>(&u);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float2 v = __bfloat1622float2(b[e]);
        f[2 * e] = v.x;
        f[2 * e + 1] = v.y;
    }
}
__device__ __forceinline__ void ln_load(const float *p, float (&f)[1]) { f[0] = *p; }
__device__ __forceinline__ void ln_load(const __nv_bfloat16 *p, float (&f)[1]) { f[0] = __bfloat162float(*p); }
__device__ __forceinline__ void ln_store(float *p, const float (&f)[4]) {
    *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]);
}
__device__ __forceinline__ void ln_store(__nv_bfloat16 *p, const float (&f)[8]) {
    uint4 u;
    __nv_bfloat162 *b = reinterpret_cast<__nv_bfloat162 *>(&u);
#pragma unroll
    for (int e = 0; e < 4; ++e) b[e] = __floats2bfloat162_rn(f[2 * e], f[2 * e + 1]);
    *reinterpret_cast<uint4 *>(p) = u;
}
__device__ __forceinline__ void ln_store(float *p, const float (&f)[1]) { *p = f[0]; }
__device__ __forceinline__ void ln_store(__nv_bfloat16 *p, const float (&f)[1]) { *p = __float2bfloat16_rn(f[0]); }

// W consecutive weights (nullptr: zeros).
template <int W>
__device__ __forceinline__ void ln_weights(const float *p, int c, float (&f)[W]) {
    if (p == nullptr) {
#pragma unroll
        for (int e = 0; e < W; ++e) f[e] = 0.f;
    } else if constexpr (W >= 4) {
#pragma unroll
        for (int e = 0; e < W; e += 4) {
            const float4 v = __ldg(reinterpret_cast<const float4 *>(p + c + e));
            f[e] = v.x; f[e + 1] = v.y; f[e + 2] = v.z; f[e + 3] = v.w;
        }
    } else {
        f[0] = __ldg(p + c);
    }
}

// Sums of N values over the `warps` warps of a row, in every thread.  `red`: 32 N
// floats of shared memory that no other call of this row's warps still reads (a
// row's calls alternate between two).
template <int N>
__device__ __forceinline__ void ln_reduce(float (&v)[N], int warps, int wr, int lane, int bar, float *red) {
#pragma unroll
    for (int n = 0; n < N; ++n)
        for (int o = 16; o > 0; o >>= 1) v[n] += __shfl_xor_sync(0xffffffffu, v[n], o);
    if (warps == 1) return;
    if (lane == 0)
#pragma unroll
        for (int n = 0; n < N; ++n) red[32 * n + wr] = v[n];
    named_barrier_sync(1u + bar, 32u * warps);
#pragma unroll
    for (int n = 0; n < N; ++n) {
        float s = lane < warps ? red[32 * n + lane] : 0.f;
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        v[n] = s;
    }
}

struct LnShape {
    int64_t L, x_ld, y_ld, g_ld;  // g_ld: dy
    int d;
    int warps;  // of a row
    float inv_d, eps;
};

// One row per `warps` warps, NV vectors of W values per thread (NV 0: any number, x
// read three times, from L2 after the first).
template <class T, int W, int NV>
__global__ void __launch_bounds__(1024) ln_forward_kernel(const T *__restrict__ x, const float *__restrict__ gamma,
                                  const float *__restrict__ beta, T *__restrict__ y, float *__restrict__ mean,
                                  float *__restrict__ rstd, const LnShape s) {
    __shared__ float red[2][8 * 32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int grp = warp / s.warps, wr = warp - grp * s.warps;
    const int64_t row = (int64_t)blockIdx.x * (blockDim.x / 32 / s.warps) + grp;
    if (row >= s.L) return;  // the whole row's warps
    const int t0 = (wr * 32 + lane) * W, step = s.warps * 32 * W;
    const T *xr = x + row * s.x_ld;
    T *yr = y + row * s.y_ld;
    float sum[1] = {0.f}, sq[1] = {0.f};
    float mu, rs;
    if constexpr (NV > 0) {
        float v[NV][W];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = t0 + k * step;
            if (c < s.d) {
                ln_load(xr + c, v[k]);
            } else {
#pragma unroll
                for (int e = 0; e < W; ++e) v[k][e] = 0.f;
            }
        }
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < W; ++e) sum[0] += v[k][e];
        ln_reduce<1>(sum, s.warps, wr, lane, grp, red[0] + grp * 32);
        mu = sum[0] * s.inv_d;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (t0 + k * step < s.d)
#pragma unroll
                for (int e = 0; e < W; ++e) {
                    v[k][e] -= mu;
                    sq[0] = fmaf(v[k][e], v[k][e], sq[0]);
                }
        ln_reduce<1>(sq, s.warps, wr, lane, grp, red[1] + grp * 32);
        rs = 1.f / sqrtf(fmaf(sq[0], s.inv_d, s.eps));
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = t0 + k * step;
            if (c < s.d) {
                float g[W], b[W];
                ln_weights<W>(gamma, c, g);
                ln_weights<W>(beta, c, b);
#pragma unroll
                for (int e = 0; e < W; ++e) v[k][e] = fmaf(v[k][e] * rs, g[e], b[e]);
                ln_store(yr + c, v[k]);
            }
        }
    } else {
        float v[W], g[W], b[W];
        for (int c = t0; c < s.d; c += step) {
            ln_load(xr + c, v);
#pragma unroll
            for (int e = 0; e < W; ++e) sum[0] += v[e];
        }
        ln_reduce<1>(sum, s.warps, wr, lane, grp, red[0] + grp * 32);
        mu = sum[0] * s.inv_d;
        for (int c = t0; c < s.d; c += step) {
            ln_load(xr + c, v);
#pragma unroll
            for (int e = 0; e < W; ++e) sq[0] = fmaf(v[e] - mu, v[e] - mu, sq[0]);
        }
        ln_reduce<1>(sq, s.warps, wr, lane, grp, red[1] + grp * 32);
        rs = 1.f / sqrtf(fmaf(sq[0], s.inv_d, s.eps));
        for (int c = t0; c < s.d; c += step) {
            ln_load(xr + c, v);
            ln_weights<W>(gamma, c, g);
            ln_weights<W>(beta, c, b);
#pragma unroll
            for (int e = 0; e < W; ++e) v[e] = fmaf((v[e] - mu) * rs, g[e], b[e]);
            ln_store(yr + c, v);
        }
    }
    if (wr == 0 && lane == 0) {
        if (mean) mean[row] = mu;
        if (rstd) rstd[row] = rs;
    }
}

// Warps per row at most: what the registers of a thread's values and sums leave.
constexpr int ln_backward_warps(int W, int nv) { return W * nv >= 8 && nv > 1 ? 16 : 32; }

// Rows blockIdx.x * groups + group, then every gridDim.x * groups-th; `part`: two
// partial rows (dgamma, dbeta) per block, [gridDim.x][2][d].  Shared memory: 2 d
// floats where a block has several groups.  NV 0: any number of vectors, the sums
// kept in the block's partial rows (one group).
template <class T, int W, int NV>
__global__ void __launch_bounds__(32 * ln_backward_warps(W, NV)) ln_backward_kernel(const T *__restrict__ dy, const T *__restrict__ x, const float *__restrict__ gamma,
                                   const float *__restrict__ mean, const float *__restrict__ rstd, T *__restrict__ dx,
                                   float *__restrict__ part, const LnShape s) {
    extern __shared__ float s_sum[];
    __shared__ float red[2][8 * 64];
    griddep_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int grp = warp / s.warps, wr = warp - grp * s.warps, groups = blockDim.x / 32 / s.warps;
    const int t0 = (wr * 32 + lane) * W, step = s.warps * 32 * W;
    float *out = part + (int64_t)blockIdx.x * 2 * s.d;
    int par = 0;
    if constexpr (NV > 0) {
        float ag[NV][W], ab[NV][W];
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < W; ++e) ag[k][e] = ab[k][e] = 0.f;
        for (int64_t row = (int64_t)blockIdx.x * groups + grp; row < s.L; row += (int64_t)gridDim.x * groups, par ^= 1) {
            float xv[NV][W], gv[NV][W];
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int c = t0 + k * step;
                if (c < s.d) {
                    ln_load(x + row * s.x_ld + c, xv[k]);
                    ln_load(dy + row * s.g_ld + c, gv[k]);
                } else {
#pragma unroll
                    for (int e = 0; e < W; ++e) xv[k][e] = gv[k][e] = 0.f;
                }
            }
            const float mu = __ldg(mean + row), rs = __ldg(rstd + row);
            float sums[2] = {0.f, 0.f};
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int c = t0 + k * step;
                if (c < s.d) {
                    float g[W];
                    ln_weights<W>(gamma, c, g);
#pragma unroll
                    for (int e = 0; e < W; ++e) {
                        const float xh = (xv[k][e] - mu) * rs;
                        ag[k][e] = fmaf(gv[k][e], xh, ag[k][e]);
                        ab[k][e] += gv[k][e];
                        const float t = gv[k][e] * g[e];
                        xv[k][e] = xh;
                        gv[k][e] = t;
                        sums[0] += t;
                        sums[1] = fmaf(t, xh, sums[1]);
                    }
                }
            }
            ln_reduce<2>(sums, s.warps, wr, lane, grp, red[par] + grp * 64);
            const float c1 = sums[0] * s.inv_d, c2 = sums[1] * s.inv_d;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int c = t0 + k * step;
                if (c < s.d) {
                    float o[W];
#pragma unroll
                    for (int e = 0; e < W; ++e) o[e] = rs * (gv[k][e] - fmaf(xv[k][e], c2, c1));
                    ln_store(dx + row * s.y_ld + c, o);
                }
            }
        }
        // the groups' sums in group order, then the block's partial rows
        for (int q = 0; q < groups; ++q) {
            if (q == grp) {
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    const int c = t0 + k * step;
                    if (c < s.d) {
#pragma unroll
                        for (int e = 0; e < W; ++e) {
                            const float pg = q > 0 ? s_sum[c + e] + ag[k][e] : ag[k][e];
                            const float pb = q > 0 ? s_sum[s.d + c + e] + ab[k][e] : ab[k][e];
                            if (q == groups - 1) {
                                out[c + e] = pg;
                                out[s.d + c + e] = pb;
                            } else {
                                s_sum[c + e] = pg;
                                s_sum[s.d + c + e] = pb;
                            }
                        }
                    }
                }
            }
            if (groups > 1) __syncthreads();
        }
    } else {
        for (int c = t0; c < s.d; c += step)
#pragma unroll
            for (int e = 0; e < W; ++e) out[c + e] = out[s.d + c + e] = 0.f;
        for (int64_t row = blockIdx.x; row < s.L; row += gridDim.x, par ^= 1) {
            const T *xr = x + row * s.x_ld, *gr = dy + row * s.g_ld;
            const float mu = __ldg(mean + row), rs = __ldg(rstd + row);
            float sums[2] = {0.f, 0.f};
            for (int c = t0; c < s.d; c += step) {
                float xv[W], gv[W], g[W];
                ln_load(xr + c, xv);
                ln_load(gr + c, gv);
                ln_weights<W>(gamma, c, g);
#pragma unroll
                for (int e = 0; e < W; ++e) {
                    const float xh = (xv[e] - mu) * rs, t = gv[e] * g[e];
                    out[c + e] = fmaf(gv[e], xh, out[c + e]);
                    out[s.d + c + e] += gv[e];
                    sums[0] += t;
                    sums[1] = fmaf(t, xh, sums[1]);
                }
            }
            ln_reduce<2>(sums, s.warps, wr, lane, grp, red[par] + grp * 64);
            const float c1 = sums[0] * s.inv_d, c2 = sums[1] * s.inv_d;
            for (int c = t0; c < s.d; c += step) {
                float xv[W], gv[W], g[W];
                ln_load(xr + c, xv);
                ln_load(gr + c, gv);
                ln_weights<W>(gamma, c, g);
#pragma unroll
                for (int e = 0; e < W; ++e) xv[e] = rs * (gv[e] * g[e] - fmaf((xv[e] - mu) * rs, c2, c1));
                ln_store(dx + row * s.y_ld + c, xv);
            }
        }
    }
}

// dgamma (blockIdx.y 0) and dbeta: 32 columns per block, its 16 warps each every 16th
// partial row, then the warps' sums in order.
constexpr int kLnSumWarps = 16;
__global__ void __launch_bounds__(32 * kLnSumWarps)
    ln_weight_sum_kernel(const float *__restrict__ part, int nparts, int d, float *dgamma, float *dbeta) {
    __shared__ float s_w[kLnSumWarps][32];
    griddep_wait();
    float *out = blockIdx.y == 0 ? dgamma : dbeta;
    if (!out) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int c = blockIdx.x * 32 + lane;
    float sum = 0.f;
    if (c < d) {
        const float *p = part + (int64_t)blockIdx.y * d + c;
#pragma unroll 4
        for (int q = warp; q < nparts; q += kLnSumWarps) sum += __ldcg(p + (int64_t)q * 2 * d);
    }
    s_w[warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && c < d) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < kLnSumWarps; ++w) t += s_w[w][lane];
        out[c] = t;
    }
}

// Warps per row, vectors per thread and rows per block for rows of `vecs` vectors.
// most: vectors per thread that the kernel is compiled for.
struct LnPlan {
    int warps, nv, groups;
};

static LnPlan ln_plan(int64_t L, int64_t vecs, int W, int most, bool backward, int sms) {
    LnPlan p{};
    // few rows: one vector per thread, so that a row's loads leave together; many:
    // up to `most`, which spends fewer instructions on reductions
    for (p.nv = 1;; p.nv *= 2) {
        const int64_t warps = cdiv(vecs, 32 * p.nv);
        const bool fits = warps <= (backward ? ln_backward_warps(W, p.nv) : 32);
        if (fits && (p.nv == most || L <= 8 * (int64_t)sms || warps <= 4)) break;
        if (p.nv == most) {
            p.nv = 0;
            break;
        }
    }
    p.warps = p.nv == 0 ? 32 : (int)cdiv(vecs, 32 * p.nv);
    p.groups = p.nv == 0 || p.warps > 4 ? 1 : 8 / p.warps;
    if (L < 2 * (int64_t)sms) p.groups = 1;
    return p;
}

// Blocks of the backward pass: a fixed function of the sizes, for the workspace.
static int64_t ln_blocks(int64_t L, int groups, int sms) {
    const int64_t most = std::min<int64_t>(4 * sms, kLnMaxBlocks);
    return std::max<int64_t>(1, std::min(cdiv(L, groups), most));
}

template <class T, int W>
static attt_status ln_forward_run(const T *x, const float *gamma, const float *beta, T *y, float *mean, float *rstd,
                                  LnShape s, int sms, cudaStream_t stream) {
    const LnPlan p = ln_plan(s.L, cdiv(s.d, W), W, W == 1 ? 8 : 4, false, sms);
    s.warps = p.warps;
    const dim3 grid((unsigned)cdiv(s.L, p.groups)), block(32 * p.warps * p.groups);
    switch (p.nv) {
        case 1: ln_forward_kernel<T, W, 1><<<grid, block, 0, stream>>>(x, gamma, beta, y, mean, rstd, s); break;
        case 2: ln_forward_kernel<T, W, 2><<<grid, block, 0, stream>>>(x, gamma, beta, y, mean, rstd, s); break;
        case 4: ln_forward_kernel<T, W, 4><<<grid, block, 0, stream>>>(x, gamma, beta, y, mean, rstd, s); break;
        case 8:
            if constexpr (W == 1)
                ln_forward_kernel<T, W, 8><<<grid, block, 0, stream>>>(x, gamma, beta, y, mean, rstd, s);
            break;
        default: ln_forward_kernel<T, W, 0><<<grid, block, 0, stream>>>(x, gamma, beta, y, mean, rstd, s); break;
    }
    count_launch();
    return cudaGetLastError() == cudaSuccess ? ATTT_OK : ATTT_ERR_CUDA;
}

template <class T, int W>
static attt_status ln_backward_run(const T *dy, const T *x, const float *gamma, const float *mean, const float *rstd,
                                   T *dx, float *dgamma, float *dbeta, float *part, LnShape s, int sms,
                                   cudaStream_t stream) {
    int64_t nparts = 0;
    if (s.L > 0) {
        const LnPlan p = ln_plan(s.L, cdiv(s.d, W), W, W == 8 ? 2 : W == 4 ? 4 : 8, true, sms);
        s.warps = p.warps;
        nparts = ln_blocks(s.L, p.groups, sms);
        const dim3 grid((unsigned)nparts), block(32 * p.warps * p.groups);
        const size_t smem = p.groups > 1 ? sizeof(float) * 2 * (size_t)s.d : 0;
        switch (p.nv) {
            case 1: ln_backward_kernel<T, W, 1><<<grid, block, smem, stream>>>(dy, x, gamma, mean, rstd, dx, part, s); break;
            case 2: ln_backward_kernel<T, W, 2><<<grid, block, smem, stream>>>(dy, x, gamma, mean, rstd, dx, part, s); break;
            case 4:
                if constexpr (W <= 4)
                    ln_backward_kernel<T, W, 4><<<grid, block, smem, stream>>>(dy, x, gamma, mean, rstd, dx, part, s);
                break;
            case 8:
                if constexpr (W == 1)
                    ln_backward_kernel<T, W, 8><<<grid, block, smem, stream>>>(dy, x, gamma, mean, rstd, dx, part, s);
                break;
            default: ln_backward_kernel<T, W, 0><<<grid, block, 0, stream>>>(dy, x, gamma, mean, rstd, dx, part, s); break;
        }
        count_launch();
        if (cudaGetLastError() != cudaSuccess) return ATTT_ERR_CUDA;
    }
    if (!dgamma && !dbeta) return ATTT_OK;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)cdiv(s.d, 32), 2);
    cfg.blockDim = dim3(32 * kLnSumWarps);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, ln_weight_sum_kernel, (const float *)part, (int)nparts, s.d, dgamma, dbeta) !=
        cudaSuccess)
        return ATTT_ERR_CUDA;
    count_launch();
    return cudaGetLastError() == cudaSuccess ? ATTT_OK : ATTT_ERR_CUDA;
}

static bool ln_sizes(int64_t L, int64_t d, int dtype) {
    return L >= 0 && d >= 1 && (dtype == ATTT_BF16 || dtype == ATTT_F32);
}

// Whether rows from p, `ld` elements apart, may be read 16 bytes at a time.
static bool ln_vector(const void *p, int64_t ld, int64_t d, size_t esize) {
    return aligned16(p) && ld * esize % 16 == 0 && d * esize % 16 == 0;
}

}  // namespace attt

extern "C" {

attt_status attt_layer_norm_forward(const void *d_x, int64_t x_ld, const float *d_gamma, const float *d_beta,
                                    int64_t L, int64_t d, float eps, int dtype, void *d_y, int64_t y_ld, float *d_mean,
                                    float *d_rstd, attt_stream stream) {
    ATTT_NVTX_RANGE();
    using namespace attt;
    if (!ln_sizes(L, d, dtype) || !(eps >= 0.f) || x_ld < d || y_ld < d) return ATTT_ERR_INVALID_ARG;
    if (!d_gamma || (L > 0 && (!d_x || !d_y))) return ATTT_ERR_INVALID_ARG;
    const size_t es = dtype == ATTT_BF16 ? 2 : 4;
    if (reinterpret_cast<uintptr_t>(d_x) % es || reinterpret_cast<uintptr_t>(d_y) % es) return ATTT_ERR_INVALID_ARG;
    if (L > (1ll << 31) - 1 || d > (1ll << 24) || x_ld > (1ll << 36) || y_ld > (1ll << 36)) return ATTT_ERR_UNSUPPORTED;
    if (L == 0) return ATTT_OK;
    int dev;
    const attt_status st = current_device(&dev);
    if (st != ATTT_OK) return st;
    LnShape s{};
    s.L = L; s.d = (int)d; s.x_ld = x_ld; s.y_ld = y_ld; s.eps = eps; s.inv_d = 1.f / (float)d;
    const bool vec = ln_vector(d_x, x_ld, d, es) && ln_vector(d_y, y_ld, d, es) && aligned16(d_gamma) &&
                     (!d_beta || aligned16(d_beta));
    const int sms = num_sms(dev);
    if (dtype == ATTT_BF16) {
        const auto *x = static_cast<const __nv_bfloat16 *>(d_x);
        auto *y = static_cast<__nv_bfloat16 *>(d_y);
        return vec ? ln_forward_run<__nv_bfloat16, 8>(x, d_gamma, d_beta, y, d_mean, d_rstd, s, sms, stream)
                   : ln_forward_run<__nv_bfloat16, 1>(x, d_gamma, d_beta, y, d_mean, d_rstd, s, sms, stream);
    }
    const auto *x = static_cast<const float *>(d_x);
    auto *y = static_cast<float *>(d_y);
    return vec ? ln_forward_run<float, 4>(x, d_gamma, d_beta, y, d_mean, d_rstd, s, sms, stream)
               : ln_forward_run<float, 1>(x, d_gamma, d_beta, y, d_mean, d_rstd, s, sms, stream);
}

size_t attt_layer_norm_workspace_bytes(int64_t L, int64_t d) {
    if (L < 0 || d < 1) return 0;
    const int64_t rows = std::max<int64_t>(1, std::min<int64_t>(L, attt::kLnMaxBlocks));
    return (size_t)attt::round_up(rows * 2 * d * (int64_t)sizeof(float), 256);
}

attt_status attt_layer_norm_backward(const void *d_dy, int64_t dy_ld, const void *d_x, int64_t x_ld,
                                     const float *d_gamma, const float *d_mean, const float *d_rstd, int64_t L,
                                     int64_t d, int dtype, void *d_dx, int64_t dx_ld, float *d_dgamma, float *d_dbeta,
                                     void *d_ws, size_t ws_bytes, attt_stream stream) {
    ATTT_NVTX_RANGE();
    using namespace attt;
    if (!ln_sizes(L, d, dtype) || dy_ld < d || x_ld < d || dx_ld < d) return ATTT_ERR_INVALID_ARG;
    if (!d_gamma || (L > 0 && (!d_dy || !d_x || !d_mean || !d_rstd || !d_dx))) return ATTT_ERR_INVALID_ARG;
    const size_t es = dtype == ATTT_BF16 ? 2 : 4;
    for (const void *p : {d_dy, d_x, (const void *)d_dx})
        if (reinterpret_cast<uintptr_t>(p) % es) return ATTT_ERR_INVALID_ARG;
    if (L > (1ll << 31) - 1 || d > (1ll << 24) || dy_ld > (1ll << 36) || x_ld > (1ll << 36) || dx_ld > (1ll << 36))
        return ATTT_ERR_UNSUPPORTED;
    if (!d_ws || !aligned256(d_ws) || ws_bytes < attt_layer_norm_workspace_bytes(L, d)) return ATTT_ERR_WORKSPACE;
    int dev;
    const attt_status st = current_device(&dev);
    if (st != ATTT_OK) return st;
    LnShape s{};
    s.L = L; s.d = (int)d; s.x_ld = x_ld; s.y_ld = dx_ld; s.g_ld = dy_ld; s.inv_d = 1.f / (float)d;
    const bool vec = ln_vector(d_x, x_ld, d, es) && ln_vector(d_dy, dy_ld, d, es) && ln_vector(d_dx, dx_ld, d, es) &&
                     aligned16(d_gamma);
    float *part = static_cast<float *>(d_ws);
    const int sms = num_sms(dev);
    if (dtype == ATTT_BF16) {
        const auto *x = static_cast<const __nv_bfloat16 *>(d_x), *dy = static_cast<const __nv_bfloat16 *>(d_dy);
        auto *dx = static_cast<__nv_bfloat16 *>(d_dx);
        return vec ? ln_backward_run<__nv_bfloat16, 8>(dy, x, d_gamma, d_mean, d_rstd, dx, d_dgamma, d_dbeta, part, s, sms, stream)
                   : ln_backward_run<__nv_bfloat16, 1>(dy, x, d_gamma, d_mean, d_rstd, dx, d_dgamma, d_dbeta, part, s, sms, stream);
    }
    const auto *x = static_cast<const float *>(d_x), *dy = static_cast<const float *>(d_dy);
    auto *dx = static_cast<float *>(d_dx);
    return vec ? ln_backward_run<float, 4>(dy, x, d_gamma, d_mean, d_rstd, dx, d_dgamma, d_dbeta, part, s, sms, stream)
               : ln_backward_run<float, 1>(dy, x, d_gamma, d_mean, d_rstd, dx, d_dgamma, d_dbeta, part, s, sms, stream);
}

}  // extern "C"

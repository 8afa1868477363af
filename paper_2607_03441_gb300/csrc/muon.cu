// muon.cu -- the adapters' step along orthogonalised momentum (K. Jordan et al.,
// "Muon: an optimizer for hidden layers in neural networks", 2024), for every
// projection of a call in one launch.
//
// For each matrix (A [din, r], B [r, dout]; n the width beside r) with gradient g and
// momentum m:
//   m <- mu m + g,  u = g + mu m (Nesterov) or m
//   X_0 = u / (|u|_F + eps);  X_{k+1} = (a I + b G_k + c G_k^2) X_k, G_k = X_k X_k^T
//   p <- p (1 - lr wd) - lr rms sqrt(max(rows, columns)) X_K
// G_k is taken on the r side, whichever side is longer: X f(X^T X) = f(X X^T) X.  With
// B_k = a I + b G_k + c G_k^2, two steps need one pass over X instead of two:
//   G_{k+1} = B_k G_k B_k,  X_{k+2} = (B_{k+1} B_k) X_k,
// r x r products otherwise (all symmetric and commuting).  Not more than two: small
// singular values are lost in a Gram matrix (relative to u^2, not u), and what a
// longer chain makes of that grows by 3.44^2 a step.  Off the 64-bit result (r 64,
// n 5,120, singular values over a factor of 100 / 10,000): all five steps on one Gram
// matrix 4.8e-5 / 1.7e-4, pairs 2e-6 / 5e-6, a Gram matrix per step 2e-6 / 8e-6.
// |u|_F^2 is the trace of the first one.
//
// A matrix belongs to one cluster; each CTA holds a range of columns in shared
// memory from the first read of g and m to the update of p (what does not fit
// goes through a workspace that stays in L2).  The CTAs' Gram matrices are summed
// through distributed shared memory in CTA order; at r > 32 each CTA forms a slab of
// rows of every r x r product and stores it to all of them, below that all form
// all of it, which takes less time than a barrier.  fp32 FMA throughout: the
// Gram matrices need their 24 bits.
// Bound: fp32 FMA issue at r 64 (6 r^2 n of them), barriers below.
#include <algorithm>
#include <cmath>

#include "attt_common.cuh"
#include "attt_host.h"

namespace attt {

constexpr int kMuonMats = 16;  // two per projection
constexpr int kMuonCols = 128;  // columns of a tile
constexpr int kMuonThreads = 512;
constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;

struct MuonMat {
    float *p, *m;
    const float *g;
    __nv_bfloat16 *p16;
    float *x;    // [n][RP], columns that do not stay in shared memory
    int64_t n;   // width beside r
    int64_t per; // columns of a CTA, a multiple of 8
    int tall;    // [n, r] (A), else [r, n] (B)
    float step;  // lr rms sqrt(max(rows, columns))
};

struct MuonArgs {
    MuonMat mat[kMuonMats];
    int r, nesterov, steps, slots, cluster;
    float mu, keep, eps;  // keep = 1 - lr wd
};

template <int RP>
struct MuonShape {
    static constexpr int LD = RP + 4;  // rows of 16-byte groups that start 4 banks apart
    static constexpr bool kSlabs = RP > 32;
    static constexpr int TJ = RP > 32 ? 8 : 4;                       // a thread's Gram tile: 4 x TJ
    static constexpr int kTiles = (RP / 4) * (RP / TJ);              // threads of a Gram matrix
    static constexpr int kSubs = kMuonThreads / kTiles;              // that many share the columns
    static constexpr int NC = RP * kMuonCols / 4 / kMuonThreads;     // a thread's product tile: NC columns x 4
    static constexpr int CL = kMuonCols / NC;
    static constexpr int kMat = RP * LD, kTile = kMuonCols * LD;     // floats
    static constexpr int kScratch = kSubs * RP * RP;
    // G, B, T over the scratch of the subsets' sums (never needed together); then the
    // CTA's part of the Gram matrix, two in turn where no barrier follows its reads
    static constexpr int kFirst = 3 * kMat > kScratch ? 3 * kMat : kScratch;
    static constexpr int kParts = kSlabs ? 1 : 2;
    static constexpr int kFixed = kFirst + kParts * RP * RP;
};

__device__ __forceinline__ float4 ld_cluster_f4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                 : "r"(addr)
                 : "memory");
    return v;
}

__device__ __forceinline__ void st_cluster_f4(uint32_t addr, float4 v) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(v.x), "f"(v.y), "f"(v.z),
                 "f"(v.w)
                 : "memory");
}

__device__ __forceinline__ float4 shfl_xor4(float4 v, int o) {
    return make_float4(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o),
                       __shfl_xor_sync(0xffffffffu, v.z, o), __shfl_xor_sync(0xffffffffu, v.w, o));
}

__device__ __forceinline__ float4 add4(float4 a, float4 b) {
    return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w);
}

// Calls f(at, c, k) for the elements of columns [0, cols) of the tile from c0: `at` the
// index in global memory, c < cols, k < r.  Threads of a warp take neighbours in
// memory whose places s[c][k] lie in different banks.
template <int RP, class F>
__device__ __forceinline__ void muon_elements(const MuonMat &t, int r, int64_t c0, int cols, F &&f) {
    if (t.tall) {
        for (int e = threadIdx.x; e < cols * r; e += kMuonThreads) {
            const int c = e / r;
            f(c0 * r + e, c, e - c * r);
        }
    } else {  // a warp: 8 columns x 4 rows
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, groups = (cols + 7) / 8;
        for (int b = warp; b < groups * (RP / 4); b += kMuonThreads / 32) {
            const int k = b / groups * 4 + (lane >> 3), c = b % groups * 8 + (lane & 7);
            if (k < r && c < cols) f(k * t.n + c0 + c, c, k);
        }
    }
}

// u of a tile into s (rows of r..RP stay 0), m updated when `first`.
template <int RP>
__device__ __forceinline__ void muon_load(const MuonArgs &a, const MuonMat &t, float *s, int64_t c0, int cols,
                                          bool first) {
    constexpr int LD = MuonShape<RP>::LD;
    if (a.r < RP)
        for (int e = threadIdx.x; e < cols * (RP - a.r); e += kMuonThreads)
            s[e / (RP - a.r) * LD + a.r + e % (RP - a.r)] = 0.f;
    muon_elements<RP>(t, a.r, c0, cols, [&](int64_t at, int c, int k) {
        const float g = __ldg(t.g + at);
        float m = t.m[at];
        if (first) {
            m = fmaf(a.mu, m, g);
            t.m[at] = m;
        }
        s[c * LD + k] = a.nesterov ? fmaf(a.mu, m, g) : m;
    });
}

// acc += the tile's columns' part of X X^T, this thread's 4 x TJ elements and its
// share of the columns.
template <int RP>
__device__ __forceinline__ void muon_gram(const float *s, int cols, float (&acc)[4][MuonShape<RP>::TJ]) {
    using S = MuonShape<RP>;
    const int tile = threadIdx.x % S::kTiles, sub = threadIdx.x / S::kTiles;
    const int i0 = tile / (RP / S::TJ) * 4, j0 = tile % (RP / S::TJ) * 4;
#pragma unroll 4
    for (int c = sub; c < cols; c += S::kSubs) {
        const float4 x = *reinterpret_cast<const float4 *>(s + c * S::LD + i0);
        const float xv[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int h = 0; h < S::TJ / 4; ++h) {  // columns j0 .. + 3 and, at TJ 8, j0 + RP / 2 ..
            const float4 y = *reinterpret_cast<const float4 *>(s + c * S::LD + j0 + h * (RP / 2));
            const float yv[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][4 * h + j] = fmaf(xv[i], yv[j], acc[i][4 * h + j]);
        }
    }
}

// The cluster's Gram matrix into G of every CTA, from the threads' shares.
template <int RP>
__device__ __forceinline__ void muon_gram_sum(const float (&acc)[4][MuonShape<RP>::TJ], float *scratch, float *part,
                                              float *G, int cluster, int rank) {
    using S = MuonShape<RP>;
    const int tile = threadIdx.x % S::kTiles, sub = threadIdx.x / S::kTiles;
    const int i0 = tile / (RP / S::TJ) * 4, j0 = tile % (RP / S::TJ) * 4;
    __syncthreads();  // scratch aliases matrices that other threads may still read
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int h = 0; h < S::TJ / 4; ++h)
            *reinterpret_cast<float4 *>(scratch + sub * RP * RP + (i0 + i) * RP + j0 + h * (RP / 2)) =
                make_float4(acc[i][4 * h], acc[i][4 * h + 1], acc[i][4 * h + 2], acc[i][4 * h + 3]);
    __syncthreads();
    for (int e = threadIdx.x; e < RP * RP / 4; e += kMuonThreads) {
        float4 v = *reinterpret_cast<const float4 *>(scratch + 4 * e);
        for (int k = 1; k < S::kSubs; ++k)
            v = add4(v, *reinterpret_cast<const float4 *>(scratch + k * RP * RP + 4 * e));
        *reinterpret_cast<float4 *>(part + 4 * e) = v;
    }
    cluster_sync();  // every part is there (and nobody reads the aliased matrices)
    const int rows = S::kSlabs ? RP / cluster : RP, outs = rows * RP / 4, subs = kMuonThreads / outs;
    const int o = threadIdx.x / subs, q = threadIdx.x % subs;
    const int i = (S::kSlabs ? rank * rows : 0) + o / (RP / 4), j = o % (RP / 4) * 4;
    const uint32_t src = smem_u32(part + i * RP + j);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int c = q; c < cluster; c += subs) v = add4(v, ld_cluster_f4(mapa_shared(src, c)));
    for (int s = 1; s < subs; s <<= 1) v = add4(v, shfl_xor4(v, s));
    if constexpr (S::kSlabs) {
        const uint32_t dst = smem_u32(G + i * S::LD + j);
        for (int c = q; c < cluster; c += subs) st_cluster_f4(mapa_shared(dst, c), v);
        cluster_sync();
    } else {
        if (q == 0) *reinterpret_cast<float4 *>(G + i * S::LD + j) = v;
        __syncthreads();
    }
}

// z = alpha x y (+ beta w) + diag I in every CTA, x and y symmetric and commuting, z
// none of the others.
template <int RP>
__device__ __forceinline__ void muon_product(const float *x, const float *y, float *z, float alpha, const float *w,
                                             float beta, float diag, int cluster, int rank) {
    using S = MuonShape<RP>;
    const int rows = S::kSlabs ? RP / cluster : RP, outs = rows * RP / 4, subs = kMuonThreads / outs;
    const int o = threadIdx.x / subs, q = threadIdx.x % subs;
    const int i = (S::kSlabs ? rank * rows : 0) + o / (RP / 4), j = o % (RP / 4) * 4;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int k = q; k < RP; k += subs) {
        const float xv = x[i * S::LD + k];
        const float4 yv = *reinterpret_cast<const float4 *>(y + k * S::LD + j);
        v.x = fmaf(xv, yv.x, v.x); v.y = fmaf(xv, yv.y, v.y);
        v.z = fmaf(xv, yv.z, v.z); v.w = fmaf(xv, yv.w, v.w);
    }
    for (int s = 1; s < subs; s <<= 1) v = add4(v, shfl_xor4(v, s));
    v.x *= alpha; v.y *= alpha; v.z *= alpha; v.w *= alpha;
    if (w) {
        const float4 u = *reinterpret_cast<const float4 *>(w + i * S::LD + j);
        v.x = fmaf(beta, u.x, v.x); v.y = fmaf(beta, u.y, v.y);
        v.z = fmaf(beta, u.z, v.z); v.w = fmaf(beta, u.w, v.w);
    }
    if (i == j) v.x += diag;
    if (i == j + 1) v.y += diag;
    if (i == j + 2) v.z += diag;
    if (i == j + 3) v.w += diag;
    if constexpr (S::kSlabs) {
        const uint32_t dst = smem_u32(z + i * S::LD + j);
        for (int c = q; c < cluster; c += subs) st_cluster_f4(mapa_shared(dst, c), v);
        cluster_sync();
    } else {
        if (q == 0) *reinterpret_cast<float4 *>(z + i * S::LD + j) = v;
        __syncthreads();
    }
}

// X <- P X for a tile, in place.
template <int RP>
__device__ __forceinline__ void muon_apply(float *s, const float *P, int cols) {
    using S = MuonShape<RP>;
    const int cl = threadIdx.x % S::CL, i0 = threadIdx.x / S::CL * 4;
    float acc[S::NC][4] = {};
#pragma unroll 4
    for (int k = 0; k < RP; k += 4) {
        float pv[4][4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float4 p = *reinterpret_cast<const float4 *>(P + (k + e) * S::LD + i0);
            pv[e][0] = p.x; pv[e][1] = p.y; pv[e][2] = p.z; pv[e][3] = p.w;
        }
#pragma unroll
        for (int n = 0; n < S::NC; ++n) {
            if (n * S::CL >= cols) break;  // block-uniform; rows past cols within are never read back
            const float4 x = *reinterpret_cast<const float4 *>(s + (cl + n * S::CL) * S::LD + k);
            const float xv[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[n][i] = fmaf(xv[e], pv[e][i], acc[n][i]);
        }
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < S::NC; ++n)
        if (cl + n * S::CL < cols)
            *reinterpret_cast<float4 *>(s + (cl + n * S::CL) * S::LD + i0) =
                make_float4(acc[n][0], acc[n][1], acc[n][2], acc[n][3]);
    __syncthreads();
}

template <int RP>
__global__ void __launch_bounds__(kMuonThreads, 1) muon_kernel(const __grid_constant__ MuonArgs a) {
    using S = MuonShape<RP>;
    extern __shared__ float4 s_raw[];
    float *G = reinterpret_cast<float *>(s_raw), *B = G + S::kMat, *T = B + S::kMat, *part = G + S::kFirst;
    float *tiles = G + S::kFixed;
    __shared__ float s_scale;
    const int rank = (int)cluster_ctarank();
    const MuonMat &t = a.mat[blockIdx.x / a.cluster];
    const int64_t c_begin = rank * t.per, c_end = min(t.n, c_begin + t.per);
    const int ntiles = c_end > c_begin ? (int)((c_end - c_begin + kMuonCols - 1) / kMuonCols) : 0;
    const int resident = ntiles <= a.slots ? ntiles : a.slots - 1;
    auto place = [&](int q) { return tiles + (q < resident ? q : a.slots - 1) * S::kTile; };
    auto first_col = [&](int q) { return c_begin + (int64_t)q * kMuonCols; };
    auto columns = [&](int q) { return (int)min((int64_t)kMuonCols, c_end - first_col(q)); };

    float acc[4][S::TJ] = {};
    for (int q = 0; q < ntiles; ++q) {
        if (q >= resident) __syncthreads();  // the place's last tile has been read
        muon_load<RP>(a, t, place(q), first_col(q), columns(q), true);
        if (q >= resident) {
            __syncthreads();
            muon_gram<RP>(place(q), columns(q), acc);
        }
    }
    __syncthreads();
    for (int q = 0; q < resident; ++q) muon_gram<RP>(place(q), columns(q), acc);

    const int groups = (a.steps + 1) / 2, single = a.steps % 2 ? groups / 2 : -1;  // pairs, the odd step amidst them
    for (int gi = 0; gi < groups; ++gi) {
        muon_gram_sum<RP>(acc, G, part + gi % S::kParts * RP * RP, G, a.cluster, rank);
        float scale = 1.f;
        if (gi == 0) {
            if (threadIdx.x < 32) {
                float v = 0.f;
                for (int i = threadIdx.x; i < RP; i += 32) v += G[i * S::LD + i];
                for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
                if (threadIdx.x == 0) s_scale = 1.f / (sqrtf(v) + a.eps);
            }
            __syncthreads();
            scale = s_scale;
            for (int e = threadIdx.x; e < RP * RP; e += kMuonThreads) {
                float &x = G[e / RP * S::LD + e % RP];
                x = x * scale * scale;
            }
            __syncthreads();
        }
        // B = a I + b G + c G^2, and for a pair of steps G <- B G B, P = (a I + b G + c G^2) B
        const float *P = B;
        muon_product<RP>(G, G, B, kNsC, G, kNsB, kNsA, a.cluster, rank);
        if (gi != single) {
            muon_product<RP>(B, G, T, 1.f, nullptr, 0.f, 0.f, a.cluster, rank);
            muon_product<RP>(T, B, G, 1.f, nullptr, 0.f, 0.f, a.cluster, rank);
            muon_product<RP>(G, G, T, kNsC, G, kNsB, kNsA, a.cluster, rank);
            muon_product<RP>(T, B, G, scale, nullptr, 0.f, 0.f, a.cluster, rank);
            P = G;
        } else if (gi == 0) {
            for (int e = threadIdx.x; e < RP * RP; e += kMuonThreads) B[e / RP * S::LD + e % RP] *= scale;
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < S::TJ; ++j) acc[i][j] = 0.f;
        const bool last = gi + 1 == groups;
        for (int q = 0; q < ntiles; ++q) {
            float *s = place(q);
            const int64_t c0 = first_col(q);
            const int cols = columns(q);
            if (q >= resident) {
                __syncthreads();
                if (gi == 0) {
                    muon_load<RP>(a, t, s, c0, cols, false);
                } else {
                    for (int e = threadIdx.x; e < cols * (RP / 4); e += kMuonThreads)
                        *reinterpret_cast<float4 *>(s + e / (RP / 4) * S::LD + e % (RP / 4) * 4) =
                            __ldcg(reinterpret_cast<const float4 *>(t.x + c0 * RP) + e);
                }
                __syncthreads();
            }
            muon_apply<RP>(s, P, cols);
            if (last) {
                muon_elements<RP>(t, a.r, c0, cols, [&](int64_t at, int c, int k) {
                    const float p = fmaf(-t.step, s[c * S::LD + k], t.p[at] * a.keep);
                    t.p[at] = p;
                    if (t.p16) t.p16[at] = __float2bfloat16_rn(p);
                });
            } else {
                muon_gram<RP>(s, cols, acc);
                if (q >= resident)
                    for (int e = threadIdx.x; e < cols * (RP / 4); e += kMuonThreads)
                        __stcg(reinterpret_cast<float4 *>(t.x + c0 * RP) + e,
                               *reinterpret_cast<const float4 *>(s + e / (RP / 4) * S::LD + e % (RP / 4) * 4));
            }
        }
    }
    cluster_sync();  // no CTA leaves while another reads its part
}

static int muon_rp(int r) { return r <= 16 ? 16 : r <= 32 ? 32 : 64; }

// Floats of the workspace: a row of RP per column, whether it is used or not.
static int64_t muon_columns(int nproj, const int64_t *din, const int64_t *dout) {
    int64_t n = 0;
    for (int i = 0; i < nproj; ++i) n += din[i] + dout[i];
    return n;
}

static bool muon_sizes(int nproj, const int64_t *din, const int64_t *dout, int r) {
    if (nproj < 1 || nproj > kMuonMats / 2 || !din || !dout || r < 1 || r > 64) return false;
    for (int i = 0; i < nproj; ++i)
        if (din[i] < 1 || dout[i] < 1 || din[i] > (1ll << 31) || dout[i] > (1ll << 31)) return false;
    return true;
}

template <int RP>
static attt_status muon_run(MuonArgs a, int nmat, int dev, cudaStream_t stream) {
    using S = MuonShape<RP>;
    constexpr size_t kMax = 232448 - 1024;  // 227 KB opt-in less the static part
    const void *kern = reinterpret_cast<const void *>(muon_kernel<RP>);
    const int most = (int)((kMax - sizeof(float) * S::kFixed) / (sizeof(float) * S::kTile));
    a.cluster = 8;
    int64_t per = 0;
    for (int i = 0; i < nmat; ++i) {
        a.mat[i].per = round_up(cdiv(a.mat[i].n, a.cluster), 8);
        per = std::max(per, a.mat[i].per);
    }
    a.slots = (int)std::min<int64_t>(most, cdiv(per, kMuonCols));
    const size_t smem = sizeof(float) * (S::kFixed + (size_t)a.slots * S::kTile);
    if (!set_smem_limit(kern, smem, dev)) return ATTT_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(nmat * a.cluster));
    cfg.blockDim = dim3(kMuonThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)a.cluster;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, muon_kernel<RP>, a) != cudaSuccess) return ATTT_ERR_CUDA;
    count_launch();
    return cudaGetLastError() == cudaSuccess ? ATTT_OK : ATTT_ERR_CUDA;
}

}  // namespace attt

extern "C" {

size_t attt_lora_muon_workspace_bytes(int nproj, const int64_t *din, const int64_t *dout, int r) {
    if (!attt::muon_sizes(nproj, din, dout, r)) return 0;
    return (size_t)attt::round_up(attt::muon_columns(nproj, din, dout) * attt::muon_rp(r) * 4, 256);
}

attt_status attt_lora_muon_step(int nproj, float *const *d_A32, float *const *d_B32, const float *const *d_dA,
                                const float *const *d_dB, float *const *d_mA, float *const *d_mB, const int64_t *din,
                                const int64_t *dout, int r, float lr, float momentum, int nesterov, float weight_decay,
                                float rms, float eps, int ns_steps, attt_bf16 *const *d_A16, attt_bf16 *const *d_B16,
                                void *d_ws, size_t ws_bytes, attt_stream stream) {
    ATTT_NVTX_RANGE();
    using namespace attt;
    if (!muon_sizes(nproj, din, dout, r) || !d_A32 || !d_B32 || !d_dA || !d_dB || !d_mA || !d_mB)
        return ATTT_ERR_INVALID_ARG;
    if (!(momentum >= 0.f && momentum < 1.f) || !(weight_decay >= 0.f) || !(rms > 0.f) || !(eps > 0.f) ||
        !std::isfinite(lr) || !std::isfinite(rms) || !std::isfinite(eps) || !std::isfinite(weight_decay) ||
        ns_steps < 1 || ns_steps > 16)
        return ATTT_ERR_INVALID_ARG;
    for (int i = 0; i < nproj; ++i)
        if (!d_A32[i] || !d_B32[i] || !d_dA[i] || !d_dB[i] || !d_mA[i] || !d_mB[i]) return ATTT_ERR_INVALID_ARG;
    if (!d_ws || !aligned256(d_ws) || ws_bytes < attt_lora_muon_workspace_bytes(nproj, din, dout, r))
        return ATTT_ERR_WORKSPACE;
    int dev;
    const attt_status st = current_device(&dev);
    if (st != ATTT_OK) return st;
    MuonArgs a{};
    a.r = r; a.nesterov = nesterov ? 1 : 0; a.steps = ns_steps;
    a.mu = momentum; a.keep = (float)(1.0 - (double)lr * weight_decay); a.eps = eps;
    float *x = static_cast<float *>(d_ws);
    for (int i = 0; i < 2 * nproj; ++i) {
        MuonMat &t = a.mat[i];
        const int p = i / 2;
        t.tall = i % 2 == 0;
        t.p = t.tall ? d_A32[p] : d_B32[p];
        t.g = t.tall ? d_dA[p] : d_dB[p];
        t.m = t.tall ? d_mA[p] : d_mB[p];
        attt_bf16 *const *h = t.tall ? d_A16 : d_B16;
        t.p16 = h ? reinterpret_cast<__nv_bfloat16 *>(h[p]) : nullptr;
        t.n = t.tall ? din[p] : dout[p];
        t.x = x;
        x += t.n * muon_rp(r);
        t.step = (float)((double)lr * rms * std::sqrt((double)std::max<int64_t>(t.n, r)));
    }
    return r <= 16 ? muon_run<16>(a, 2 * nproj, dev, stream)
         : r <= 32 ? muon_run<32>(a, 2 * nproj, dev, stream)
                   : muon_run<64>(a, 2 * nproj, dev, stream);
}

}  // extern "C"

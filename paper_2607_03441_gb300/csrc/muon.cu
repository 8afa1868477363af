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
// through distributed shared memory in CTA order: each CTA gets its slab of rows from
// all of them, sums, and gives it to all; up to r 16 each gets all of it from all.  At
// r > 32 the r x r products are formed in slabs too; below that one or two warps of
// every CTA form all of it, which takes less time than an exchange.  Exchanges are bulk
// copies between the CTAs' shared memories counted on mbarriers (measured at 8 / 12 to 16
// CTAs of 512 threads, 17 KB to each: 0.8 us; plain stores and a cluster barrier 1.1 /
// 1.6).  fp32 FMA throughout: the Gram matrices need their 24 bits.  Ranks up to 5 and
// (where the columns of every matrix of the call fit) of 33 to 64 have kernels of their
// own, below and in muon_tc.cu.
// Bound: fp32 FMA issue at r 64 (5 r^2 n of them), exchanges and launch below.  The step of
// q and v of 3,584 at r 16 (4 matrices, clusters of 16) takes 23 us, its bytes 0.6; of
// seven projections up to 18,944 wide 128 us at r 8, 386 at r 32 and, on this kernel for
// all of them, 1,170 at r 64.
#include <algorithm>
#include <array>
#include <cmath>
#include <functional>
#include <map>
#include <mutex>
#include <utility>

#include "muon.cuh"

namespace attt {

template <int RP>
struct MuonShape {
    static constexpr int LD = RP + 4;  // rows of 16-byte groups that start 4 banks apart
    static constexpr bool kSlabs = RP > 32;
    // A thread's Gram tile: 4 x TJ.  At r 64 a warp forms one of three 32 x 32 quadrants
    // (the fourth is the second's mirror image): 3 bank-conflict-free reads for 32 FMAs.
    static constexpr int TJ = RP > 32 ? 8 : 4;
    static constexpr int kTiles = RP > 32 ? 96 : (RP / 4) * (RP / 4);
    static constexpr int kSubs = kMuonThreads / kTiles;  // that many threads share a tile's columns
    static constexpr int CL = kMuonThreads / (RP / 8);   // product: columns at a time, 8 rows of X per thread
    static constexpr int kMat = RP * LD;                 // floats
    static constexpr int kScratch = kSubs * kTiles * 4 * TJ;
    // G, B, T over the scratch of the threads' sums (never needed together); the CTA's own
    // Gram matrix; what the others send of its slab of theirs
    static constexpr int kFirst = 3 * kMat > kScratch ? 3 * kMat : kScratch;
    // (cluster x rows of a slab, which are not even: up to RP + cluster rows)
    static constexpr int kRecv = (RP + kMuonMaxCluster) * LD;
    // this CTA's slab of the sum, to be sent (G itself is written again at once)
    static constexpr int kSlab = (RP / kMuonMinCluster) * LD;
    // RP 16: every CTA's whole matrix goes to all others, and one warp forms the products;
    // the matrix and what comes for two groups in turn
    static constexpr bool kWarp = RP == 16;
    static constexpr int kTurn = (1 + kMuonMaxCluster) * kMat;
    static constexpr int kFixed = kFirst + (kWarp ? 2 * kTurn : kMat + kRecv + kSlab);
    // Row and column of a Gram tile's first element.
    __device__ static __forceinline__ void tile(int t, int &i0, int &j0) {
        if constexpr (RP > 32) {
            const int quad = t / 32, lane = t % 32;
            i0 = (quad == 2 ? 32 : 0) + lane / 4 * 4;
            j0 = (quad >= 1 ? 32 : 0) + lane % 4 * 8;
        } else {
            i0 = t / (RP / 4) * 4;
            j0 = t % (RP / 4) * 4;
        }
    }
};

__device__ __forceinline__ float4 shfl_xor4(float4 v, int o) {
    return make_float4(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o),
                       __shfl_xor_sync(0xffffffffu, v.z, o), __shfl_xor_sync(0xffffffffu, v.w, o));
}

__device__ __forceinline__ float4 add4(float4 a, float4 b) {
    return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w);
}

// u of the columns into s (rows of r..RP stay 0), m updated when `first`.  (The passes over
// columns are functions of their own: inlined, what lives across them spills inside
// their loops.)
template <int RP, bool V4>
__device__ __forceinline__ void muon_load_as(const MuonArgs &a, const MuonMat &t, float *s, int64_t c0, int cols,
                                             bool first) {
    constexpr int LD = MuonShape<RP>::LD, W = V4 ? 4 : 1, U = V4 ? 3 : 6;
    const int64_t o = muon_origin(t, a.r, c0);
    const float *pg = t.g + o;
    float *pm = t.m + o;
    float g[U][W], m[U][W];
    muon_items<RP, LD, U, V4>(
        t, a.r, a.inv_r, cols,
        [&](int u, uint32_t at) {
            if constexpr (V4) {
                const float4 x = __ldg(reinterpret_cast<const float4 *>(pg + at));
                const float4 y = *reinterpret_cast<const float4 *>(pm + at);
                g[u][0] = x.x; g[u][1] = x.y; g[u][2] = x.z; g[u][3] = x.w;
                m[u][0] = y.x; m[u][1] = y.y; m[u][2] = y.z; m[u][3] = y.w;
            } else {
                g[u][0] = __ldg(pg + at);
                m[u][0] = pm[at];
            }
        },
        [&](int u, uint32_t at, int so) {
            if (first) {
#pragma unroll
                for (int w = 0; w < W; ++w) m[u][w] = fmaf(a.mu, m[u][w], g[u][w]);
                if constexpr (V4)
                    *reinterpret_cast<float4 *>(pm + at) = make_float4(m[u][0], m[u][1], m[u][2], m[u][3]);
                else
                    pm[at] = m[u][0];
            }
            if (a.nesterov)
#pragma unroll
                for (int w = 0; w < W; ++w) m[u][w] = fmaf(a.mu, m[u][w], g[u][w]);
            if (V4 && t.tall) {
                *reinterpret_cast<float4 *>(s + so) = make_float4(m[u][0], m[u][W / 4], m[u][W / 2], m[u][W - 1]);
            } else {
#pragma unroll
                for (int w = 0; w < W; ++w) s[so + w * LD] = m[u][w];
            }
        });
}

template <int RP>
__device__ __noinline__ void muon_load(const MuonArgs &a, const MuonMat &t, int s_at, int64_t c0, int cols,
                                       bool first) {
    constexpr int LD = MuonShape<RP>::LD;
    float *s = muon_smem(s_at);
    if (a.r < RP)
        for (int e = threadIdx.x; e < cols * (RP - a.r); e += kMuonThreads)
            s[e / (RP - a.r) * LD + a.r + e % (RP - a.r)] = 0.f;
    if (t.vec) muon_load_as<RP, true>(a, t, s, c0, cols, first);
    else muon_load_as<RP, false>(a, t, s, c0, cols, first);
}

// acc += the columns' part of X X^T, this thread's 4 x TJ elements and its share of the
// columns.
template <int RP>
__device__ __forceinline__ void muon_gram(const float *s, int cols, float (&acc)[4][MuonShape<RP>::TJ]) {
    using S = MuonShape<RP>;
    const int sub = threadIdx.x / S::kTiles;
    if (sub >= S::kSubs) return;
    int i0, j0;
    S::tile(threadIdx.x % S::kTiles, i0, j0);
#pragma unroll 2
    for (int c = sub; c < cols; c += S::kSubs) {
        const float4 x = *reinterpret_cast<const float4 *>(s + c * S::LD + i0);
        const float xv[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int h = 0; h < S::TJ / 4; ++h) {
            const float4 y = *reinterpret_cast<const float4 *>(s + c * S::LD + j0 + 4 * h);
            const float yv[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][4 * h + j] = fmaf(xv[i], yv[j], acc[i][4 * h + j]);
        }
    }
}

// The CTA's Gram matrix into `part`, from the threads' shares.
template <int RP>
__device__ __forceinline__ void muon_gram_part(const float (&acc)[4][MuonShape<RP>::TJ], float *scratch, float *part) {
    using S = MuonShape<RP>;
    constexpr int kVecs = S::kTiles * S::TJ;  // vectors of 4 of one set of tiles
    const int sub = threadIdx.x / S::kTiles, tile = threadIdx.x % S::kTiles;
    __syncthreads();  // scratch aliases matrices that other threads may still read
    if (sub < S::kSubs) {  // vector v of a tile at [v][tile]: neighbours write neighbours
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int h = 0; h < S::TJ / 4; ++h)
                *reinterpret_cast<float4 *>(scratch + 4 * (sub * kVecs + (i * (S::TJ / 4) + h) * S::kTiles + tile)) =
                    make_float4(acc[i][4 * h], acc[i][4 * h + 1], acc[i][4 * h + 2], acc[i][4 * h + 3]);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < kVecs; e += kMuonThreads) {
        float4 v = *reinterpret_cast<const float4 *>(scratch + 4 * e);
#pragma unroll 4
        for (int k = 1; k < S::kSubs; ++k) v = add4(v, *reinterpret_cast<const float4 *>(scratch + 4 * (k * kVecs + e)));
        int i, j;
        S::tile(e % S::kTiles, i, j);
        const int at = e / S::kTiles;
        i += at / (S::TJ / 4);
        j += at % (S::TJ / 4) * 4;
        *reinterpret_cast<float4 *>(part + i * S::LD + j) = v;
        if (RP > 32 && i < 32 && j >= 32) {
            part[j * S::LD + i] = v.x;
            part[(j + 1) * S::LD + i] = v.y;
            part[(j + 2) * S::LD + i] = v.z;
            part[(j + 3) * S::LD + i] = v.w;
        }
    }
}

// The cluster's Gram matrix into G of every CTA, from the threads' shares (exchanges n and
// n + 1).  `part`: kMat floats, `recv`: kRecv.
template <int RP>
__device__ __forceinline__ void muon_gram_sum(const float (&acc)[4][MuonShape<RP>::TJ], float *scratch, float *part,
                                              float *recv, float *G, const MuonLink &link, uint32_t n) {
    using S = MuonShape<RP>;
    muon_gram_part<RP>(acc, scratch, part);
    const int r0 = muon_row(RP, link.rank, link.cluster), r1 = muon_row(RP, link.rank + 1, link.cluster);
    float *const slab = recv + S::kRecv;
    link.gather<RP, S::LD>(n, part, recv, r0, r1, [&](int at, float4 v) {
        *reinterpret_cast<float4 *>(G + r0 * S::LD + at) = v;
        *reinterpret_cast<float4 *>(slab + at) = v;
    });
    link.share<S::LD>(n + 1, slab, G, r0, r1, RP);
}

// z = alpha x y (+ beta w, w_at >= 0) + diag I in every CTA, x and y symmetric and
// commuting, z none of the others; each CTA forms a slab of it (exchange n).
template <int RP>
__device__ __noinline__ void muon_product(int x_at, int y_at, int z_at, float alpha, int w_at, float beta, float diag,
                                          const MuonLink &link, uint32_t n) {
    using S = MuonShape<RP>;
    const float *x = muon_smem(x_at), *y = muon_smem(y_at), *w = w_at < 0 ? nullptr : muon_smem(w_at);
    float *z = muon_smem(z_at);
    const int r0 = muon_row(RP, link.rank, link.cluster), r1 = muon_row(RP, link.rank + 1, link.cluster);
    // threads per vector of 4 results: all of them, as far as a power of two allows
    const int subs = link.cluster >= 8 ? 4 : 2;
    const int o = threadIdx.x / subs, q = threadIdx.x % subs;
    const int i = r0 + o / (RP / 4), j = o % (RP / 4) * 4;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (i < r1) {
#pragma unroll 8
        for (int k = q; k < RP; k += subs) {
            const float xv = x[i * S::LD + k];
            const float4 yv = *reinterpret_cast<const float4 *>(y + k * S::LD + j);
            v.x = fmaf(xv, yv.x, v.x); v.y = fmaf(xv, yv.y, v.y);
            v.z = fmaf(xv, yv.z, v.z); v.w = fmaf(xv, yv.w, v.w);
        }
    }
    for (int s = 1; s < subs; s <<= 1) v = add4(v, shfl_xor4(v, s));
    if (i < r1 && q == 0) {
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
        *reinterpret_cast<float4 *>(z + i * S::LD + j) = v;
    }
    link.share<S::LD>(n, z + r0 * S::LD, z, r0, r1, RP);
}

// z = alpha x y (+ beta w, w_at >= 0) + diag I by one warp, x and y 16 x 16, symmetric and
// commuting, z none of the others.
__device__ __noinline__ void muon_warp_product(int x_at, int y_at, int z_at, float alpha, int w_at, float beta,
                                               float diag) {
    constexpr int LD = MuonShape<16>::LD;
    const int lane = threadIdx.x & 31, i = lane >> 1, j = (lane & 1) * 8;
    const float *x = muon_smem(x_at) + i * LD, *y = muon_smem(y_at) + j;
    float v[8] = {};
#pragma unroll
    for (int k = 0; k < 16; k += 4) {
        const float4 xk = *reinterpret_cast<const float4 *>(x + k);
        const float xe[4] = {xk.x, xk.y, xk.z, xk.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float4 a = *reinterpret_cast<const float4 *>(y + (k + e) * LD),
                         b = *reinterpret_cast<const float4 *>(y + (k + e) * LD + 4);
            v[0] = fmaf(xe[e], a.x, v[0]); v[1] = fmaf(xe[e], a.y, v[1]);
            v[2] = fmaf(xe[e], a.z, v[2]); v[3] = fmaf(xe[e], a.w, v[3]);
            v[4] = fmaf(xe[e], b.x, v[4]); v[5] = fmaf(xe[e], b.y, v[5]);
            v[6] = fmaf(xe[e], b.z, v[6]); v[7] = fmaf(xe[e], b.w, v[7]);
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        v[e] *= alpha;
        if (w_at >= 0) v[e] = fmaf(beta, muon_smem(w_at)[i * LD + j + e], v[e]);
        if (i == j + e) v[e] += diag;
    }
    float4 *z = reinterpret_cast<float4 *>(muon_smem(z_at) + i * LD + j);
    z[0] = make_float4(v[0], v[1], v[2], v[3]);
    z[1] = make_float4(v[4], v[5], v[6], v[7]);
    __syncwarp();
}

// The same by two warps, x and y 32 x 32: a thread has a tile of 4 x 4 (symmetric: row k of x
// is its column k), 2 vector reads for 16 FMAs.  q and v of 3,584 at r 32: 37 us, 45 with
// vectors of 4 by all threads, whose reads took longer than the sums.
__device__ __noinline__ void muon_two_product(int x_at, int y_at, int z_at, float alpha, int w_at, float beta,
                                              float diag) {
    constexpr int LD = MuonShape<32>::LD;
    const int i0 = threadIdx.x / 8 * 4, j0 = threadIdx.x % 8 * 4;
    const float *x = muon_smem(x_at) + i0, *y = muon_smem(y_at) + j0;
    float v[4][4] = {}, o[4][4] = {};  // even and odd k: half the length of a sum
#pragma unroll 4
    for (int k = 0; k < 32; k += 2) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float4 xk = *reinterpret_cast<const float4 *>(x + (k + h) * LD),
                         yk = *reinterpret_cast<const float4 *>(y + (k + h) * LD);
            const float xe[4] = {xk.x, xk.y, xk.z, xk.w}, ye[4] = {yk.x, yk.y, yk.z, yk.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) (h ? o : v)[i][j] = fmaf(xe[i], ye[j], (h ? o : v)[i][j]);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
        if (w_at >= 0) w = *reinterpret_cast<const float4 *>(muon_smem(w_at) + (i0 + i) * LD + j0);
        const float we[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[i][j] = fmaf(beta, we[j], (v[i][j] + o[i][j]) * alpha);
            if (i0 + i == j0 + j) v[i][j] += diag;
        }
        *reinterpret_cast<float4 *>(muon_smem(z_at) + (i0 + i) * LD + j0) = make_float4(v[i][0], v[i][1], v[i][2], v[i][3]);
    }
    named_barrier_sync(1, 64);
}

// One warp: exchange n (the CTAs' whole matrices, this one's at `turn`, the others' behind
// it), their sum in rank order and the group's products.  Both take a
// warp's time and not the block's: q and v of 3,584 at r 16 took 24.6 us with two
// exchanges (slabs of the sum) a group and products by all threads, 22.7 so.
__device__ __noinline__ void muon_warp_matrix(const MuonLink &link, uint32_t n, int turn, bool first, bool pair,
                                             float eps) {
    using S = MuonShape<16>;
    constexpr int oG = 0, oB = S::kMat, oT = 2 * S::kMat;
    constexpr uint32_t kBytes = 4 * S::kMat;
    const int lane = threadIdx.x & 31;
    float *const G = muon_smem(oG), *const part = muon_smem(turn), *const recv = part + S::kMat;
    if (lane == 0) link.expect(n, (uint32_t)(link.cluster - 1) * kBytes);
    if (lane < link.cluster && lane != link.rank && !link.lost())
        link.send(n, smem_u32(recv + link.rank * S::kMat), smem_u32(part), kBytes, lane);
    __syncwarp();
    link.receive(n);
    float trace = 0.f;
    float4 sum[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int e = lane + 32 * h, at = e / 4 * S::LD + e % 4 * 4;
        sum[h] = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int c = 0; c < link.cluster; ++c)
            sum[h] = add4(sum[h], *reinterpret_cast<const float4 *>((c == link.rank ? part : recv + c * S::kMat) + at));
        const int k = e / 4 - e % 4 * 4;  // the diagonal's place in the vector
        trace += k == 0 ? sum[h].x : k == 1 ? sum[h].y : k == 2 ? sum[h].z : k == 3 ? sum[h].w : 0.f;
    }
    float scale = 1.f;
    if (first) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) trace += __shfl_xor_sync(0xffffffffu, trace, o);
        scale = muon_scale(trace, eps);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int e = lane + 32 * h;
        *reinterpret_cast<float4 *>(G + e / 4 * S::LD + e % 4 * 4) =
            make_float4(sum[h].x * scale * scale, sum[h].y * scale * scale, sum[h].z * scale * scale,
                        sum[h].w * scale * scale);
    }
    __syncwarp();
    const float s0 = pair ? 1.f : scale;
    muon_warp_product(oG, oG, oB, kNsC * s0, oG, kNsB * s0, kNsA * s0);
    if (!pair) return;  // P is B
    muon_warp_product(oB, oG, oT, 1.f, -1, 0.f, 0.f);
    muon_warp_product(oT, oB, oG, 1.f, -1, 0.f, 0.f);
    muon_warp_product(oG, oG, oT, kNsC, oG, kNsB, kNsA);
    muon_warp_product(oT, oB, oG, scale, -1, 0.f, 0.f);  // P is over G
}

// X <- P X for NC x CL columns (`left` of them, more than (NC - 1) x CL), in place.
template <int RP, int NC>
__device__ __forceinline__ void muon_apply_columns(float *s, const float *P, int left) {
    using S = MuonShape<RP>;
    const int cl = threadIdx.x % S::CL, i0 = threadIdx.x / S::CL * 8;
    float acc[NC][8] = {};
    const float *p0 = P + i0, *x0 = s + cl * S::LD;
    // only the last of a thread's columns may lie past `left`: it then reads column 0
    const int last = cl + (NC - 1) * S::CL < left ? (NC - 1) * S::CL * S::LD : -cl * S::LD;
#pragma unroll 1
    for (int k = 0; k < RP; k += 4, p0 += 4 * S::LD, x0 += 4) {
        float4 x[NC];
#pragma unroll
        for (int n = 0; n < NC; ++n)
            x[n] = *reinterpret_cast<const float4 *>(x0 + (n == NC - 1 ? last : n * S::CL * S::LD));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float4 p = *reinterpret_cast<const float4 *>(p0 + e * S::LD);
            const float4 q = *reinterpret_cast<const float4 *>(p0 + e * S::LD + 4);
#pragma unroll
            for (int n = 0; n < NC; ++n) {
                const float v = e == 0 ? x[n].x : e == 1 ? x[n].y : e == 2 ? x[n].z : x[n].w;
                acc[n][0] = fmaf(v, p.x, acc[n][0]); acc[n][1] = fmaf(v, p.y, acc[n][1]);
                acc[n][2] = fmaf(v, p.z, acc[n][2]); acc[n][3] = fmaf(v, p.w, acc[n][3]);
                acc[n][4] = fmaf(v, q.x, acc[n][4]); acc[n][5] = fmaf(v, q.y, acc[n][5]);
                acc[n][6] = fmaf(v, q.z, acc[n][6]); acc[n][7] = fmaf(v, q.w, acc[n][7]);
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NC; ++n)
        if (cl + n * S::CL < left) {
            float *to = s + (cl + n * S::CL) * S::LD + i0;
            *reinterpret_cast<float4 *>(to) = make_float4(acc[n][0], acc[n][1], acc[n][2], acc[n][3]);
            *reinterpret_cast<float4 *>(to + 4) = make_float4(acc[n][4], acc[n][5], acc[n][6], acc[n][7]);
        }
}

template <int RP>
__device__ __noinline__ void muon_apply(int s_at, int p_at, int cols) {
    using S = MuonShape<RP>;
    float *s = muon_smem(s_at);
    const float *P = muon_smem(p_at);
    while (cols > 0) {  // even passes of at most 4 x CL columns
        const int units = (cols + S::CL - 1) / S::CL, passes = (units + 3) / 4, nc = (units + passes - 1) / passes;
        const int now = min(cols, nc * S::CL);
        if (nc == 4) muon_apply_columns<RP, 4>(s, P, now);
        else if (nc == 3) muon_apply_columns<RP, 3>(s, P, now);
        else if (nc == 2) muon_apply_columns<RP, 2>(s, P, now);
        else muon_apply_columns<RP, 1>(s, P, now);
        s += now * S::LD;
        cols -= now;
    }
    __syncthreads();
}

// STREAM: columns of a CTA may exceed what its shared memory holds.
template <int RP, bool STREAM>
__global__ void __launch_bounds__(kMuonThreads, 1) muon_kernel(const __grid_constant__ MuonArgs a) {
    using S = MuonShape<RP>;
    constexpr int oG = 0, oB = S::kMat, oT = 2 * S::kMat, oX = S::kFixed;
    float *const G = muon_smem(oG), *const B = muon_smem(oB), *const part = muon_smem(S::kFirst),
          *const recv = part + S::kMat, *const X = muon_smem(oX);
    __shared__ float s_scale;
    __shared__ __align__(8) uint64_t s_bars[2];
    __shared__ int s_abort;
    const int rank = (int)cluster_ctarank();
    const MuonMat &t = a.mat[blockIdx.x / a.cluster];
    const int64_t c_begin = rank * t.per, c_end = min(t.n, c_begin + t.per);
    const int64_t cols = c_end > c_begin ? c_end - c_begin : 0;
    // the first columns stay; the others pass through the last kMuonStage places
    const int stay = (int)(!STREAM || cols <= a.room ? cols : a.room - kMuonStage);
    const int o_stage = oX + (a.room - kMuonStage) * S::LD;
    float *const stage = muon_smem(o_stage);
    const MuonLink link{smem_u32(s_bars), a.cluster, rank, &s_abort, a.status};
    uint32_t n = 0;  // exchanges so far
    if (threadIdx.x == 0) {
        mbar_init(link.bar0, 1);
        mbar_init(link.bar0 + 8u, 1);
        s_abort = 0;
        fence_mbar_init();
    }
    muon_load<RP>(a, t, oX, c_begin, stay, true);
    cluster_sync();  // X is there, and the barriers of all CTAs

    float acc[4][S::TJ] = {};
    muon_gram<RP>(X, stay, acc);
    if constexpr (STREAM) {
        for (int64_t c = stay; c < cols; c += kMuonStage) {
            const int now = (int)min((int64_t)kMuonStage, cols - c);
            muon_load<RP>(a, t, o_stage, c_begin + c, now, true);
            __syncthreads();
            muon_gram<RP>(stage, now, acc);
            __syncthreads();
        }
    }

    const int groups = (a.steps + 1) / 2, single = a.steps % 2 ? groups / 2 : -1;  // pairs, the odd step amidst them
    for (int gi = 0; gi < groups; ++gi) {
        int oP = oB;
        if constexpr (S::kWarp) {
            // (two groups' places in turn: what a CTA sends for the next but one follows all that
            // the others sent for the next, and so their reading of this)
            const int turn = S::kFirst + (gi & 1) * S::kTurn;
            muon_gram_part<RP>(acc, G, muon_smem(turn));
            fence_proxy_async_smem();
            __syncthreads();
            if (threadIdx.x < 32) muon_warp_matrix(link, (uint32_t)gi, turn, gi == 0, gi != single, a.eps);
            if (gi != single) oP = oG;
            __syncthreads();
        } else {
            if (gi > 0) cluster_sync();  // every CTA has what this one's matrices were sent for
            muon_gram_sum<RP>(acc, G, part, recv, G, link, n);
            n += 2;
            float scale = 1.f;
            if (gi == 0) {
                if (threadIdx.x < 32) {
                    float v = 0.f;
                    for (int i = threadIdx.x; i < RP; i += 32) v += G[i * S::LD + i];
                    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
                    if (threadIdx.x == 0) s_scale = muon_scale(v, a.eps);
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
            // (a single first step takes the scale into B, as X_0 has it in u)
            const float s0 = gi == single ? scale : 1.f;
            if (gi != single) oP = oG;
            if constexpr (S::kSlabs) {
                muon_product<RP>(oG, oG, oB, kNsC * s0, oG, kNsB * s0, kNsA * s0, link, n++);
                if (gi != single) {
                    muon_product<RP>(oB, oG, oT, 1.f, -1, 0.f, 0.f, link, n++);
                    muon_product<RP>(oT, oB, oG, 1.f, -1, 0.f, 0.f, link, n++);
                    muon_product<RP>(oG, oG, oT, kNsC, oG, kNsB, kNsA, link, n++);
                    muon_product<RP>(oT, oB, oG, scale, -1, 0.f, 0.f, link, n++);
                }
            } else {
                if (threadIdx.x < 64) {
                    muon_two_product(oG, oG, oB, kNsC * s0, oG, kNsB * s0, kNsA * s0);
                    if (gi != single) {
                        muon_two_product(oB, oG, oT, 1.f, -1, 0.f, 0.f);
                        muon_two_product(oT, oB, oG, 1.f, -1, 0.f, 0.f);
                        muon_two_product(oG, oG, oT, kNsC, oG, kNsB, kNsA);
                        muon_two_product(oT, oB, oG, scale, -1, 0.f, 0.f);
                    }
                }
                __syncthreads();
            }
        }
        const bool last = gi + 1 == groups;
        muon_apply<RP>(oX, oP, stay);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < S::TJ; ++j) acc[i][j] = 0.f;
        if (last) muon_update<RP>(a, t, oX, c_begin, stay, link);
        else muon_gram<RP>(X, stay, acc);
        if constexpr (STREAM) {
            for (int64_t c = stay; c < cols; c += kMuonStage) {
                const int now = (int)min((int64_t)kMuonStage, cols - c);
                float4 *x = reinterpret_cast<float4 *>(t.x + (c_begin + c) * RP);
                if (gi == 0) {
                    muon_load<RP>(a, t, o_stage, c_begin + c, now, false);
                } else {
                    for (int e = threadIdx.x; e < now * (RP / 4); e += kMuonThreads)
                        *reinterpret_cast<float4 *>(stage + e / (RP / 4) * S::LD + e % (RP / 4) * 4) = __ldcg(x + e);
                }
                __syncthreads();
                muon_apply<RP>(o_stage, oP, now);
                if (last) {
                    muon_update<RP>(a, t, o_stage, c_begin + c, now, link);
                } else {
                    muon_gram<RP>(stage, now, acc);
                    for (int e = threadIdx.x; e < now * (RP / 4); e += kMuonThreads)
                        __stcg(x + e, *reinterpret_cast<const float4 *>(stage + e / (RP / 4) * S::LD + e % (RP / 4) * 4));
                }
                __syncthreads();
            }
        }
    }
    cluster_sync();  // no CTA leaves while it is sent to
}

// ---------------------------------------------------------------------------
// Ranks up to 5: matrices of no more elements than a warp has lanes.  With the Gram matrix
// in twice 24 bits (pairs of fp32: T. J. Dekker, "A floating-point technique for extending
// the available precision", 1971) nothing of the small singular values is lost, and every
// step is taken on that one matrix: X_K = P X_0 with P formed in 64 bits by one warp, lane
// i r + j its element i, j, and applied in pairs, since P has up to 3.44^K where X comes to
// 1.  One exchange (128 bytes from each CTA to each) instead of six.  Over 138 matrices of
// rank 4 the step is off the 64-bit one by 1.2e-7 as a rule and 3.7e-7 at most (the other
// ranks' kernel: 3.3e-7 and 1e-6; element by element in fp32: up to 7e-7).  Two projections
// of 3,584 at rank 5 take 16.5 us, 22.7 with the other ranks' kernel; seven of up to 5,120
// at rank 4 18.5, 28.8.  Bound: launch, load and update, and 64-bit FMA issue (a warp's
// takes some 60 cycles, which is why r 8 would gain nothing).
// ---------------------------------------------------------------------------

constexpr int kMuonLaneRank = 5, kMuonLaneSums = 16;  // 15 elements of a symmetric matrix, and one of 0

// The value h + l.
struct MuonPair {
    float h, l;
    __device__ __forceinline__ void add(float p, float e) {
        const float s = __fadd_rn(h, p), v = __fadd_rn(s, -h);
        l += __fadd_rn(__fadd_rn(h, -__fadd_rn(s, -v)), __fadd_rn(p, -v)) + e;
        h = s;
    }
    // + (ah + al) x
    __device__ __forceinline__ void add_product(float ah, float al, float x) {
        const float p = __fmul_rn(ah, x);
        add(p, __fmaf_rn(al, x, __fmaf_rn(ah, x, -p)));
    }
    __device__ __forceinline__ MuonPair shfl_xor(int o) const {
        return MuonPair{__shfl_xor_sync(0xffffffffu, h, o), __shfl_xor_sync(0xffffffffu, l, o)};
    }
};

// Place of element i <= j among the sums.
__host__ __device__ constexpr int muon_lane_sum(int i, int j) { return i * kMuonLaneRank - i * (i - 1) / 2 + j - i; }

struct MuonLaneShape {
    static constexpr int RP = 8, LD = RP + 4;
    static constexpr int oP = 0;                                   // 25 pairs
    static constexpr int oWarps = 64;                              // [warps][sums] pairs
    static constexpr int oOwn = oWarps + kMuonThreads / 32 * 2 * kMuonLaneSums;  // the CTA's sums
    static constexpr int oRecv = oOwn + 2 * kMuonLaneSums;         // the others'
    static constexpr int kFixed = oRecv + kMuonMaxCluster * 2 * kMuonLaneSums;
};
template <>
struct MuonShape<8> : MuonLaneShape {};

// Matrices in a warp's lanes.
__device__ __forceinline__ double muon_lane_product(double x, double y, int r, int i, int j) {
    double z = 0.;
#pragma unroll
    for (int k = 0; k < kMuonLaneRank; ++k) {
        const double a = __shfl_sync(0xffffffffu, x, (i * r + k) & 31), b = __shfl_sync(0xffffffffu, y, (k * r + j) & 31);
        if (k < r) z = fma(a, b, z);
    }
    return z;
}

__device__ __forceinline__ void muon_lane_gram(const float *s, int cols, MuonPair (&acc)[kMuonLaneSums]) {
    for (int c = threadIdx.x; c < cols; c += kMuonThreads) {
        const float4 a = *reinterpret_cast<const float4 *>(s + c * MuonLaneShape::LD);
        const float x[kMuonLaneRank] = {a.x, a.y, a.z, a.w, s[c * MuonLaneShape::LD + 4]};
#pragma unroll
        for (int i = 0; i < kMuonLaneRank; ++i)
#pragma unroll
            for (int j = i; j < kMuonLaneRank; ++j) acc[muon_lane_sum(i, j)].add_product(x[i], 0.f, x[j]);
    }
}

__device__ __forceinline__ void muon_lane_apply(float *s, int cols) {
    const float2 *p = reinterpret_cast<const float2 *>(muon_smem(MuonLaneShape::oP));
    for (int c = threadIdx.x; c < cols; c += kMuonThreads) {
        float4 *at = reinterpret_cast<float4 *>(s + c * MuonLaneShape::LD);
        const float4 a = *at;
        const float x[kMuonLaneRank] = {a.x, a.y, a.z, a.w, s[c * MuonLaneShape::LD + 4]};
        float y[kMuonLaneRank];
#pragma unroll
        for (int i = 0; i < kMuonLaneRank; ++i) {
            MuonPair v{0.f, 0.f};
#pragma unroll
            for (int k = 0; k < kMuonLaneRank; ++k) {
                const float2 q = p[i * kMuonLaneRank + k];
                v.add_product(q.x, q.y, x[k]);
            }
            y[i] = v.h + v.l;
        }
        *at = make_float4(y[0], y[1], y[2], y[3]);
        s[c * MuonLaneShape::LD + 4] = y[4];
    }
}

// One warp: the cluster's Gram matrix from the CTAs' sums, in rank order, and P (0 past r).
__device__ __noinline__ void muon_lane_matrix(const MuonArgs &a, int rank) {
    using S = MuonLaneShape;
    const int lane = threadIdx.x & 31, r = a.r, e = min(lane, r * r - 1), i = e / r, j = e - i * r;
    const float2 *own = reinterpret_cast<const float2 *>(muon_smem(S::oOwn)),
                 *recv = reinterpret_cast<const float2 *>(muon_smem(S::oRecv));
    MuonPair sum{0.f, 0.f};
    for (int c = 0; c < a.cluster; ++c) {
        const float2 q = c == rank ? own[lane & 15] : recv[c * kMuonLaneSums + (lane & 15)];
        sum.add(q.x, q.y);
    }
    double g = __shfl_sync(0xffffffffu, (double)sum.h + (double)sum.l, muon_lane_sum(min(i, j), max(i, j)));
    double v = 0.;
    for (int k = 0; k < r; ++k) v += __shfl_sync(0xffffffffu, g, k * (r + 1));
    // (as muon_scale: beyond fp32 NaN, although this sum would hold it)
    const double scale = v <= (double)FLT_MAX ? 1. / (sqrt(v) + (double)a.eps) : __longlong_as_double(0x7ff8000000000000ll);
    const double diag = i == j ? kNsA64 : 0.;
    g *= scale * scale;
    double p = i == j ? scale : 0.;
    for (int k = 0; k < a.steps; ++k) {
        const double b = fma(kNsC64, muon_lane_product(g, g, r, i, j), fma(kNsB64, g, diag));
        p = k == 0 ? b * scale : muon_lane_product(b, p, r, i, j);
        if (k + 1 < a.steps) g = muon_lane_product(muon_lane_product(b, g, r, i, j), b, r, i, j);
    }
    float2 *out = reinterpret_cast<float2 *>(muon_smem(S::oP));
    if (lane < kMuonLaneRank * kMuonLaneRank) out[lane] = make_float2(0.f, 0.f);
    __syncwarp();
    const float h = (float)p;
    if (lane < r * r) out[i * kMuonLaneRank + j] = make_float2(h, (float)(p - (double)h));
}

template <bool STREAM>
__global__ void __launch_bounds__(kMuonThreads, 1) muon_lane_kernel(const __grid_constant__ MuonArgs a) {
    using S = MuonLaneShape;
    constexpr int RP = S::RP, oX = S::kFixed;
    __shared__ __align__(8) uint64_t s_bars[2];
    __shared__ int s_abort;
    float *const X = muon_smem(oX);
    const int rank = (int)cluster_ctarank(), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const MuonMat &t = a.mat[blockIdx.x / a.cluster];
    const int64_t c_begin = rank * t.per, c_end = min(t.n, c_begin + t.per);
    const int64_t cols = c_end > c_begin ? c_end - c_begin : 0;
    // the first columns stay; the others pass through the last kMuonStage places, twice
    const int stay = (int)(!STREAM || cols <= a.room ? cols : a.room - kMuonStage);
    const int o_stage = oX + (a.room - kMuonStage) * S::LD;
    float *const stage = muon_smem(o_stage);
    const MuonLink link{smem_u32(s_bars), a.cluster, rank, &s_abort, a.status};
    if (threadIdx.x == 0) {
        mbar_init(link.bar0, 1);
        mbar_init(link.bar0 + 8u, 1);
        s_abort = 0;
        fence_mbar_init();
    }
    muon_load<RP>(a, t, oX, c_begin, stay, true);
    cluster_sync();  // X is there, and the barriers of all CTAs
    MuonPair acc[kMuonLaneSums];
#pragma unroll
    for (int i = 0; i < kMuonLaneSums; ++i) acc[i] = MuonPair{0.f, 0.f};
    muon_lane_gram(X, stay, acc);
    if constexpr (STREAM) {
        for (int64_t c = stay; c < cols; c += kMuonStage) {
            const int now = (int)min((int64_t)kMuonStage, cols - c);
            muon_load<RP>(a, t, o_stage, c_begin + c, now, true);
            __syncthreads();
            muon_lane_gram(stage, now, acc);
            __syncthreads();
        }
    }
    // the warp's sums: with every exchange half as many in a lane, each of twice as many lanes,
    // until lanes 2 e and 2 e + 1 hold sum e
#pragma unroll
    for (int o = 16, n = 8; n > 0; o >>= 1, n >>= 1) {
        const bool up = lane & o;
#pragma unroll
        for (int k = 0; k < n; ++k) {
            const MuonPair mine = up ? acc[k + n] : acc[k], other = (up ? acc[k] : acc[k + n]).shfl_xor(o);
            acc[k] = mine;
            acc[k].add(other.h, other.l);
        }
    }
    const MuonPair other = acc[0].shfl_xor(1);
    float2 *const warps = reinterpret_cast<float2 *>(muon_smem(S::oWarps));
    // both lanes in the same order
    MuonPair sum = lane & 1 ? other : acc[0];
    const MuonPair second = lane & 1 ? acc[0] : other;
    sum.add(second.h, second.l);
    if ((lane & 1) == 0) warps[warp * kMuonLaneSums + (lane >> 1)] = make_float2(sum.h, sum.l);
    __syncthreads();
    if (warp == 0) {
        sum = MuonPair{0.f, 0.f};
#pragma unroll 4
        for (int w = 0; w < kMuonThreads / 32; ++w) {
            const float2 q = warps[w * kMuonLaneSums + (lane & 15)];
            sum.add(q.x, q.y);
        }
        constexpr uint32_t kBytes = 8 * kMuonLaneSums;
        float *const own = muon_smem(S::oOwn);
        if (lane < kMuonLaneSums) reinterpret_cast<float2 *>(own)[lane] = make_float2(sum.h, sum.l);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) link.expect(0, (uint32_t)(a.cluster - 1) * kBytes);
        if (lane < a.cluster && lane != rank)
            link.send(0, smem_u32(muon_smem(S::oRecv) + rank * 2 * kMuonLaneSums), smem_u32(own), kBytes, lane);
        __syncwarp();
        link.receive(0);
        muon_lane_matrix(a, rank);
    }
    __syncthreads();
    muon_lane_apply(X, stay);
    __syncthreads();
    muon_update<RP>(a, t, oX, c_begin, stay, link);
    if constexpr (STREAM) {
        for (int64_t c = stay; c < cols; c += kMuonStage) {
            const int now = (int)min((int64_t)kMuonStage, cols - c);
            muon_load<RP>(a, t, o_stage, c_begin + c, now, false);
            __syncthreads();
            muon_lane_apply(stage, now);
            __syncthreads();
            muon_update<RP>(a, t, o_stage, c_begin + c, now, link);
            __syncthreads();
        }
    }
    cluster_sync();  // no CTA leaves while it is sent to
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
        if (din[i] < 1 || dout[i] < 1 || din[i] > (1ll << 25) || dout[i] > (1ll << 25)) return false;
    return true;
}

// Whether no two of a call's arrays start at the same place, but for gradients, which are
// only read.
static bool muon_apart(int nproj, float *const *A32, float *const *B32, const float *const *dA,
                       const float *const *dB, float *const *mA, float *const *mB, attt_bf16 *const *A16,
                       attt_bf16 *const *B16) {
    const void *written[3 * kMuonMats];
    int n = 0;
    for (int i = 0; i < nproj; ++i)
        for (const void *p : {(const void *)A32[i], (const void *)B32[i], (const void *)mA[i], (const void *)mB[i],
                              (const void *)(A16 ? A16[i] : nullptr), (const void *)(B16 ? B16[i] : nullptr)})
            if (p) written[n++] = p;
    std::sort(written, written + n, std::less<const void *>());
    if (std::adjacent_find(written, written + n) != written + n) return false;
    for (int i = 0; i < nproj; ++i)
        for (const void *p : {(const void *)dA[i], (const void *)dB[i]})
            if (std::binary_search(written, written + n, p, std::less<const void *>())) return false;
    return true;
}

bool muon_clusters(const void *kern, size_t smem, int dev, int (&most)[kMuonMaxCluster + 1]) {
    static std::mutex mu;
    static std::map<std::pair<const void *, int>, std::array<int, kMuonMaxCluster + 1>> known;
    std::lock_guard<std::mutex> lock(mu);
    const auto key = std::make_pair(kern, dev);
    auto it = known.find(key);
    if (it == known.end()) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return false;
        std::array<int, kMuonMaxCluster + 1> n{};
        for (int c = kMuonMinCluster; c <= kMuonMaxCluster; ++c) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3((unsigned)(kMuonMats * c));
            cfg.blockDim = dim3(kMuonThreads);
            cfg.dynamicSmemBytes = smem;
            cudaLaunchAttribute attr[1];
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim.x = (unsigned)c;
            attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
            cfg.attrs = attr;
            cfg.numAttrs = 1;
            if (cudaOccupancyMaxActiveClusters(&n[c], kern, &cfg) != cudaSuccess) {
                n[c] = 0;
                (void)cudaGetLastError();
            }
        }
        it = known.emplace(key, n).first;
    }
    std::copy(it->second.begin(), it->second.end(), most);
    return true;
}

int muon_cluster(const int (&most)[kMuonMaxCluster + 1], int nmat, int64_t n, int64_t room, int64_t *cost) {
    int best = 0;
    for (int c = kMuonMinCluster; c <= kMuonMaxCluster; ++c) {
        const int64_t per = round_up(cdiv(n, c), 8);
        if (most[c] < 1 || (room > 0 && per > room)) continue;
        const int64_t now = cdiv(nmat, most[c]) * per;
        if (best == 0 || now < *cost) {
            *cost = now;
            best = c;
        }
    }
    return best;
}

attt_status muon_launch(const void *kern, MuonArgs &a, int nmat, size_t smem, cudaStream_t stream) {
    for (int i = 0; i < nmat; ++i) a.mat[i].per = round_up(cdiv(a.mat[i].n, a.cluster), 8);
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
    void *args[] = {&a};
    if (cudaLaunchKernelExC(&cfg, kern, args) != cudaSuccess) return ATTT_ERR_CUDA;
    count_launch();
    return cudaGetLastError() == cudaSuccess ? ATTT_OK : ATTT_ERR_CUDA;
}

template <int RP>
static attt_status muon_run(MuonArgs a, int nmat, int dev, cudaStream_t stream) {
    using S = MuonShape<RP>;
    constexpr size_t kMax = 232448 - 1024;  // 227 KB opt-in less the static part
    const void *kerns[2];
    if constexpr (RP == 8) {
        kerns[0] = reinterpret_cast<const void *>(muon_lane_kernel<false>);
        kerns[1] = reinterpret_cast<const void *>(muon_lane_kernel<true>);
    } else {
        kerns[0] = reinterpret_cast<const void *>(muon_kernel<RP, false>);
        kerns[1] = reinterpret_cast<const void *>(muon_kernel<RP, true>);
    }
    a.room = (int)((kMax - sizeof(float) * S::kFixed) / (sizeof(float) * S::LD)) / 8 * 8;
    const size_t smem = sizeof(float) * (S::kFixed + (size_t)a.room * S::LD);
    int most[2][kMuonMaxCluster + 1];
    for (int k = 0; k < 2; ++k)
        if (!set_smem_limit(kerns[k], smem, dev) || !muon_clusters(kerns[k], smem, dev, most[k])) return ATTT_ERR_CUDA;
    int64_t n = 0, cost = 0;
    for (int i = 0; i < nmat; ++i) n = std::max(n, a.mat[i].n);
    a.cluster = muon_cluster(most[0], nmat, n, 0, &cost);
    if (a.cluster == 0) return ATTT_ERR_CUDA;
    return muon_launch(kerns[round_up(cdiv(n, a.cluster), 8) <= a.room ? 0 : 1], a, nmat, smem, stream);
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
    if (!(momentum >= 0.f && momentum < 1.f) || !(weight_decay >= 0.f) || !(rms > 0.f) || !(eps >= kMuonMinEps) ||
        !std::isfinite(lr) || !std::isfinite(rms) || !std::isfinite(eps) || !std::isfinite(weight_decay) ||
        ns_steps < 1 || ns_steps > 16)
        return ATTT_ERR_INVALID_ARG;
    for (int i = 0; i < nproj; ++i)
        if (!d_A32[i] || !d_B32[i] || !d_dA[i] || !d_dB[i] || !d_mA[i] || !d_mB[i] ||
            !aligned_to(4, d_A32[i], d_B32[i], d_dA[i], d_dB[i], d_mA[i], d_mB[i]) ||
            !aligned_to(2, d_A16 ? d_A16[i] : nullptr, d_B16 ? d_B16[i] : nullptr))
            return ATTT_ERR_INVALID_ARG;
    if (!muon_apart(nproj, d_A32, d_B32, d_dA, d_dB, d_mA, d_mB, d_A16, d_B16)) return ATTT_ERR_INVALID_ARG;
    if (!d_ws || !aligned256(d_ws) || ws_bytes < attt_lora_muon_workspace_bytes(nproj, din, dout, r))
        return ATTT_ERR_WORKSPACE;
    int dev;
    const attt_status st = current_device(&dev);
    if (st != ATTT_OK) return st;
    MuonArgs a{};
    int *status = device_status_word(dev);
    if (!status) return ATTT_ERR_CUDA;
    a.r = r; a.nesterov = nesterov ? 1 : 0; a.steps = ns_steps;
    a.inv_r = r > 1 ? (uint32_t)(((1ull << 32) + r - 1) / r) : 0u; a.status = status;
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
        t.vec = (t.tall ? r : t.n) % 4 == 0 && aligned16(t.p) && aligned16(t.g) && aligned16(t.m) &&
                reinterpret_cast<uintptr_t>(t.p16) % 8 == 0;
        t.x = x;
        x += t.n * muon_rp(r);
        t.step = (float)((double)lr * rms * std::sqrt((double)std::max<int64_t>(t.n, r)));
    }
    if (r > 32) {
        bool done = false;
        const attt_status tc = muon_tc_run(a, 2 * nproj, dev, stream, &done);
        if (done || tc != ATTT_OK) return tc;
    }
    if (r <= kMuonLaneRank) return muon_run<8>(a, 2 * nproj, dev, stream);
    return r <= 16 ? muon_run<16>(a, 2 * nproj, dev, stream)
         : r <= 32 ? muon_run<32>(a, 2 * nproj, dev, stream)
                   : muon_run<64>(a, 2 * nproj, dev, stream);
}

}  // extern "C"

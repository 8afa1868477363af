// muon_tc.cu -- the Muon step (muon.cu) for ranks of 33 to 64, with its products on the
// tensor cores.  Same formulas, same clusters, same pairs of steps on one Gram matrix.
//
// fp32 values are split into three bf16 each, x = h + m + l (8 + 8 + 8 bits, exact), and
// a product of two matrices is six of theirs, l h + h l + m m + m h + h m + h h, the small
// ones first: what is left out is below 2^-24 of |x| |y|, and what the accumulators
// truncate is of the order of an fp32 sum's rounding (updates 0.6e-6 to 1.5e-6 off for ranks
// of 33 to 64, 3,000 columns and singular values over a factor of 1 to 100; the plain steps
// in fp32 1.1e-6 to 2.6e-6).
//
// A CTA's columns of X are kept as three tiles of [column][64] bf16 (128-byte rows,
// 128-byte swizzle).  Read with the rank along K they are the A operand of X <- P X
// (128 columns on M, P on N); read with the columns along K they are both operands of
// the Gram matrix (rank on M and N).  M is 128 throughout: where a matrix has 64 rows the
// other 64 are whatever follows in shared memory, and their results, in the upper
// TMEM lanes, are never read.  The r x r products are formed by every CTA on its own
// (1.4 us each; in slabs with an exchange they took 2.1 in muon.cu), so that only the
// Gram matrices travel.  They are formed without a multiple of I: with M = m I + M', m from
// the mean of G's diagonal, x y is x'y' by the MMAs and x y' + x'y + x y I in fp32.  An MMA
// cuts off what its smaller products have below the last bit of its largest, always towards
// zero, so that a diagonal far above the rest loses some of its own sum in every product:
// products of the whole matrices left X off by up to 9e-6 where the singular values are alike.
// Why: on CUDA cores the products were bound by the 128 bytes that shared memory returns
// per cycle (a 4 x 8 tile per thread: 128 FMAs per 12 vector reads).  The step of q, k, v
// and o of 5,120 at r 64 (8 matrices, clusters of 12) takes 67 us, 121 with muon.cu's
// kernel; its bytes would take 7.  Bound: a chain of loads, three Gram matrices with two
// exchanges of 0.8 us each, eleven r x r products (with these some 20 us), three products
// with X and the update; how the rest is shared among its links was not measured.
#include <algorithm>

#include "muon.cuh"

namespace attt {

constexpr int kTcCols = 432;                          // columns of a CTA at most, a multiple of an MMA's 16
constexpr uint32_t kTcSplit = kTcCols * 128u;         // bytes of one of X's tiles
constexpr uint32_t kTcMat = 64 * 128u;                // of one of an r x r matrix's
constexpr uint32_t kTcTmem = 512;
constexpr uint32_t kTcPoly = 256, kTcGram = 320;      // TMEM columns of the r x r products (64), the Gram matrix (192)
// fp32 matrices for the exchanges, in floats, over two r x r matrices' tiles; rows of 68:
// vectors of 8 neighbouring rows then lie in different banks
constexpr int kTcLD = 68;
constexpr int kTcPart = 0, kTcRecv = 64 * kTcLD, kTcG = kTcRecv + (64 + kMuonMaxCluster) * kTcLD;
constexpr int kTcSlab = kTcG + 64 * kTcLD;            // beside the tiles: outgoing copies may still read it
constexpr uint32_t kTcRest = (kTcSlab + 64 / kMuonMinCluster * kTcLD) * 4u;
static_assert(kTcSlab * 4u >= 6 * kTcMat && kTcRest >= 7 * kTcMat, "two matrices of three tiles, and a seventh to overrun");
static_assert(kTcCols % 16 == 0 && kTcSplit % 1024 == 0 && kTcCols * 68 * 4 <= 3 * kTcSplit, "");
constexpr size_t kTcSmem = 1024 + 3 * kTcSplit + kTcRest;
static_assert(kTcCols / 128 * 128 + 128 <= 512 && (512 - kTcCols) * 128 <= (int)kTcRest, "the last tile of 128 columns stays in bounds");

// Three bf16 whose sum is x, two values at a time, packed.
struct Split2 {
    uint32_t h, m, l;
};
__device__ __forceinline__ Split2 split2(float a, float b) {
    Split2 s;
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    const float2 hf = __bfloat1622float2(h);
    a -= hf.x;
    b -= hf.y;
    const __nv_bfloat162 m = __floats2bfloat162_rn(a, b);
    const float2 mf = __bfloat1622float2(m);
    const __nv_bfloat162 l = __floats2bfloat162_rn(a - mf.x, b - mf.y);
    s.h = *reinterpret_cast<const uint32_t *>(&h);
    s.m = *reinterpret_cast<const uint32_t *>(&m);
    s.l = *reinterpret_cast<const uint32_t *>(&l);
    return s;
}

// Byte of element k of a 128-byte row c of a swizzled tile.
__device__ __forceinline__ uint32_t tc_at(int c, int k) {
    return (uint32_t)c * 128u + (((((uint32_t)k * 2u) >> 4) ^ ((uint32_t)c & 7u)) << 4) + (((uint32_t)k * 2u) & 15u);
}

__device__ __forceinline__ void st_shared_v2(uint32_t addr, uint32_t a, uint32_t b) {
    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(addr), "r"(a), "r"(b) : "memory");
}
__device__ __forceinline__ void st_shared_u16(uint32_t addr, uint32_t a) {
    asm volatile("st.shared.u16 [%0], %1;" ::"r"(addr), "h"((unsigned short)a) : "memory");
}

// Four neighbours k .. k + 3 (k a multiple of 4) of row c into the three tiles at `base`,
// `stride` bytes apart.
__device__ __forceinline__ void tc_put4(uint32_t base, uint32_t stride, int c, int k, float4 v) {
    const Split2 a = split2(v.x, v.y), b = split2(v.z, v.w);
    const uint32_t at = base + tc_at(c, k);
    st_shared_v2(at, a.h, b.h);
    st_shared_v2(at + stride, a.m, b.m);
    st_shared_v2(at + 2 * stride, a.l, b.l);
}

// 16 neighbours k .. k + 15 (a multiple of 16) of row c.
__device__ __forceinline__ void tc_put16(uint32_t base, uint32_t stride, int c, int k, const float (&v)[16]) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        Split2 s[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = split2(v[8 * q + 2 * e], v[8 * q + 2 * e + 1]);
        const uint32_t at = base + tc_at(c, k + 8 * q);
        st_shared_v4(at, s[0].h, s[1].h, s[2].h, s[3].h);
        st_shared_v4(at + stride, s[0].m, s[1].m, s[2].m, s[3].m);
        st_shared_v4(at + 2 * stride, s[0].l, s[1].l, s[2].l, s[3].l);
    }
}

// u of the CTA's columns into the tiles at x0, m updated.
template <bool V4>
__device__ __forceinline__ void tc_load_as(const MuonArgs &a, const MuonMat &t, uint32_t x0, int64_t c0, int cols) {
    const int64_t o = muon_origin(t, a.r, c0);
    const float *pg = t.g + o;
    float *pm = t.m + o;
    if constexpr (V4) {
        if (!t.tall) {
            // a warp: 4 rows (lane & 3) x 8 groups of 4 columns; four lanes then exchange, so
            // that each has four rows of one column
            constexpr int U = 5;
            const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, groups = (cols + 31) / 32, items = groups * 16;
            for (int b0 = warp; b0 < items; b0 += U * (kMuonThreads / 32)) {
                float4 g[U], m[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int b = b0 + u * (kMuonThreads / 32), kb = b / groups, k = kb * 4 + (lane & 3),
                              c = (b - kb * groups) * 32 + (lane >> 2) * 4;
                    g[u] = m[u] = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (b < items && k < a.r && c < cols) {
                        const uint32_t at = (uint32_t)k * (uint32_t)t.n + (uint32_t)c;
                        g[u] = __ldg(reinterpret_cast<const float4 *>(pg + at));
                        m[u] = *reinterpret_cast<const float4 *>(pm + at);
                    }
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int b = b0 + u * (kMuonThreads / 32), kb = b / groups, k = kb * 4 + (lane & 3),
                              c = (b - kb * groups) * 32 + (lane >> 2) * 4;
                    if (b >= items) break;  // warp-uniform
                    float4 v = m[u];
                    v.x = fmaf(a.mu, v.x, g[u].x); v.y = fmaf(a.mu, v.y, g[u].y);
                    v.z = fmaf(a.mu, v.z, g[u].z); v.w = fmaf(a.mu, v.w, g[u].w);
                    if (k < a.r && c < cols)
                        *reinterpret_cast<float4 *>(pm + (uint32_t)k * (uint32_t)t.n + (uint32_t)c) = v;
                    if (a.nesterov) {
                        v.x = fmaf(a.mu, v.x, g[u].x); v.y = fmaf(a.mu, v.y, g[u].y);
                        v.z = fmaf(a.mu, v.z, g[u].z); v.w = fmaf(a.mu, v.w, g[u].w);
                    }
                    // 4 x 4 transpose among lanes of equal lane / 4: rows k & ~3 .. of column c + (k & 3)
                    const bool odd = lane & 1, high = lane & 2;
                    float s0 = odd ? v.x : v.y, s1 = odd ? v.z : v.w;
                    s0 = __shfl_xor_sync(0xffffffffu, s0, 1);
                    s1 = __shfl_xor_sync(0xffffffffu, s1, 1);
                    if (odd) { v.x = s0; v.z = s1; } else { v.y = s0; v.w = s1; }
                    float s2 = high ? v.x : v.z, s3 = high ? v.y : v.w;
                    s2 = __shfl_xor_sync(0xffffffffu, s2, 2);
                    s3 = __shfl_xor_sync(0xffffffffu, s3, 2);
                    if (high) { v.x = s2; v.y = s3; } else { v.z = s2; v.w = s3; }
                    const int col = c + (k & 3);
                    if (col < cols) tc_put4(x0, kTcSplit, col, k & ~3, v);
                }
            }
            return;
        }
    }
    constexpr int W = V4 ? 4 : 1, U = V4 ? 5 : 6;
    float g[U][W], m[U][W];
    muon_items<64, 64, U, V4>(
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
#pragma unroll
            for (int w = 0; w < W; ++w) m[u][w] = fmaf(a.mu, m[u][w], g[u][w]);
            if constexpr (V4) *reinterpret_cast<float4 *>(pm + at) = make_float4(m[u][0], m[u][1], m[u][2], m[u][3]);
            else pm[at] = m[u][0];
            if (a.nesterov)
#pragma unroll
                for (int w = 0; w < W; ++w) m[u][w] = fmaf(a.mu, m[u][w], g[u][w]);
            const int c = so >> 6, k = so & 63;
            if constexpr (V4) {
                tc_put4(x0, kTcSplit, c, k, make_float4(m[u][0], m[u][1], m[u][2], m[u][3]));
            } else {
                const Split2 s = split2(m[u][0], 0.f);
                const uint32_t to = x0 + tc_at(c, k);
                st_shared_u16(to, s.h);
                st_shared_u16(to + kTcSplit, s.m);
                st_shared_u16(to + 2 * kTcSplit, s.l);
            }
        });
}

__device__ __noinline__ void tc_load(const MuonArgs &a, const MuonMat &t, uint32_t x0, int64_t c0, int cols) {
    // zeros: rows of r .. 64, and columns up to the next multiple of 16
    const int all = (cols + 15) / 16 * 16;
    if (a.r < 64 || all > cols) {
        for (int e = threadIdx.x; e < 3 * all * 8; e += kMuonThreads) {
            const int tile = e / (all * 8), at = e - tile * all * 8;
            if (a.r < 64 || at / 8 >= cols) st_shared_v4(x0 + tile * kTcSplit + at * 16, 0u, 0u, 0u, 0u);
        }
        __syncthreads();
    }
    if (t.vec) tc_load_as<true>(a, t, x0, c0, cols);
    else tc_load_as<false>(a, t, x0, c0, cols);
}

// The six products of two split operands, small ones first: (tile of A, tile of B).
__device__ __forceinline__ int tc_a(int p) { return p == 0 ? 2 : p == 1 ? 0 : p <= 3 ? 1 : 0; }
__device__ __forceinline__ int tc_b(int p) { return p == 0 ? 0 : p == 1 ? 2 : p == 2 ? 1 : p == 3 ? 0 : p == 4 ? 1 : 0; }

// One thread: D[128 x 64] = A B^T over K = 64, both K-major (A's 128 rows at a0, of
// which 64 may be others'; B's 64 rows at b0).
__device__ __forceinline__ void tc_mma_k64(uint32_t d, uint32_t a0, uint32_t a_stride, uint32_t b0, uint32_t b_stride) {
    const uint32_t idesc = idesc_bf16_f32(64, false, false);
#pragma unroll 1
    for (int p = 0; p < 6; ++p) {
        const uint32_t a = a0 + tc_a(p) * a_stride, b = b0 + tc_b(p) * b_stride;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
            umma_bf16(d, smem_desc_sw128(a + kk * 32, 16, 1024), smem_desc_sw128(b + kk * 32, 16, 1024), idesc,
                      p > 0 || kk > 0 ? 1u : 0u);
    }
}

// One thread: D[128 x 192] = [h m]^T [h m l] over `steps` x 16 columns of X, the rank on M
// and N (six products of 64 x 64, of which m l is not used; one MMA reads 10 KB of
// shared memory, which is what it takes, where six of N 64 would read 36).
__device__ __forceinline__ void tc_mma_gram(uint32_t d, uint32_t x0, int steps) {
    const uint32_t idesc = idesc_bf16_f32(192, true, true);
#pragma unroll 4
    for (int s = 0; s < steps; ++s) {
        const uint64_t x = smem_desc_sw128(x0 + s * 2048, kTcSplit, 1024);
        umma_bf16(d, x, x, idesc, s > 0 ? 1u : 0u);
    }
}

// 16 columns of a warp's 32 lanes of TMEM (the lanes of quarter `q`).
__device__ __forceinline__ void tc_read(uint32_t tmem, int q, uint32_t col, float (&v)[16]) {
    tmem_ld_x16(tmem + ((uint32_t)(q * 32) << 16) + col, v);
}

__global__ void __launch_bounds__(kMuonThreads, 1) muon_tc_kernel(const __grid_constant__ MuonArgs a) {
    // 1,024-byte aligned: X's tiles, then (floats) what exchanges need over two r x r matrices' tiles
    float *const f0 = muon_smem(0);
    const uint32_t pad = (1024u - (smem_u32(f0) & 1023u)) & 1023u;
    const uint32_t x0 = smem_u32(f0) + pad, rest = x0 + 3 * kTcSplit, b1 = rest, b2 = rest + 3 * kTcMat;
    float *const R = f0 + (pad + 3 * kTcSplit) / 4;
    float *const part = R + kTcPart, *const recv = R + kTcRecv, *const G = R + kTcG, *const slab = R + kTcSlab;
    const int o_x = (int)(pad / 4);  // the update's fp32 columns, over the tiles
    __shared__ __align__(8) uint64_t s_bars[3];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, q = warp & 3, part4 = warp >> 2;
    const int rank = (int)cluster_ctarank();
    const MuonMat &t = a.mat[blockIdx.x / a.cluster];
    const int64_t c_begin = rank * t.per, c_end = min(t.n, c_begin + t.per);
    const int cols = (int)(c_end > c_begin ? c_end - c_begin : 0), tiles = (cols + 127) / 128, steps = (cols + 15) / 16;
    const MuonLink link{smem_u32(s_bars), a.cluster, rank, &s_abort, a.status};
    const uint32_t mma_bar = smem_u32(s_bars + 2);
    uint32_t n = 0, mmas = 0;  // exchanges, commits so far
    if (threadIdx.x == 0) {
        for (int i = 0; i < 3; ++i) mbar_init(smem_u32(s_bars + i), 1);
        s_abort = 0;
        fence_mbar_init();
    }
    if (warp == 0) {
        tmem_alloc(smem_u32(&s_tmem), kTcTmem);
        tmem_relinquish();
    }
    tc_load(a, t, x0, c_begin, cols);
    fence_proxy_async_smem();
    tc_fence_before();
    cluster_sync();  // X, the barriers of all CTAs, and TMEM
    tc_fence_after();
    const uint32_t tmem = s_tmem;

    // the MMAs that `issue` gives (one thread), then their results (all)
    auto run = [&](auto &&issue) {
        if (warp == 0) {
            if (elect_one()) {
                tc_fence_after();
                issue();
                umma_commit(mma_bar);
            }
            __syncwarp();
        }
    };
    auto await = [&]() {
        if (!mbar_wait(mma_bar, mmas & 1u, &s_abort)) {
            s_abort = 1;
            record_error(a.status, ATTT_ERR_TIMEOUT);
        }
        ++mmas;
        __syncwarp();
        tc_fence_after();
    };
    // results have been read and operands written: the next MMAs may come
    auto settle = [&]() {
        tc_fence_before();
        fence_proxy_async_smem();
        __syncthreads();
    };
    // The same for r x r products, among the warps that have their results: the others wait
    // for the last one's.
    auto settle_few = [&]() {
        tc_fence_before();
        fence_proxy_async_smem();
        named_barrier_sync(1, kMuonThreads / 2);
    };
    // An r x r matrix is in the first two quarters' lanes: row 32 q + lane, columns 16 part4 ..
    const bool mine = q < 2;
    const int row = 32 * q + lane, col = 16 * part4;  // (rows 64 .. 127: the upper lanes)
    // z = x y from the split x at xa and y at ya: form(i, v) turns the thread's value i of x y into
    // that of the matrix that goes to za
    auto product = [&](uint32_t xa, uint32_t ya, uint32_t za, auto &&form) {
        if (!mine) {
            ++mmas;
            return;
        }
        run([&] { tc_mma_k64(tmem + kTcPoly, xa, kTcMat, ya, kTcMat); });
        await();
        float v[16];
        tc_read(tmem, q, kTcPoly + col, v);
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = form(i, v[i]);
        tc_put16(za, kTcMat, row, col, v);
        settle_few();
    };

    const int groups = (a.steps + 1) / 2, single = a.steps % 2 ? groups / 2 : -1;  // pairs, the odd step amidst them
    for (int gi = 0; gi < groups; ++gi) {
        // the cluster's Gram matrix: exchanges over the matrices' tiles, which no CTA reads any more
        run([&] { tc_mma_gram(tmem + kTcGram, x0, steps); });
        await();
        {   // h h + h m + h l (lower lanes) + m h + m m (upper lanes) + (h l)^T
            float v[16], w[16], hl[16];
            tc_read(tmem, q, kTcGram + col, v);
            tc_read(tmem, q, kTcGram + 64 + col, w);
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = steps > 0 ? v[i] + w[i] : 0.f;  // no columns: no MMAs
            const int i0 = row & 63;
            if (mine) {
                tc_read(tmem, q, kTcGram + 128 + col, hl);
#pragma unroll
                for (int i = 0; i < 16; ++i) G[i0 * 65 + col + i] = steps > 0 ? hl[i] : 0.f;
            } else {
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    *reinterpret_cast<float4 *>(part + i0 * kTcLD + col + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
            }
            __syncthreads();
            if (mine) {
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    float4 *to = reinterpret_cast<float4 *>(part + i0 * kTcLD + col + i);
                    const float4 u = *to;
                    const float o[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        v[i + e] += o[e] + (G[i0 * 65 + col + i + e] + G[(col + i + e) * 65 + i0]);
                    *to = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                }
            }
        }
        tc_fence_before();
        if (gi > 0) cluster_sync();  // every CTA has done with the matrices' tiles that exchanges come over
        const int r0 = muon_row(64, rank, a.cluster), r1 = muon_row(64, rank + 1, a.cluster);
        link.gather<64, kTcLD>(n, part, recv, r0, r1, [&](int at, float4 v) {
            *reinterpret_cast<float4 *>(G + r0 * kTcLD + at) = v;
            *reinterpret_cast<float4 *>(slab + at) = v;
        });
        link.share<kTcLD>(n + 1, slab, G, r0, r1, 64);
        n += 2;
        // every warp for itself: |X|_F^2, the scale of the first one, and the mean d of G's diagonal
        float trace = G[lane * (kTcLD + 1)] + G[(lane + 32) * (kTcLD + 1)];
        for (int o = 16; o > 0; o >>= 1) trace += __shfl_xor_sync(0xffffffffu, trace, o);
        const float scale = gi == 0 ? muon_scale(trace, a.eps) : 1.f;
        const float d = trace * scale * scale / (float)a.r;
        // M = m I + M' for each matrix: e, eb and f are this thread's elements of some of the M'
        float e[16], eb[16], f[16];
        if (mine) {
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const float4 v = *reinterpret_cast<const float4 *>(G + row * kTcLD + col + i);
                e[i] = v.x * scale * scale; e[i + 1] = v.y * scale * scale;
                e[i + 2] = v.z * scale * scale; e[i + 3] = v.w * scale * scale;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (col + i == row) e[i] -= d;
        }
        __syncthreads();  // G has been read: the tiles may be written over it
        if (mine) tc_put16(b1, kTcMat, row, col, e);
        settle();
        // B = a I + b G + c G^2, and for a pair of steps G <- B G B, P = (a I + b G + c G^2) B
        const float db = fmaf(d, fmaf(kNsC, d, kNsB), kNsA), lin = fmaf(2.f * kNsC, d, kNsB);
        uint32_t P;
        if (gi != single) {
            const float dt = db * d, d2 = dt * db, db2 = fmaf(d2, fmaf(kNsC, d2, kNsB), kNsA),
                        lin2 = fmaf(2.f * kNsC, d2, kNsB), dp = scale * (db2 * db);
            product(b1, b1, b2, [&](int i, float v) { return eb[i] = fmaf(kNsC, v, lin * e[i]); });           // B
            product(b2, b1, b1, [&](int i, float v) { return f[i] = fmaf(db, e[i], fmaf(d, eb[i], v)); });    // B G
            product(b1, b2, b1, [&](int i, float v) { return e[i] = fmaf(dt, eb[i], fmaf(db, f[i], v)); });   // second G
            product(b1, b1, b1, [&](int i, float v) { return f[i] = fmaf(kNsC, v, lin2 * e[i]); });           // its B
            product(b1, b2, b1, [&](int i, float v) {
                const float p = scale * fmaf(db2, eb[i], fmaf(db, f[i], v));
                return col + i == row ? p + dp : p;
            });
            P = b1;
        } else {
            product(b1, b1, b2, [&](int i, float v) {
                const float p = scale * fmaf(kNsC, v, lin * e[i]);
                return col + i == row ? fmaf(scale, db, p) : p;
            });
            P = b2;
        }
        __syncthreads();
        // X <- P X: warp (q, part4) has columns 128 part4 + 32 q + lane
        const bool last = gi + 1 == groups;
        run([&] {
            for (int j = 0; j < tiles; ++j) tc_mma_k64(tmem + 64u * j, x0 + j * 16384u, kTcSplit, P, kTcMat);
        });
        await();
        const int c = 128 * part4 + 32 * q + lane;
        if (part4 < tiles) {  // warp-uniform
#pragma unroll 1
            for (int k = 0; k < 64; k += 16) {
                float v[16];
                tc_read(tmem, q, 64u * part4 + k, v);
                if (c < cols) {
                    if (last) {
                        float *to = muon_smem(o_x) + c * 68 + k;
#pragma unroll
                        for (int i = 0; i < 16; i += 4)
                            *reinterpret_cast<float4 *>(to + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                    } else {
                        tc_put16(x0, kTcSplit, c, k, v);
                    }
                }
            }
        }
        settle();
        if (last) muon_update<64>(a, t, o_x, c_begin, cols, link);
    }
    tc_fence_before();
    cluster_sync();  // no CTA leaves while it is sent to
    tc_fence_after();
    if (warp == 0) tmem_dealloc(tmem, kTcTmem);
}

attt_status muon_tc_run(const MuonArgs &args, int nmat, int dev, cudaStream_t stream, bool *done) {
    const void *kern = reinterpret_cast<const void *>(muon_tc_kernel);
    int most[kMuonMaxCluster + 1];
    if (!set_smem_limit(kern, kTcSmem, dev) || !muon_clusters(kern, kTcSmem, dev, most)) return ATTT_ERR_CUDA;
    MuonArgs a = args;
    int64_t n = 0, cost = 0;
    for (int i = 0; i < nmat; ++i) n = std::max(n, a.mat[i].n);
    a.cluster = muon_cluster(most, nmat, n, kTcCols, &cost);
    *done = a.cluster > 0;
    if (!*done) return ATTT_OK;
    return muon_launch(kern, a, nmat, kTcSmem, stream);
}

}  // namespace attt

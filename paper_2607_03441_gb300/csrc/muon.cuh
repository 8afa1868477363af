// muon.cuh -- what the two forms of the Muon step (muon.cu, muon_tc.cu) share: the
// arguments, the exchanges between the CTAs of a cluster, and the passes over a
// matrix's elements in global memory.
#pragma once

#include <cfloat>

#include "attt_common.cuh"
#include "attt_host.h"

namespace attt {

constexpr int kMuonMats = 16;  // two per projection
constexpr int kMuonThreads = 512;
constexpr int kMuonStage = 128;  // columns of a tile that does not stay
constexpr int kMuonMinCluster = 4, kMuonMaxCluster = 16;
constexpr double kNsA64 = 3.4445, kNsB64 = -4.7750, kNsC64 = 2.0315;
// The least eps: |u|_F^2 near its square is a normal fp32 number, and so are the squares of
// u's elements where they count beside eps.
constexpr float kMuonMinEps = 1e-12f;
constexpr float kNsA = (float)kNsA64, kNsB = (float)kNsB64, kNsC = (float)kNsC64;

struct MuonMat {
    float *p, *m;
    const float *g;
    __nv_bfloat16 *p16;
    float *x;    // [n][RP], columns that do not stay in shared memory
    int64_t n;   // width beside r
    int64_t per; // columns of a CTA, a multiple of 8
    int tall;    // [n, r] (A), else [r, n] (B)
    int vec;     // whether four neighbours in memory may move at once
    float step;  // lr rms sqrt(max(rows, columns))
};

struct MuonArgs {
    MuonMat mat[kMuonMats];
    int r, nesterov, steps, cluster;
    int room;        // columns that fit in shared memory
    uint32_t inv_r;  // ceil(2^32 / r), r > 1: e / r is the high half of e inv_r for e < 2^26
    float mu, keep, eps;  // keep = 1 - lr wd
    int *status;
};

// 1 / (|u|_F + eps) from |u|_F^2, the Gram matrix's trace.  Beyond fp32 NaN, and with it the whole
// matrix: the diagonal's elements may all be finite where their sum is not, and 1 / inf
// would make an update of 0.
__device__ __forceinline__ float muon_scale(float trace, float eps) {
    return trace <= FLT_MAX ? 1.f / (sqrtf(trace) + eps) : __int_as_float(0x7fc00000);
}

// Rows [first, second) of an r x r matrix that CTA `rank` of `cluster` forms.
__device__ __forceinline__ int muon_row(int RP, int rank, int cluster) { return rank * RP / cluster; }

// Exchanges of the cluster: number `n` (0, 1, ..) is counted on barrier n & 1.  A CTA
// sends for exchange n + 1 when it has all of exchange n, and so has nothing more to
// read of what exchange n came from; what CTAs send for exchange n + 2 follows this
// CTA's own data of n + 1.
struct MuonLink {
    uint32_t bar0;
    int cluster, rank;
    volatile int *abort_flag;
    int *status;

    // One thread: `bytes` will come in exchange n.
    __device__ __forceinline__ void expect(uint32_t n, uint32_t bytes) const {
        mbar_arrive_expect_tx(bar0 + 8u * (n & 1u), bytes);
    }
    // One thread per receiver: copies `bytes` of this CTA's shared memory to `dst` (an
    // address of this CTA's own) in CTA `to`.
    __device__ __forceinline__ void send(uint32_t n, uint32_t dst, uint32_t src, uint32_t bytes, int to) const {
        asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                         mapa_shared(dst, to)),
                     "r"(src), "r"(bytes), "r"(mapa_shared(bar0 + 8u * (n & 1u), to))
                     : "memory");
    }
    // Whether a wait of this CTA has run out.
    __device__ __forceinline__ bool lost() const { return *abort_flag != 0; }
    // All threads: exchange n has arrived.  If it does not within the limit, the status word
    // says so and the CTA goes on to its end on garbage, waiting for nothing, sending nothing
    // (so that the others' waits run out too) and leaving p as it is.
    __device__ __forceinline__ void receive(uint32_t n) const {
        if (!mbar_wait(bar0 + 8u * (n & 1u), (n >> 1) & 1u, abort_flag)) {
            *abort_flag = 1;
            record_error(status, ATTT_ERR_TIMEOUT);
        }
    }
    // Every CTA's rows of this one's RP x RP matrix `part` (rows of LD floats) to it, place
    // `rank` of its recv; then rows [r0, r1) of the sum over the CTAs, in their order:
    // add(at, v) for 4 of them at `at` from the first row.  Exchange n.
    template <int RP, int LD, class Add>
    __device__ __forceinline__ void gather(uint32_t n, const float *part, const float *recv, int r0, int r1,
                                           Add &&add) const {
        const int rows = r1 - r0;
        fence_proxy_async_smem();
        __syncthreads();
        if (threadIdx.x == 0) expect(n, (uint32_t)((cluster - 1) * rows * LD * 4));
        if (threadIdx.x < (unsigned)cluster && (int)threadIdx.x != rank && !lost()) {
            const int o0 = muon_row(RP, threadIdx.x, cluster), o = muon_row(RP, threadIdx.x + 1, cluster) - o0;
            if (o > 0)
                send(n, smem_u32(recv + rank * o * LD), smem_u32(part + o0 * LD), (uint32_t)(o * LD * 4), threadIdx.x);
        }
        receive(n);
        for (int e = threadIdx.x; e < rows * RP / 4; e += kMuonThreads) {
            const int at = e / (RP / 4) * LD + e % (RP / 4) * 4;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
            for (int c = 0; c < cluster; ++c) {
                const float4 q =
                    *reinterpret_cast<const float4 *>(c == rank ? part + r0 * LD + at : recv + c * rows * LD + at);
                v.x += q.x; v.y += q.y; v.z += q.z; v.w += q.w;
            }
            add(at, v);
        }
    }
    // All threads: rows [r0, r1) of z (LD floats each) to all CTAs from `src`, and theirs of
    // `total` from them.  Nothing says when `src` has been read: it stays as it is until
    // a later exchange, for which every CTA has to have these rows.
    template <int LD>
    __device__ __forceinline__ void share(uint32_t n, const float *src, const float *z, int r0, int r1,
                                          int total) const {
        fence_proxy_async_smem();
        __syncthreads();
        if (threadIdx.x == 0) expect(n, (uint32_t)((total - (r1 - r0)) * LD * 4));
        if (threadIdx.x < (unsigned)cluster && (int)threadIdx.x != rank && r1 > r0 && !lost())
            send(n, smem_u32(z + r0 * LD), smem_u32(src), (uint32_t)((r1 - r0) * LD * 4), threadIdx.x);
        receive(n);
    }
};

// Shared memory is named by its place in s_muon: functions of their own know no other
// way that an address is not global.
extern __shared__ float4 s_muon[];
__device__ __forceinline__ float *muon_smem(int at) { return reinterpret_cast<float *>(s_muon) + at; }

// The elements of columns [0, cols) from column c0 on, U items of 1 (or, V4, 4
// neighbours in memory) per thread at a time: first(u, at) for each of them, then
// second(u, at, so), so that U loads are on their way together.  `at`: index from the
// first column's first element in global memory; so: place in shared memory.
// Neighbours are the rows k .. k + 3 of a column (tall), or the columns c .. c + 3.
template <int RP, int LD, int U, bool V4, class F, class S>
__device__ __forceinline__ void muon_items(const MuonMat &t, int r, uint32_t inv_r, int cols, F &&first, S &&second) {
    constexpr int W = V4 ? 4 : 1;
    // a warp of a wide matrix's items: 8 columns x 4 rows, or 4 x 4 columns x 8 rows
    constexpr int KR = V4 ? 8 : 4, CW = V4 ? 16 : 8;
    const int groups = (cols + CW - 1) / CW, width = (int)t.n;
    const int items = t.tall ? cols * r / W : groups * (RP / KR) * 32;
    for (int e0 = threadIdx.x; e0 < items; e0 += U * kMuonThreads) {
        uint32_t at[U];
        int so[U];
        bool in[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int e = e0 + u * kMuonThreads;
            if (t.tall) {
                const int c = r == 1 ? e : (int)__umulhi((uint32_t)(W * e), inv_r);
                at[u] = (uint32_t)(W * e);
                so[u] = c * LD + W * e - c * r;
                in[u] = e < items;
            } else {
                const int b = e >> 5, lane = e & 31, kb = b / groups;
                const int k = kb * KR + (V4 ? lane >> 2 : lane >> 3);
                const int c = (b - kb * groups) * CW + (V4 ? (lane & 3) * 4 : lane & 7);
                at[u] = (uint32_t)k * (uint32_t)width + (uint32_t)c;
                so[u] = c * LD + k;
                in[u] = e < items && k < r && c < cols;
            }
            if (in[u]) first(u, at[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (in[u]) second(u, at[u], so[u]);
    }
}

// The first column's first element.
__device__ __forceinline__ int64_t muon_origin(const MuonMat &t, int r, int64_t c0) { return t.tall ? c0 * r : c0; }

// p <- keep p - step X for the columns, and the bf16 copy (muon_update: unless X is garbage).
template <int RP, bool V4>
__device__ __forceinline__ void muon_update_as(const MuonArgs &a, const MuonMat &t, const float *s, int64_t c0,
                                               int cols) {
    constexpr int LD = RP + 4, W = V4 ? 4 : 1, U = V4 ? 7 : 8;
    const int64_t o = muon_origin(t, a.r, c0);
    float *pp = t.p + o;
    __nv_bfloat16 *ph = t.p16 ? t.p16 + o : nullptr;
    float p[U][W];
    muon_items<RP, LD, U, V4>(
        t, a.r, a.inv_r, cols,
        [&](int u, uint32_t at) {
            if constexpr (V4) {
                const float4 x = *reinterpret_cast<const float4 *>(pp + at);
                p[u][0] = x.x; p[u][1] = x.y; p[u][2] = x.z; p[u][3] = x.w;
            } else {
                p[u][0] = pp[at];
            }
        },
        [&](int u, uint32_t at, int so) {
            float x[W];
            if (V4 && t.tall) {
                const float4 q = *reinterpret_cast<const float4 *>(s + so);
                x[0] = q.x; x[W / 4] = q.y; x[W / 2] = q.z; x[W - 1] = q.w;
            } else {
#pragma unroll
                for (int w = 0; w < W; ++w) x[w] = s[so + w * LD];
            }
#pragma unroll
            for (int w = 0; w < W; ++w) p[u][w] = fmaf(-t.step, x[w], p[u][w] * a.keep);
            if constexpr (V4) {
                *reinterpret_cast<float4 *>(pp + at) = make_float4(p[u][0], p[u][1], p[u][2], p[u][3]);
                if (ph) {
                    __nv_bfloat162 h[2] = {__floats2bfloat162_rn(p[u][0], p[u][1]),
                                           __floats2bfloat162_rn(p[u][2], p[u][3])};
                    *reinterpret_cast<uint2 *>(ph + at) = *reinterpret_cast<uint2 *>(h);
                }
            } else {
                pp[at] = p[u][0];
                if (ph) ph[at] = __float2bfloat16_rn(p[u][0]);
            }
        });
}

template <int RP>
__device__ __noinline__ void muon_update(const MuonArgs &a, const MuonMat &t, int s_at, int64_t c0, int cols,
                                         const MuonLink &link) {
    if (link.lost()) return;
    if (t.vec) muon_update_as<RP, true>(a, t, muon_smem(s_at), c0, cols);
    else muon_update_as<RP, false>(a, t, muon_smem(s_at), c0, cols);
}

// Clusters of each size that the device runs at once (0: none), for one kernel with one
// amount of shared memory (muon.cu).
bool muon_clusters(const void *kern, size_t smem, int dev, int (&most)[kMuonMaxCluster + 1]);

// The CTAs of a cluster for nmat matrices of at most n columns: as many as leave the
// fewest columns for a CTA in all the rounds that the clusters take (a part with 15
// clusters of 8, 8 of 12 and 7 of 16 takes 12 for 8 matrices), at most `room` columns if
// it is > 0; *cost: those columns.  0: no size does.
int muon_cluster(const int (&most)[kMuonMaxCluster + 1], int nmat, int64_t n, int64_t room, int64_t *cost);

// muon_kernel's launch for `cluster` CTAs per matrix.
attt_status muon_launch(const void *kern, MuonArgs &a, int nmat, size_t smem, cudaStream_t stream);

// The step on the tensor cores, for ranks of 33 to 64 whose columns all fit in shared
// memory (muon_tc.cu); *done: whether it was.
attt_status muon_tc_run(const MuonArgs &a, int nmat, int dev, cudaStream_t stream, bool *done);

}  // namespace attt

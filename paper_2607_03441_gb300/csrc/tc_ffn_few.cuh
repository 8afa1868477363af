// tc_ffn_few.cuh -- the gated feed-forward block's contractions for at most 96 rows,
// where the weights' bytes and the chain of launches are what they cost.
//
// A tile of columns belongs to a cluster of C CTAs (1 to 8) that share its K blocks; each
// accumulates in TMEM, copies its sums to shared memory, and after a cluster barrier sums
// a share of the columns over the CTAs in their order and finishes them: the result
// does not depend on timing, and no second kernel sums pieces.
// The adapters need no launch of their own either: beside the weights' columns a CTA
// accumulates the rank-r product of the same activations (x A: N = r more columns of
// the MMA, the adapter's matrix read from L2 by every cluster), and the sum's second
// product, (s x A) B for the tile's columns, is r more multiplications per value when the
// columns are finished (mma.sync on fragments: it is a thousandth of the tile's work and
// its operands and results are where warps have them).
// Warps 0 and 7 load weights, which are the caller's inputs, without waiting for the previous
// grid; warp 6 loads activations once that grid has ended: the second of a call's two
// launches streams weights while the first one ends.  Warps 2 to 5 bring the second matrices'
// share of the tile into shared memory meanwhile.
// Bound: HBM bytes.  1 row at 3,584 x 18,944: FEW_GLU 46.6 us (271.7 MB: 5.8 TB/s), FEW_DOWN 27.9 (135.9 MB: 4.9; the
// two overlap, 69 together); 93 rows with r = 16: FEW_GRAD 38.7, FEW_DX 60.6.  What is left is each
// launch's begin and end, some 5 us, and the sums' way through distributed shared memory.
#pragma once

#include "tc_ffn.cuh"

namespace attt {

enum FewMode : int {
    FEW_GLU = 0,   // h = act(g) u [, g, u]: gate and up columns side by side, weights MN-major
    FEW_DOWN = 1,  // y: weights MN-major
    FEW_GRAD = 2,  // dg, du from dh: weights K-major
    FEW_DX = 3,    // dx: two K ranges, weights K-major
};

constexpr int kFewThreads = 256, kFewMaxStages = 8, kFewMaxCluster = 8;
constexpr int kFewRows = 96;  // at most (ffn.cu: which calls)
constexpr int kFewStep = 4;  // fragments of a warp at a time

// A rank-r product: of the activations of segment `seg`, with matrix map r[i], into accumulator
// columns from `col`; its second matrix as [k, n] (FEW_GLU, FEW_DOWN: rows of N) or [n, k] (rows of r8).
struct FewRank {
    int seg, col, half;  // half: FEW_GLU: 0 the gate's columns, 1 the up's
    const __nv_bfloat16 *second;
    int64_t ld;
};

// Weights MN-major: columns of the box that holds a product's matrix, and with it its swizzle, twice that
// many bytes.  A box 64 wide whatever r is takes as much of a stage as 64 columns of weights, and the SM
// fills its zeros at the same rate: forward, 1 row at 3,584 x 18,944 with r = 16, 82.3 us (79.4 so).
constexpr int few_rank_cols(int rpad) { return rpad <= 16 ? 16 : rpad <= 32 ? 32 : 64; }

// A descriptor's bits 61 to 63 for an MN-major matrix in such a box (64, 32 or 128 bytes of swizzle).
__device__ __forceinline__ uint64_t few_rank_desc(uint32_t addr, int r_cols) {
    const uint64_t mode = r_cols == 64 ? 2u : r_cols == 32 ? 4u : 6u;
    return (smem_desc_sw128(addr, 8192u, (uint32_t)r_cols * 16u) & ~(uint64_t(7) << 61)) | mode << 61;
}

struct FewMaps {
    CUtensorMap a[2], b[2], r[2];
};

struct FewArgs {
    int M, N, n_tile, BN;  // columns of the result, of a tile, of its accumulator
    int nseg, kb[2], kb_total;
    int nrank, r, rpad;
    FewRank rank[2];
    float scale;
    int cluster, stages;
    uint32_t a_alloc, a_bytes, b_bytes, r_bytes;  // per stage; r_bytes: of one product
    int r_cols;            // weights MN-major: columns of a product's box (few_rank_cols)
    uint32_t ring_bytes, tmem_cols;
    int pitch, vpitch;     // of the sums (fp32) and of the rank-r products (bf16) in shared memory
    uint32_t second_at;    // behind the ring: the second matrices, [rank][column of the tile][rpad + 8]
    uint32_t bars_at;
    int weights_wait;      // the previous grid prepares an adapter's matrix
    int act, keep;
    const __nv_bfloat16 *gate, *up;
    __nv_bfloat16 *out[3];
    int *status;
};

__device__ __forceinline__ float2 ld_cluster_f2(uint32_t addr) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
    return v;
}

__device__ __forceinline__ float4 ld_cluster_f4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}

// d += a b for a 16 x 16 block of a (rows) and 16 x 8 of b.
__device__ __forceinline__ void few_mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void few_put2(__nv_bfloat16 *p, float a, float b) {
    *reinterpret_cast<__nv_bfloat162 *>(p) = __floats2bfloat162_rn(a, b);
}

template <int MODE>
__global__ void __launch_bounds__(kFewThreads, 2)
    ffn_few_kernel(const __grid_constant__ FewMaps maps, const __grid_constant__ FewArgs p) {
    constexpr bool B_MN = MODE == FEW_GLU || MODE == FEW_DOWN;
    constexpr int kHalves = MODE == FEW_GLU ? 2 : 1;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    // the ring: all A stages (an MMA reads 128 rows from a stage's begin, those past M whatever they are),
    // then weights and adapters per stage; later the sums
    const uint32_t ring = smem_u32(smem);
    const int S = p.stages;
    const uint32_t w_bytes = p.b_bytes + (uint32_t)p.nrank * p.r_bytes, ring_b = ring + (uint32_t)S * p.a_alloc;
    __nv_bfloat16 *const sv = reinterpret_cast<__nv_bfloat16 *>(smem + p.ring_bytes);
    __nv_bfloat16 *const s2 = reinterpret_cast<__nv_bfloat16 *>(smem + p.second_at);
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + p.bars_at);
    const uint32_t full0 = smem_u32(bars), empty0 = smem_u32(bars + kFewMaxStages), done = smem_u32(bars + 2 * kFewMaxStages);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + 2 * kFewMaxStages + 1);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int C = p.cluster, rank = C > 1 ? (int)cluster_ctarank() : 0;
    const int n0 = ((int)blockIdx.x / C) * p.n_tile;
    const int k0 = (int)((int64_t)p.kb_total * rank / C), k1 = (int)((int64_t)p.kb_total * (rank + 1) / C);

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(full0 + 8 * s, 2);
            mbar_init(empty0 + 8 * s, 1);
        }
        mbar_init(done, 1);
        *abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(tmem_slot), p.tmem_cols);
        tmem_relinquish();
    }
    if (warp == 2 && lane < 2) {
        tma_prefetch_desc(&maps.a[lane]);
        tma_prefetch_desc(&maps.b[lane]);
        tma_prefetch_desc(&maps.r[lane]);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    if (threadIdx.x == 0) griddep_launch_dependents();  // not before TMEM is allocated (tc_ffn.cuh)

    if (warp == 0 || warp >= 6) {
        if (elect_one()) {
            // -------- TMA producers: weights (warp 0 even blocks, warp 7 odd ones), activations (warp 6) --------
            if (warp == 6 || p.weights_wait) griddep_wait();
            int slot = 0, pos = 0;
            uint32_t phase = 1;
            bool ok = true;
            for (int kb = k0; kb < k1; ++kb, ++pos) {
                if (warp != 6 && ((pos & 1) != 0) != (warp == 7)) {
                    if (++slot == S) {
                        slot = 0;
                        phase ^= 1u;
                    }
                    continue;
                }
                if (pos >= S && !mbar_wait(empty0 + 8 * slot, phase, abort_flag)) { ok = false; break; }
                const uint32_t fb = full0 + 8 * slot;
                const int seg = p.nseg > 1 && kb >= p.kb[0] ? 1 : 0, j = 64 * (kb - (seg ? p.kb[0] : 0));
                if (warp == 6) {
                    mbar_arrive_expect_tx(fb, p.a_bytes);
                    tma_load_2d(ring + (uint32_t)slot * p.a_alloc, &maps.a[seg], fb, j, 0);
                } else {
                    uint32_t dst = ring_b + (uint32_t)slot * w_bytes;
                    uint32_t bytes = p.b_bytes;
                    for (int i = 0; i < p.nrank; ++i)
                        if (p.rank[i].seg == seg) bytes += p.r_bytes;
                    mbar_arrive_expect_tx(fb, bytes);
                    if constexpr (B_MN) {
                        for (int h = 0; h < kHalves; ++h)
                            for (int b = 0; b < p.n_tile / 64; ++b, dst += 8192u)
                                tma_load_2d(dst, &maps.b[h], fb, n0 + 64 * b, j);
                    } else {
                        tma_load_2d(dst, &maps.b[seg], fb, j, n0);
                        dst += p.b_bytes;
                    }
                    for (int i = 0; i < p.nrank; ++i, dst += p.r_bytes)
                        if (p.rank[i].seg == seg) tma_load_2d(dst, &maps.r[i], fb, B_MN ? 0 : j, B_MN ? j : 0);
                }
                if (++slot == S) {
                    slot = 0;
                    phase ^= 1u;
                }
            }
            if (!ok) {
                *abort_flag = 1;
                record_error(p.status, ATTT_ERR_TIMEOUT);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (elect_one()) {
            // ---------------- MMA issuer ----------------
            const uint32_t idesc = idesc_bf16_f32((uint32_t)p.BN, false, B_MN);
            const uint32_t idesc_r = idesc_bf16_f32((uint32_t)(p.nrank > 0 ? p.rpad : 16), false, B_MN);
            constexpr uint32_t step = (B_MN ? 2048u : 32u) >> 4, lbo = B_MN ? 8192u : 16u;  // 16 along K, in descriptor units
            const int kb0 = p.nseg > 1 ? p.kb[0] : p.kb_total;  // blocks of the first segment
            // the segment whose blocks a product takes, and its first block here; none: past the end
            const int rs0 = p.nrank > 0 ? p.rank[0].seg : 2, rs1 = p.nrank > 1 ? p.rank[1].seg : 2;
            const uint32_t rstep = B_MN ? (uint32_t)p.r_cols * 2u : step;
            const uint32_t col0 = tmem_base + (uint32_t)p.BN, col1 = col0 + (uint32_t)p.rpad;
            int slot = 0;
            uint32_t phase = 0;
            bool ok = true, ready = false;
            for (int kb = k0; kb < k1; ++kb) {
                if (!ready && !mbar_wait(full0 + 8 * slot, phase, abort_flag)) { ok = false; break; }
                tc_fence_after();
                // the next slot's barrier is read while this slot's MMAs issue
                const int next = slot + 1 == S ? 0 : slot + 1;
                const uint32_t next_phase = next == 0 ? phase ^ 1u : phase;
                ready = mbar_test_wait(full0 + 8 * next, next_phase);
                const int seg = kb >= kb0 ? 1 : 0;
                const uint32_t first = kb == k0 || kb == kb0 ? 0u : 1u;  // 0: the segment's first block here
                const uint32_t a_addr = ring + (uint32_t)slot * p.a_alloc, b_addr = ring_b + (uint32_t)slot * w_bytes;
                const uint64_t ad = smem_desc_sw128(a_addr, 16, 1024), bd = smem_desc_sw128(b_addr, lbo, 1024);
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)
                    umma_bf16(tmem_base, ad + kk * 2u, bd + kk * step, idesc, (kb > k0 || kk > 0) ? 1u : 0u);
                if (rs0 == seg) {
                    const uint32_t at = b_addr + p.b_bytes;
                    const uint64_t rd = B_MN ? few_rank_desc(at, p.r_cols) : smem_desc_sw128(at, lbo, 1024);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)
                        umma_bf16(col0, ad + kk * 2u, rd + kk * rstep, idesc_r, kk > 0 ? 1u : first);
                }
                if (rs1 == seg) {
                    const uint32_t at = b_addr + p.b_bytes + p.r_bytes;
                    const uint64_t rd = B_MN ? few_rank_desc(at, p.r_cols) : smem_desc_sw128(at, lbo, 1024);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)
                        umma_bf16(col1, ad + kk * 2u, rd + kk * rstep, idesc_r, kk > 0 ? 1u : first);
                }
                umma_commit(empty0 + 8 * slot);
                slot = next;
                phase = next_phase;
            }
            if (!ok) {
                *abort_flag = 1;
                record_error(p.status, ATTT_ERR_TIMEOUT);
                // loads already issued land before the ring is used for the sums, as far as bounded
                // waits of this thread's own can see to it
                volatile int no_abort = 0;
                for (int i = 0; i < S && mbar_wait(full0 + 8 * slot, phase, &no_abort); ++i)
                    if (++slot == S) {
                        slot = 0;
                        phase ^= 1u;
                    }
            }
            umma_commit(done);
        }
        __syncwarp();
    } else {
        // the second matrices' share of the tile, zeros past r and past the result's columns: runs of eight
        // values, four of them under way per thread (one by one, 32 to 128 trips to L2 in a row
        // were longer than the main loop of a small block)
        const int pitch = p.rpad + 8, runs = B_MN ? p.n_tile / 8 : p.rpad / 8, lines = B_MN ? p.rpad : p.n_tile;
        const int each = runs * lines, total = p.nrank * each;
        const bool whole = B_MN || p.r % 8 == 0;  // runs of a line lie on 16 bytes
        for (int j0 = threadIdx.x - 64; j0 < total; j0 += 4 * 128) {
            uint4 q[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int j = j0 + 128 * u, i = j / each, e = j - i * each, line = e / runs, x = 8 * (e - line * runs);
                q[u] = make_uint4(0, 0, 0, 0);
                if (j >= total) continue;
                const FewRank &rk = p.rank[i];
                if (B_MN ? line >= p.r || n0 + x >= p.N : n0 + line >= p.N || x >= p.r) continue;
                const __nv_bfloat16 *s = rk.second + (B_MN ? (int64_t)line * rk.ld + n0 + x : (int64_t)(n0 + line) * rk.ld + x);
                if (whole) {
                    q[u] = __ldg(reinterpret_cast<const uint4 *>(s));
                } else {
                    uint32_t w[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint16_t *h = reinterpret_cast<const uint16_t *>(s) + 2 * k;
                        w[k] = (x + 2 * k < p.r ? (uint32_t)__ldg(h) : 0u) | (x + 2 * k + 1 < p.r ? (uint32_t)__ldg(h + 1) << 16 : 0u);
                    }
                    q[u] = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int j = j0 + 128 * u, i = j / each, e = j - i * each, line = e / runs, x = 8 * (e - line * runs);
                if (j >= total) continue;
                __nv_bfloat16 *to = s2 + (int64_t)i * p.n_tile * pitch;
                if constexpr (B_MN) {
                    const __nv_bfloat16 *v = reinterpret_cast<const __nv_bfloat16 *>(&q[u]);
#pragma unroll
                    for (int k = 0; k < 8; ++k) to[(x + k) * pitch + line] = v[k];
                } else {
                    *reinterpret_cast<uint4 *>(to + line * pitch + x) = q[u];
                }
            }
        }
    }

    // every MMA has completed (bounded wait), and with them every load of the ring
    {
        volatile int no_abort = 0;
        int ok = 1;
        if (lane == 0) ok = mbar_wait(done, 0u, &no_abort) ? 1 : 0;
        ok = __shfl_sync(0xffffffffu, ok, 0);
        if (!ok && lane == 0) record_error(p.status, ATTT_ERR_TIMEOUT);
        if (ok) (void)mbar_try_wait(done, 0u);
        tc_fence_after();
    }
    __syncthreads();  // (a producer that gave up has stopped before the ring is written)
    const int cols = p.BN + p.nrank * p.rpad;
    {   // a warp's 32 rows (those of its number modulo 4), every other run of 16 columns
        const int q = warp & 3, row = q * 32 + lane;
        const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16);
        if (q * 32 < p.M)
            for (int c = 16 * (warp >> 2); c < cols; c += 32) {
                float v[16];
                tmem_ld_x16(taddr + (uint32_t)c, v);
                // a product whose K blocks are all another CTA's has no sums here
                bool empty = false;
                for (int i = 0; i < p.nrank; ++i)
                    if (c >= p.rank[i].col && c < p.rank[i].col + p.rpad && p.nseg > 1)
                        empty = p.rank[i].seg == 0 ? k0 >= p.kb[0] : k1 <= p.kb[0];
                if (row < p.M)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        st_shared_f4(ring + (uint32_t)(row * p.pitch + c + 4 * j) * 4u,
                                     empty ? make_float4(0.f, 0.f, 0.f, 0.f)
                                           : make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]));
            }
        tc_fence_before();
    }
    if (C > 1) cluster_sync();  // every CTA's sums are in its shared memory
    else __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem_base, p.tmem_cols);
    }
    uint32_t base[kFewMaxCluster];
#pragma unroll
    for (int j = 0; j < kFewMaxCluster; ++j) base[j] = mapa_shared(ring, (uint32_t)(j < C ? j : 0));
    auto sum2 = [&](int row, int col) {  // columns col and col + 1 of a row, over the CTAs in their order
        float2 s = make_float2(0.f, 0.f);
        if (C == 1) return *reinterpret_cast<const float2 *>(smem + (size_t)(row * p.pitch + col) * 4u);
#pragma unroll
        for (int j = 0; j < kFewMaxCluster; ++j)
            if (j < C) {
                const float2 v = ld_cluster_f2(base[j] + (uint32_t)(row * p.pitch + col) * 4u);
                s.x += v.x;
                s.y += v.y;
            }
        return s;
    };
    griddep_wait();  // what is read and overwritten from here on may be the previous grid's
    if (p.nrank > 0) {
        const int vc = p.nrank * p.rpad / 4;  // four columns at a time: with two, 1 to 4 us more of a call
        for (int i = threadIdx.x; i < p.M * vc; i += kFewThreads) {
            const int row = i / vc, c = 4 * (i - row * vc);
            const uint32_t at = (uint32_t)(row * p.pitch + p.BN + c) * 4u;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (C == 1) {
                v = *reinterpret_cast<const float4 *>(smem + at);
            } else {
#pragma unroll
                for (int j = 0; j < kFewMaxCluster; ++j)
                    if (j < C) {
                        const float4 w = ld_cluster_f4(base[j] + at);
                        v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
                    }
            }
            few_put2(sv + row * p.vpitch + c, p.scale * v.x, p.scale * v.y);
            few_put2(sv + row * p.vpitch + c + 2, p.scale * v.z, p.scale * v.w);
        }
        __syncthreads();
    }
    // fragments of 16 rows x 8 columns, this CTA's share of the tile's columns, four to a warp at a time
    const int g = lane >> 2, t = lane & 3, col = 2 * t;
    const int f0 = (p.n_tile / 8) * rank / C, f1 = (p.n_tile / 8) * (rank + 1) / C, nq = (f1 - f0 + kFewStep - 1) / kFewStep;
    const int rows16 = (p.M + 15) / 16;
    for (int w = warp; w < rows16 * nq; w += kFewThreads / 32) {
        const int rb = w / nq, fr = f0 + (w - rb * nq) * kFewStep;
        const int row = rb * 16 + g;
        const bool lo = row < p.M, hi = row + 8 < p.M;
        // N is a multiple of 8: a fragment is within it or past it
        auto there = [&](int j, int e) { return fr + j < f1 && n0 + 8 * (fr + j) < p.N && (e ? hi : lo); };
        auto at = [&](int j, int e) { return (int64_t)(row + 8 * e) * p.N + n0 + 8 * (fr + j) + col; };
        [[maybe_unused]] uint32_t gv[kFewStep][2], uv[kFewStep][2];
        if constexpr (MODE == FEW_GRAD) {
#pragma unroll
            for (int j = 0; j < kFewStep; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    gv[j][e] = uv[j][e] = 0u;
                    if (there(j, e)) {
                        gv[j][e] = *reinterpret_cast<const uint32_t *>(p.gate + at(j, e));  // (not __ldg: tc_ffn.cuh)
                        uv[j][e] = *reinterpret_cast<const uint32_t *>(p.up + at(j, e));
                    }
                }
        }
        float d[kFewStep][kHalves][4];
#pragma unroll
        for (int j = 0; j < kFewStep; ++j)
#pragma unroll
            for (int h = 0; h < kHalves; ++h)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float2 x = there(j, e) ? sum2(row + 8 * e, h * p.n_tile + 8 * (fr + j) + col) : make_float2(0.f, 0.f);
                    d[j][h][2 * e] = x.x;
                    d[j][h][2 * e + 1] = x.y;
                }
        for (int i = 0; i < p.nrank; ++i) {
            const bool second = kHalves == 2 && p.rank[i].half != 0;
            for (int k = 0; k < p.rpad; k += 16) {
                uint32_t a[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)  // rows row, row + 8; k + 2 t, k + 8 + 2 t
                    a[e] = (e & 1 ? hi : lo) ? *reinterpret_cast<const uint32_t *>(
                                                   sv + (row + (e & 1) * 8) * p.vpitch + i * p.rpad + k + (e >> 1) * 8 + col)
                                             : 0u;
#pragma unroll
                for (int j = 0; j < kFewStep; ++j) {
                    if (fr + j >= f1) continue;
                    const __nv_bfloat16 *b = s2 + ((int64_t)i * p.n_tile + 8 * (fr + j) + g) * (p.rpad + 8) + k + col;
                    const uint32_t b0 = *reinterpret_cast<const uint32_t *>(b), b1 = *reinterpret_cast<const uint32_t *>(b + 8);
                    if (second) few_mma(d[j][kHalves - 1], a, b0, b1);
                    else few_mma(d[j][0], a, b0, b1);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < kFewStep; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if (!there(j, e)) continue;
                const int64_t o = at(j, e);
                const float x = d[j][0][2 * e], y = d[j][0][2 * e + 1];
                if constexpr (MODE == FEW_GLU) {
                    const float ux = d[j][kHalves - 1][2 * e], uy = d[j][kHalves - 1][2 * e + 1];
                    float ax, ay, slope;
                    ffn_act(p.act, x, ax, slope);
                    ffn_act(p.act, y, ay, slope);
                    few_put2(p.out[0] + o, ax * ux, ay * uy);
                    if (p.keep) {
                        few_put2(p.out[1] + o, x, y);
                        few_put2(p.out[2] + o, ux, uy);
                    }
                } else if constexpr (MODE == FEW_GRAD) {
                    const float2 gf = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&gv[j][e]));
                    const float2 uf = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&uv[j][e]));
                    float ax, ay, sx, sy;
                    ffn_act(p.act, gf.x, ax, sx);
                    ffn_act(p.act, gf.y, ay, sy);
                    few_put2(p.out[0] + o, x * uf.x * sx, y * uf.y * sy);
                    few_put2(p.out[1] + o, x * ax, y * ay);
                } else {
                    few_put2(p.out[0] + o, x, y);
                }
            }
    }
    if (C > 1) cluster_sync();  // no CTA leaves while another reads its sums
}

}  // namespace attt

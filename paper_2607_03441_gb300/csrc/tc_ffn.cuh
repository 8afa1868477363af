// tc_ffn.cuh -- the tcgen05 contractions of the gated feed-forward block.
//
// D[M x N] = sum over segments A_i B_i^T, bf16 operands, fp32 accumulation; the
// segments follow one another along K (activations with weights, then the
// adapters' rank-r products).  The pipeline is that of tc_gemm.cuh: warps 0 and
// 6 issue TMA loads of 64-deep K blocks into a ring, warp 1 issues the MMAs,
// epilogue warps drain one of two TMEM accumulators while the next tile's MMAs
// fill the other; a tile belongs to one CTA (128 rows) or to a pair (256 rows).
// What is particular to the block:
//   * DUAL: the B tile is half gate, half up weights -- the same columns of both --
//     so that one accumulator tile holds both factors of the same BN / 2 columns
//     of the product, and x is read once for the two.  Weights [K, columns] are
//     read MN-major in 64-column boxes; in a CTA pair the even CTA stages the
//     gate's half and the odd one the up's.  One MMA sees one A for all of its
//     columns, so the adapters' part of K, s (x Ag) beside s (x Au), meets Bg beside
//     zeros and zeros beside Bu: boxes outside a tensor are filled with zeros.
//   * FFN_GLU: the activation of the gate's half times the up's half, in bf16, and
//     if wanted both factors;
//   * FFN_GLU_GRAD: from the product's gradient (the accumulator) and the two
//     factors, those of the factors.
// Bound: tensor cores.  1,024 rows at 3,584 x 18,944: FFN_GLU 152 to 156 us (tensor pipe 91% busy), FFN_OUT over both
// K ranges 149 to 153 (94%), FFN_GLU_GRAD 93 (74%: per tile 2 bytes of each factor in and of each gradient out
// for 2 d operations; with a second set of epilogue warps the same).
#pragma once

#include "gemm_launch.cuh"

namespace attt {

enum FfnEpi : int {
    FFN_GLU = 0,       // h = act(g) u [, g, u]
    FFN_GLU_GRAD = 1,  // dg = dh u act'(g), du = dh act(g)
    FFN_OUT = 2,       // the contraction in bf16
    FFN_PART = 3,      // K pieces of every tile, fp32 (a second kernel sums them)
};
enum FfnAct : int { FFN_SILU = ATTT_SILU, FFN_GELU_TANH = ATTT_GELU_TANH };

// K blocks up to `end`: block j of the segment is A[:, a_k + 64 j ..] with B[:, b_k + 64 j ..]
// (DUAL: b for the gate's half, b2 for the up's), tensor maps by index.
constexpr int kFfnSegs = 4;
struct FfnSeg {
    int a, a_k, b, b_k, b2, b2_k, end;
};

struct FfnMaps {
    CUtensorMap a[3], b[4], c[3];
};

struct FfnArgs {
    GemmArgs g;  // N: columns of the result; tiles_n: tiles of them
    int nseg;
    FfnSeg seg[kFfnSegs];
    int act;
    int keep;  // FFN_GLU: g and u are stored too (maps c[1], c[2])
    // FFN_GLU_GRAD: the factors, [M, N].  dg and du may be written to where they lie (a warp has its 32 x 32 values
    // before it stores over them), so that they are not read as what no one writes (__ldg).
    const __nv_bfloat16 *gate, *up;
};

// a = act(g), slope = act'(g).  Both activations are g p(z), p the logistic function:
// z = g (SiLU), z = 2 sqrt(2 / pi) (g + 0.044715 g^3) (GELU by tanh, since (1 + tanh(y)) / 2 =
// p(2 y)).  Past |g| = 16 the latter's p is 0 or 1 in fp32, so z and the slope's factors
// stop there and stay finite for every number g (a NaN stays one: not by fminf and fmaxf, which drop it).
__device__ __forceinline__ void ffn_act(int act, float g, float &a, float &slope) {
    float z = g, zp = 1.f, c = g;
    if (act == FFN_GELU_TANH) {
        c = fabsf(g) > 16.f ? copysignf(16.f, g) : g;
        const float q = c * c;
        z = 1.5957691216057308f * c * fmaf(0.044715f, q, 1.f);
        zp = 1.5957691216057308f * fmaf(3.f * 0.044715f, q, 1.f);
    }
    const float p = __fdividef(1.f, 1.f + __expf(-z));
    a = g * p;
    slope = p * fmaf(c * (1.f - p), zp, 1.f);
}

__device__ __forceinline__ void ffn_pack(const float (&v)[32], uint32_t (&pk)[16]) {
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
        __nv_bfloat162 b = __floats2bfloat162_rn(v[i], v[i + 1]);
        pk[i / 2] = *reinterpret_cast<uint32_t *>(&b);
    }
}

// 32 bf16 of a row from column x, those from `n` on (a multiple of 8) as zeros.
struct FfnRow {
    uint4 q[4];
    __device__ __forceinline__ void load(const __nv_bfloat16 *row, int x, int n) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            q[i] = row && x + 8 * i < n ? *reinterpret_cast<const uint4 *>(row + x + 8 * i) : make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ float2 pair(int i) const {  // values 2 i, 2 i + 1
        const uint4 &u = q[i >> 2];
        const uint32_t w = (i & 3) == 0 ? u.x : (i & 3) == 1 ? u.y : (i & 3) == 2 ? u.z : u.w;
        return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&w));
    }
};

// FFN_GLU for this warp's 32 rows from y: columns [c0, c1) of the half tile whose first
// column of the product is n0.
__device__ __forceinline__ void ffn_glu_tile(const FfnArgs &p, const FfnMaps &maps, uint32_t sE, uint32_t &ec, int lane,
                                             int y, int n0, int c0, int c1, uint32_t taddr) {
    if (y >= p.g.M) return;  // every row of this warp lies past M (warp-uniform)
    const uint32_t half = (uint32_t)p.g.BN / 2;
    for (int c = c0; c < c1; c += 32) {
        const int x = n0 + c;
        if (x >= p.g.N) break;
        float a[32], u[32];
        tmem_ld_x32(taddr + (uint32_t)c, a);
        tmem_ld_x32(taddr + half + (uint32_t)c, u);
        uint32_t pk[16];
        if (p.keep) {
            ffn_pack(a, pk);
            e_block_store(&maps.c[1], sE, (int)(ec++), lane, pk, x, y);
            ffn_pack(u, pk);
            e_block_store(&maps.c[2], sE, (int)(ec++), lane, pk, x, y);
        }
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            float f, slope;
            ffn_act(p.act, a[i], f, slope);
            a[i] = f * u[i];
        }
        ffn_pack(a, pk);
        e_block_store(&maps.c[0], sE, (int)(ec++), lane, pk, x, y);
    }
}

// FFN_GLU_GRAD for this warp's 32 rows from y: columns [c0, c1) of the tile from column n0.
// The factors of the next 32 columns are loaded while these are worked on; `gu` holds
// those of the first.
__device__ __forceinline__ void ffn_grad_tile(const FfnArgs &p, const FfnMaps &maps, uint32_t sE, uint32_t &ec,
                                              int lane, int y, int n0, int c0, int c1, uint32_t taddr, FfnRow (&gu)[2],
                                              const __nv_bfloat16 *grow, const __nv_bfloat16 *urow) {
    if (y >= p.g.M) return;
    for (int c = c0; c < c1; c += 32) {
        const int x = n0 + c;
        if (x >= p.g.N) break;
        float d[32];
        tmem_ld_x32(taddr + (uint32_t)c, d);
        const FfnRow g = gu[0], u = gu[1];
        if (c + 32 < c1) {
            gu[0].load(grow, x + 32, p.g.N);
            gu[1].load(urow, x + 32, p.g.N);
        }
        uint32_t pg[16], pu[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float2 gv = g.pair(i), uv = u.pair(i);
            float a0, a1, s0, s1;
            ffn_act(p.act, gv.x, a0, s0);
            ffn_act(p.act, gv.y, a1, s1);
            __nv_bfloat162 b = __floats2bfloat162_rn(d[2 * i] * uv.x * s0, d[2 * i + 1] * uv.y * s1);
            pg[i] = *reinterpret_cast<uint32_t *>(&b);
            b = __floats2bfloat162_rn(d[2 * i] * a0, d[2 * i + 1] * a1);
            pu[i] = *reinterpret_cast<uint32_t *>(&b);
        }
        e_block_store(&maps.c[0], sE, (int)(ec++), lane, pg, x, y);
        e_block_store(&maps.c[1], sE, (int)(ec++), lane, pu, x, y);
    }
}

constexpr int ffn_threads(int sets) { return gemm_pair_threads(sets); }

template <int EPI, bool DUAL, bool PAIR, int SETS>
__global__ void __launch_bounds__(ffn_threads(SETS), 1)
    ffn_kernel(const __grid_constant__ FfnMaps maps, const __grid_constant__ FfnArgs p) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const GemmArgs &g = p.g;
    const int S = g.stages;
    const int bn_cta = PAIR ? g.BN / 2 : g.BN;  // B rows that this CTA stages
    const int n_tile = DUAL ? g.BN / 2 : g.BN;  // columns of the result per tile
    const uint32_t b_bytes = gemm_b_stage_bytes(bn_cta);
    uint8_t *sA = smem;
    uint8_t *sB = smem + (size_t)S * kABytes;
    uint8_t *sE = sB + (size_t)S * b_bytes;
    uint64_t *bars = reinterpret_cast<uint64_t *>(sE + g.e_stage_bytes);
    const uint32_t full0 = smem_u32(bars), empty0 = smem_u32(bars + S), tfull0 = smem_u32(bars + 2 * S),
                   tempty0 = smem_u32(bars + 2 * S + 2), drain0 = smem_u32(bars + 2 * S + 4);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + 2 * S + 5);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
    const bool leader = rank == 0;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(full0 + 8 * s, 1);
            mbar_init(empty0 + 8 * s, 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(tfull0 + 8 * a, 1);
            mbar_init(tempty0 + 8 * a, (PAIR ? 8 : 4) * SETS);
        }
        mbar_init(drain0, 1);
        *abort_flag = 0;
        fence_mbar_init();
        for (int i = 0; i < 3; ++i) tma_prefetch_desc(&maps.a[i]);
        for (int i = 0; i < 4; ++i) tma_prefetch_desc(&maps.b[i]);
    }
    if (PAIR) cluster_sync();  // both CTAs' barriers exist before any cross-CTA signal
    if (warp == 1) {
        if (PAIR) {
            tmem_alloc_pair(smem_u32(tmem_slot), g.tmem_cols);
            tmem_relinquish_pair();
        } else {
            tmem_alloc(smem_u32(tmem_slot), g.tmem_cols);
            tmem_relinquish();
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    // not before TMEM is allocated: a CTA of the next grid that shares the SM could otherwise take the columns
    // that this one needs, and wait for this grid
    if (threadIdx.x == 0) griddep_launch_dependents();

    const int tiles_m = PAIR ? (g.tiles_m + 1) / 2 : g.tiles_m;  // of the accumulator's height
    const int nwork = work_count(g, tiles_m);
    const int unit = PAIR ? blockIdx.x >> 1 : blockIdx.x, units = PAIR ? gridDim.x >> 1 : gridDim.x;
    const uint32_t lead_full0 = PAIR ? mapa_shared(full0, 0) : full0;
    const uint32_t lead_tempty0 = PAIR ? mapa_shared(tempty0, 0) : tempty0;

    if (warp == 0 || warp == 6) {
        if (elect_one()) {
            // ---------------- TMA producers (warp 0 even, warp 6 odd stages) ----------------
            bool waited = false;  // for the previous grid
            if (!g.operands_ready) {
                griddep_wait();
                waited = true;
            }
            const uint32_t pid = warp == 0 ? 0u : 1u;
            uint32_t pos = 0;
            int stage = 0;
            uint32_t phase = 0;
            uint32_t issued_mask = 0, issued_parity = 0;  // leader: stages whose bytes it expects
            bool ok = true;
            for (int w = unit; w < nwork && ok; w += units) {
                const Work wi = work_item(g, w, tiles_m);
                const int arow = PAIR ? wi.tm * 256 + 128 * (int)rank : wi.tm * 128;
                const int brow = DUAL ? wi.tn * n_tile : wi.tn * g.BN + (PAIR ? bn_cta * (int)rank : 0);
                int si = 0, first = 0;  // segment of block kb, its first block
                for (int kb = wi.kb0; kb < wi.kb1; ++kb) {
                    if (((pos++) & 1u) != pid) {
                        if (++stage == S) { stage = 0; phase ^= 1u; }
                        continue;
                    }
                    if (!mbar_wait(empty0 + 8 * stage, phase ^ 1u, abort_flag)) { ok = false; break; }
                    while (kb >= p.seg[si].end) first = p.seg[si++].end;
                    const FfnSeg &sg = p.seg[si];
                    if (si > 0 && !waited) {  // what follows the first operands comes from the previous grid
                        griddep_wait();
                        waited = true;
                    }
                    if (leader) {
                        mbar_arrive_expect_tx(full0 + 8 * stage, (PAIR ? 2u : 1u) * (g.a_bytes + b_bytes));
                        issued_mask |= 1u << stage;
                        issued_parity = (issued_parity & ~(1u << stage)) | (phase << stage);
                    }
                    const uint32_t fb = lead_full0 + 8 * stage;
                    const uint32_t a_dst = smem_u32(sA + (size_t)stage * kABytes);
                    const uint32_t b_dst = smem_u32(sB + (size_t)stage * b_bytes);
                    const int j = 64 * (kb - first);
                    auto load = [&](uint32_t dst, const CUtensorMap *tm, int c0, int c1) {
                        if (PAIR) tma_load_2d_pair(dst, tm, fb, c0, c1);
                        else tma_load_2d(dst, tm, fb, c0, c1);
                    };
                    load(a_dst, &maps.a[sg.a], sg.a_k + j, arow);
                    if constexpr (DUAL) {
                        const int boxes = n_tile / 64;
                        for (int b = 0; b < boxes; ++b) {
                            if (!PAIR || rank == 0)
                                load(b_dst + 8192 * b, &maps.b[sg.b], brow + 64 * b, sg.b_k + j);
                            if (!PAIR || rank == 1)
                                load(b_dst + 8192 * (PAIR ? b : boxes + b), &maps.b[sg.b2], brow + 64 * b, sg.b2_k + j);
                        }
                    } else {
                        load(b_dst, &maps.b[sg.b], sg.b_k + j, brow);
                    }
                    if (++stage == S) { stage = 0; phase ^= 1u; }
                }
            }
            if (!ok) {
                *abort_flag = 1;
                record_error(g.status, ATTT_ERR_TIMEOUT);
                // the loads of every stage that the leader expects land on its barrier: wait
                // (bounded, a flag of its own) for them before the CTAs retire
                volatile int no_abort = 0;
                for (int s = 0; s < S; ++s)
                    if (issued_mask & (1u << s))
                        (void)mbar_wait(full0 + 8 * s, (issued_parity >> s) & 1u, &no_abort);
            }
        }
    } else if (warp == 1) {
        if (leader && elect_one()) {
            // ---------------- MMA issuer ----------------
            const uint32_t idesc = idesc_bf16_f32((uint32_t)g.BN, false, DUAL, PAIR ? 256u : 128u);
            int stage = 0;
            uint32_t phase = 0;
            int it = 0;
            bool ok = true, ready = false;
            for (int w = unit; w < nwork && ok; w += units, ++it) {
                const Work wi = work_item(g, w, tiles_m);
                const int acc = it & 1;
                if (!mbar_wait(tempty0 + 8 * acc, (((uint32_t)it >> 1) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
                tc_fence_after();
                const uint32_t d_tmem = tmem_base + (uint32_t)(acc * g.BN);
                for (int kb = wi.kb0; kb < wi.kb1; ++kb) {
                    if (!ready && !mbar_wait(full0 + 8 * stage, phase, abort_flag)) { ok = false; break; }
                    tc_fence_after();
                    // the next stage's barrier is read while this stage's MMAs issue
                    const int next = stage + 1 == S ? 0 : stage + 1;
                    const uint32_t next_phase = next == 0 ? phase ^ 1u : phase;
                    ready = mbar_test_wait(full0 + 8 * next, next_phase);
                    const uint32_t a_addr = smem_u32(sA + (size_t)stage * kABytes);
                    const uint32_t b_addr = smem_u32(sB + (size_t)stage * b_bytes);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk) {
                        const uint64_t ad = smem_desc_sw128(a_addr + kk * 32, 16, 1024);
                        const uint64_t bd = DUAL ? smem_desc_sw128(b_addr + kk * 2048, 8192, 1024)
                                                 : smem_desc_sw128(b_addr + kk * 32, 16, 1024);
                        if (PAIR) umma_bf16_pair(d_tmem, ad, bd, idesc, (kb > wi.kb0 || kk > 0) ? 1u : 0u);
                        else umma_bf16(d_tmem, ad, bd, idesc, (kb > wi.kb0 || kk > 0) ? 1u : 0u);
                    }
                    if (PAIR) umma_commit_pair(empty0 + 8 * stage, 3);
                    else umma_commit(empty0 + 8 * stage);
                    stage = next;
                    phase = next_phase;
                }
                if (!ok) break;
                if (PAIR) umma_commit_pair(tfull0 + 8 * acc, 3);
                else umma_commit(tfull0 + 8 * acc);
            }
            if (!ok) {
                *abort_flag = 1;
                record_error(g.status, ATTT_ERR_TIMEOUT);
            }
            // every MMA issued by this thread completes before TMEM is freed (bounded wait)
            if (PAIR) umma_commit_pair(drain0, 1);
            else umma_commit(drain0);
            volatile int no_abort = 0;
            if (!mbar_wait(drain0, 0u, &no_abort)) record_error(g.status, ATTT_ERR_TIMEOUT);
        }
    } else {
        // ---------------- epilogue (warps 2..5 and 7..10) ----------------
        griddep_wait();  // what the epilogue reads or overwrites may come from the previous grid
        const int q = warp & 3, set = warp >= 7 ? 1 : 0;
        const uint32_t ebuf = smem_u32(sE) + (uint32_t)(q + 4 * set) * 4096u;
        [[maybe_unused]] F32Stage fst{smem_u32(sE) + (uint32_t)q * 8192u, 0u, 0u};
        [[maybe_unused]] uint32_t ec = 0;  // blocks stored by this warp
        int it = 0;
        for (int w = unit; w < nwork; w += units, ++it) {
            const Work wi = work_item(g, w, tiles_m);
            const int acc = it & 1;
            const uint32_t par = ((uint32_t)it >> 1) & 1u;
            const int gm_base = PAIR ? wi.tm * 256 + 128 * (int)rank : wi.tm * 128;
            const int y = gm_base + 32 * q, n0 = wi.tn * n_tile;
            const int c0 = set * (n_tile / SETS), c1 = c0 + n_tile / SETS;
            [[maybe_unused]] const __nv_bfloat16 *grow = nullptr, *urow = nullptr;
            [[maybe_unused]] FfnRow gu[2];
            if constexpr (EPI == FFN_GLU_GRAD) {
                if (y + lane < g.M) {
                    grow = p.gate + (int64_t)(y + lane) * g.N;
                    urow = p.up + (int64_t)(y + lane) * g.N;
                }
                gu[0].load(grow, n0 + c0, g.N);
                gu[1].load(urow, n0 + c0, g.N);
            }
            int ok = 1;
            if (lane == 0) ok = mbar_wait(tfull0 + 8 * acc, par, abort_flag) ? 1 : 0;
            // one decision for all epilogue warps
            ok = named_barrier_and(1, 128 * SETS, __shfl_sync(0xffffffffu, ok, 0));
            if (!ok) {
                if (lane == 0) { *abort_flag = 1; record_error(g.status, ATTT_ERR_TIMEOUT); }
                break;
            }
            (void)mbar_try_wait(tfull0 + 8 * acc, par);  // per-thread acquire of the completed phase
            tc_fence_after();
            const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * g.BN);
            if constexpr (EPI == FFN_GLU) {
                ffn_glu_tile(p, maps, ebuf, ec, lane, y, n0, c0, c1, taddr);
            } else if constexpr (EPI == FFN_GLU_GRAD) {
                ffn_grad_tile(p, maps, ebuf, ec, lane, y, n0, c0, c1, taddr, gu, grow, urow);
            } else if constexpr (EPI == FFN_OUT) {
                bf16_tile_store(g, &maps.c[0], ebuf, ec, lane, y, n0, min(g.N, n0 + g.BN),
                                [&](int c, float(&v)[32]) { tmem_ld_x32(taddr + (uint32_t)c, v); });
            } else {
                if (y < g.M)
                    f32_part_store(g, &maps.c[0], fst, lane,
                                   (int)part_row(wi.tm, wi.tn, tiles_m, wi.piece, g.tail_s, PAIR ? 256 : 128) +
                                       128 * (int)rank + 32 * q,
                                   DUAL ? g.BN : min(g.N - n0, g.BN), taddr);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (PAIR) mbar_arrive_cluster(lead_tempty0 + 8 * acc);
                else mbar_arrive(tempty0 + 8 * acc);
            }
        }
        // every TMA store of the epilogue has landed before the CTA retires
        if (lane == 0) bulk_wait<0>();
    }

    tc_fence_before();
    if (PAIR) cluster_sync();  // no CTA leaves while the pair's MMAs or signals are in flight
    else __syncthreads();
    tc_fence_after();
    if (warp == 1) {
        if (PAIR) tmem_dealloc_pair(tmem_base, g.tmem_cols);
        else tmem_dealloc(tmem_base, g.tmem_cols);
    }
}

}  // namespace attt

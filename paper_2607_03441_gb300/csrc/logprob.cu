// logprob.cu -- log probabilities of given tokens through the frozen LM head,
// with the entropy of every row's distribution and its most probable
// alternatives, and their gradient with respect to the hidden states; the
// [L, V] logits never reach HBM.
//
// With z = h W^T, T the temperature, p = softmax(z / T):
//   logp_j = z_{j,t_j} / T - lse_j,   lse_j = log sum_v exp(z_jv / T),
//   H_j = -sum_v p_jv log p_jv.
// Forward: one contraction over the whole vocabulary (2 L V d FLOPs).  Every SM, or pair
// of SMs, takes a run of tiles along rows; its epilogue keeps each row's max, the sum of
// exponentials, that sum's first moment, and its few largest logits in registers from
// tile to tile (tc_gemm.cuh, EPI_LOGP*); a second kernel merges a row's runs.
// Gradient: with given da_j = dL/dlogp_j and db_j = dL/dH_j,
//   dL/dz_jv = (da_j [v = t_j] - p_jv (da_j + db_j (log p_jv + H_j))) / T,
// formed from the logits in the epilogue of the same contraction (the
// softmax needs no second sweep: lse and H are the forward call's) as a bf16 block
// G, then dh = G W (4 L V d FLOPs: the logits are formed again).
// The gradient takes rows in blocks so that G stays bounded.
// Bound: the tensor core from a few hundred rows on, the head's bytes below.  Through a head
// of 152,064 x 3,584: 2,048 rows with 8 alternatives 1.16 ms (the burst GEMM rate), 403 rows
// 324 us (of which a fifth is the padding to 512), the gradient of 93 rows 341 us (the
// head is read twice: 322 of bytes); of 4,096 rows through 152,064 x 5,120 7.1 ms (1.79
// PFLOP/s).
#include <algorithm>

#include "gemm_launch.cuh"

namespace attt {

constexpr int kLpTopMax = 20;
constexpr int kLpUnits = 160;  // SMs, or pairs of SMs, that take runs, at most
constexpr int kLpWarps = 16;   // of a reduction block
constexpr int64_t kLpGBytes = 2048ll << 20;  // the gradient block of a row block, at most
constexpr int64_t kLpHiddenBytes = 48ll << 20;  // the hidden states of a row block of the forward call, at most
constexpr int64_t kLpHeadBytes = 48ll << 20;    // a head that L2 holds beside them (tc_gemm.cuh: Span)
constexpr int64_t kLpRunRows = 16384;           // and its rows
constexpr int kFewRows = 32;  // rows of a call that reads the head as the M operand, at most
// Rows of a gradient call whose block takes two bf16 per value, at most: both blocks fit one
// tile of 128 rows.  More would pay for what they do not need, as dh is rounded to bf16 itself
// (1.66e-3 of its norm): 93 rows x 3,584 through 152,064 340 us with one, error 1.79e-3, and
// 367 with two, 1.67e-3; 4,096 x 5,120 7.1 ms, 1.84e-3, and 11.3 ms, 1.68e-3.
constexpr int kLoRows = 64;
constexpr int kLpSplitRegions = 320;  // K pieces of the second contraction: 128 KB each

inline int lp_sets(int64_t d) { return cdiv(d, 64) <= kTwoSetBlocks ? 2 : 1; }
// Rows of a block of `total` rows at `row_bytes` of workspace each: equal blocks, a
// multiple of 256.
inline int64_t lp_block_rows(int64_t total, int64_t row_bytes, int64_t bound) {
    int64_t most = bound / row_bytes / 256 * 256;
    if (most < 256) most = 256;
    if (total <= most) return total;
    return round_up(cdiv(total, cdiv(total, most)), 256);
}

struct LpLayout {
    int64_t plane, ld;  // elements of a plane [slots, L]; places for a row's largest logits
    float *part, *ztgt, *top_v;
    int32_t *top_i;
    size_t bytes;
};

// Rows of a block, all of whose tiles share the head's from L2: their hidden states stay
// there too, and a run is at most a row of tiles long.
inline int64_t lp_forward_rows(int64_t L, int64_t d) {
    return lp_block_rows(L, 2 * d, std::min<int64_t>(kLpHiddenBytes, 2 * d * kLpRunRows));
}

// Slots: U units of runs over m rows of tiles leave at most U / m + 2 runs in each (a
// run and its neighbours' ends), and no more than U, of up to two slots each if m > 1
// (tc_gemm.cuh: logp_flush).
static LpLayout lp_layout(void *ws, int64_t L, int64_t d, int64_t V, int topk) {
    LpLayout c{};
    const int64_t rows = L <= kFewRows ? L : lp_forward_rows(L, d), least = L % rows ? L % rows : rows;
    auto slots = [](int64_t r) {
        return r <= 128 ? kLpUnits : 2 * std::min<int64_t>(kLpUnits, kLpUnits / cdiv(r, 256) + 2);
    };
    c.plane = std::max(slots(rows) * rows, slots(least) * least) * (L <= kFewRows ? 1 : lp_sets(d));
    c.ld = L <= kFewRows ? 32 : round_up(topk, 4);
    const int64_t tops = topk > 0 ? c.plane * c.ld : 0;
    Carve cv{static_cast<char *>(ws), 0};
    c.part = cv.take<float>((size_t)(3 * c.plane));
    c.ztgt = cv.take<float>((size_t)L);
    c.top_v = cv.take<float>((size_t)tops);
    c.top_i = cv.take<int32_t>((size_t)tops);
    c.bytes = (size_t)round_up((int64_t)cv.used, 256);
    return c;
}

// (max, sum, moment) of some of a row's logits, as epilogue_logp forms them: the sum leaves
// out the max's own term, which is 1.  While the max is -inf the sum means nothing but that
// it may be NaN.
struct LpPart {
    float m, s, t;
    __device__ __forceinline__ void merge(const LpPart &o, float c2) {
        const bool mine = m >= o.m;
        const LpPart lo = mine ? o : *this, hi = mine ? *this : o;
        if (hi.m == -INFINITY) {
            s += o.s;
            return;
        }
        const float d = (lo.m - hi.m) * c2, f = ex2(d), n = 1.f + lo.s;
        t = fmaf(f, fmaf(n, fmaxf(d, -1e4f), lo.t), hi.t);
        s = fmaf(f, n, hi.s);
        m = hi.m;
    }
    __device__ __forceinline__ LpPart shfl_xor(int o) const {
        return LpPart{__shfl_xor_sync(0xffffffffu, m, o), __shfl_xor_sync(0xffffffffu, s, o),
                      __shfl_xor_sync(0xffffffffu, t, o)};
    }
};

struct LpReduceArgs {
    const float *part, *ztgt, *top_v;
    const int32_t *top_i;
    int64_t plane;
    // sets of a row: `nsets`, or (tile_rows > 0) those of its row tile's runs (tc_gemm.cuh: logp_flush)
    int nsets, tile_rows, tiles_n, nwork, units, sets, split;
    int rows, V, topk, top_ld;
    float inv_temp;
    const int32_t *tgt;
    float *logp, *entropy, *lse, *top_logp;
    int32_t *top_id;
    int *status;
};

// The log of a row's whole sum (in units of the max's term): small values keep their 24 bits,
// and with them the entropies and log probabilities of rows that are nearly sure.
__device__ __forceinline__ float lp_log_sum(const LpPart &p) {
    if (p.m == -INFINITY) return logf(p.s);
    return p.m < INFINITY ? log1pf(p.s) : __int_as_float(0x7fc00000);
}

// A row's lse, entropy and log probability of its given token, from its (max, sum,
// moment) and that log.
__device__ __forceinline__ void lp_row(const LpReduceArgs &a, int j, const LpPart &p, float ln) {
    if (a.lse) a.lse[j] = fmaf(p.m, a.inv_temp, ln);
    if (a.entropy) a.entropy[j] = ln - 0.69314718055994531f * (p.t / (p.m == -INFINITY ? p.s : 1.f + p.s));
    if (a.logp) {
        const int t = a.tgt[j];
        float lp = 0.f;
        if (t >= 0 && t < a.V) {
            lp = (__ldcg(a.ztgt + j) - p.m) * a.inv_temp - ln;
        } else if (t != -1) {
            record_error(a.status, ATTT_ERR_TOKEN_RANGE);
            lp = __int_as_float(0x7fc00000);
        }
        a.logp[j] = lp;
    }
}

// ---------------------------------------------------------------------------
// Few rows (single tokens of some episodes): the head is read once and bounds the
// call, so its rows go to the M side of the MMAs (128 vocabulary ids x 16 or 32 hidden
// states, nothing padded to 128 rows), and the epilogue works across the lanes, one
// vocabulary id each.  A lane keeps the (max, sum, moment) of its own ids for each of
// 16 rows from tile to tile; a warp keeps each row's 32 largest logits, one per
// lane in order, and merges a tile's 32 new ones into them (sorted by 15 exchanges,
// merged by 5) or, where at most two beat the least that counts, inserts those.  At the
// end of the kernel a CTA's four warps merge, and one block per row merges the CTAs.
// Through 152,064 x 3,584 with 5 alternatives one row takes 165 us (98% of the copy
// bandwidth; 228 with the row padded to 128 and the alternatives kept by its one lane),
// 16 rows through 152,064 x 5,120 with 20 take 236 (97%; 307).  A small head is bound by
// the exchanges, each of which waits for the one before: those of four rows go side by
// side, and so do the merges of a level (24 rows x 648 through 16,971 with 5: 22.5 us, 41
// row by row and list by list).
// ---------------------------------------------------------------------------

constexpr int kFewMaxStages = 10;

// A place of a list: larger keys are larger logits, of equal ones the lower id.  Empty: -inf
// and id -1, after every id.
using LpKey = unsigned long long;
constexpr LpKey kLpNone = 0x007fffffull << 32;
__device__ __forceinline__ LpKey lp_key(float v, int id) {  // v not NaN
    const uint32_t u = __float_as_uint(v + 0.f);  // -0 is equal to 0
    return (LpKey)((int)u < 0 ? ~u : u | 0x80000000u) << 32 | ~(uint32_t)id;
}
__device__ __forceinline__ float lp_value(LpKey k) {
    const uint32_t u = (uint32_t)(k >> 32);
    return __uint_as_float((int)u < 0 ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ int lp_id(LpKey k) { return (int)~(uint32_t)k; }

// One compare-exchange of a warp-wide sort: the lane keeps the larger of its own and its
// partner's (lane ^ o) where `first`, else the smaller.
__device__ __forceinline__ void lp_exchange(LpKey &k, int o, bool first) {
    const LpKey other = __shfl_xor_sync(0xffffffffu, k, o);
    if ((other > k) == first) k = other;
}

// Sorts the warp's 32 places, lane 0 the first.
__device__ __forceinline__ void lp_sort(LpKey &v, int lane) {
#pragma unroll
    for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
        for (int o = k >> 1; o > 0; o >>= 1) lp_exchange(v, o, ((lane & o) == 0) == ((lane & k) == 0));
}

// v: the first 32 of two sorted lists.
__device__ __forceinline__ void lp_merge(LpKey &v, LpKey o, int lane) {
    o = __shfl_xor_sync(0xffffffffu, o, 31);
    if (o > v) v = o;
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) lp_exchange(v, s, (lane & s) == 0);
}

// Four lists and a tile's 32 logits for each, sorted and merged into them: exchanges of
// one list wait for each other, those of four fill the time.  A call, not one copy per four
// rows: a call of few tiles would spend its time on fetching them.
struct LpKeys {
    LpKey k[4];
};
__device__ __noinline__ LpKeys lp_sort_in(LpKeys l, LpKeys n, int lane) {
#pragma unroll
    for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
        for (int o = k >> 1; o > 0; o >>= 1)
#pragma unroll
            for (int r = 0; r < 4; ++r) lp_exchange(n.k[r], o, ((lane & o) == 0) == ((lane & k) == 0));
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const LpKey o = __shfl_xor_sync(0xffffffffu, n.k[r], 31);
        if (o > l.k[r]) l.k[r] = o;
    }
#pragma unroll
    for (int s = 16; s > 0; s >>= 1)
#pragma unroll
        for (int r = 0; r < 4; ++r) lp_exchange(l.k[r], s, (lane & s) == 0);
    return l;
}

// The places of `mask` of one tile's 32 into a list, one by one.
__device__ __forceinline__ void lp_insert(LpKey &l, LpKey n, unsigned mask, int lane) {
    while (mask) {
        const LpKey k = __shfl_sync(0xffffffffu, n, __ffs(mask) - 1);
        mask &= mask - 1;
        const int at = __popc(__ballot_sync(0xffffffffu, l >= k));
        const LpKey up = __shfl_up_sync(0xffffffffu, l, 1);
        if (lane >= at) l = lane > at ? up : k;
    }
}

struct FewArgs {
    int L, V, kb, stages, tiles, topk;
    float c2;  // log2 e / T
    const int32_t *tgt;
    float *ztgt;
    float *part;   // [CTAs][L] max, then sum, then moment, kLpUnits * L apart
    float *top_v;  // [CTAs][L][32]
    int32_t *top_i;
    int *status;
};

// Warps: 0 TMA producer, 1 MMA, then four per 16 rows.
__host__ __device__ constexpr int few_threads(int sets) { return 64 + 128 * sets; }
__host__ __device__ constexpr uint32_t few_stage_bytes(int sets) { return kABytes + 2048u * sets; }

template <bool TOP, int SETS>
__global__ void __launch_bounds__(few_threads(SETS), 1)
    logprob_few_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmH,
                       const FewArgs a) {
    constexpr int N = 16 * SETS;
    constexpr uint32_t kStage = few_stage_bytes(SETS), kCols = SETS == 1 ? 32 : 64;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int S = a.stages;
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + (size_t)S * kStage);
    const uint32_t full0 = smem_u32(bars), empty0 = smem_u32(bars + S), tfull0 = smem_u32(bars + 2 * S),
                   tempty0 = smem_u32(bars + 2 * S + 2), drain0 = smem_u32(bars + 2 * S + 4);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + 2 * S + 5);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(full0 + 8 * s, 1);
            mbar_init(empty0 + 8 * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(tfull0 + 8 * b, 1);
            mbar_init(tempty0 + 8 * b, 4 * SETS);
        }
        mbar_init(drain0, 1);
        *abort_flag = 0;
        fence_mbar_init();
        tma_prefetch_desc(&tmW);
        tma_prefetch_desc(&tmH);
        griddep_launch_dependents();
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(tmem_slot), kCols);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;

    if (warp == 0) {
        if (elect_one()) {
            int stage = 0;
            uint32_t phase = 0, issued_mask = 0, issued_parity = 0;
            bool ok = true;
            for (int w = blockIdx.x; w < a.tiles && ok; w += gridDim.x) {
                for (int kb = 0; kb < a.kb; ++kb) {
                    if (!mbar_wait(empty0 + 8 * stage, phase ^ 1u, abort_flag)) { ok = false; break; }
                    const uint32_t fb = full0 + 8 * stage, dst = smem_u32(smem + (size_t)stage * kStage);
                    mbar_arrive_expect_tx(fb, kStage);
                    tma_load_2d(dst, &tmW, fb, kb * 64, w * 128);
                    tma_load_2d(dst + kABytes, &tmH, fb, kb * 64, 0);
                    issued_mask |= 1u << stage;
                    issued_parity = (issued_parity & ~(1u << stage)) | (phase << stage);
                    if (++stage == S) { stage = 0; phase ^= 1u; }
                }
            }
            if (!ok) {
                *abort_flag = 1;
                record_error(a.status, ATTT_ERR_TIMEOUT);
                // every load already issued lands before the CTA retires (bounded)
                volatile int no_abort = 0;
                for (int s = 0; s < S; ++s)
                    if (issued_mask & (1u << s)) (void)mbar_wait(full0 + 8 * s, (issued_parity >> s) & 1u, &no_abort);
            }
        }
    } else if (warp == 1) {
        if (elect_one()) {
            const uint32_t idesc = idesc_bf16_f32(N, false, false);
            int stage = 0, it = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int w = blockIdx.x; w < a.tiles && ok; w += gridDim.x, ++it) {
                const int acc = it & 1;
                if (!mbar_wait(tempty0 + 8 * acc, (((uint32_t)it >> 1) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
                tc_fence_after();
                for (int kb = 0; kb < a.kb; ++kb) {
                    if (!mbar_wait(full0 + 8 * stage, phase, abort_flag)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t at = smem_u32(smem + (size_t)stage * kStage);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)
                        umma_bf16(tmem_base + (uint32_t)(acc * N), smem_desc_sw128(at + kk * 32, 16, 1024),
                                  smem_desc_sw128(at + kABytes + kk * 32, 16, 1024), idesc, (kb > 0 || kk > 0) ? 1u : 0u);
                    umma_commit(empty0 + 8 * stage);
                    if (++stage == S) { stage = 0; phase ^= 1u; }
                }
                if (!ok) break;
                umma_commit(tfull0 + 8 * acc);
            }
            if (!ok) {
                *abort_flag = 1;
                record_error(a.status, ATTT_ERR_TIMEOUT);
            }
            umma_commit(drain0);
            volatile int no_abort = 0;
            if (!mbar_wait(drain0, 0u, &no_abort)) record_error(a.status, ATTT_ERR_TIMEOUT);
        }
    } else {
        const int q = warp & 3, set = (warp - 2) >> 2, row0 = 16 * set, rows = min(16, a.L - row0);
        LpPart st[16];
        LpKeys top[TOP ? 4 : 1];
#pragma unroll
        for (int t = 0; t < 16; ++t) {
            st[t] = LpPart{-INFINITY, 0.f, 0.f};
            if constexpr (TOP) top[t / 4].k[t % 4] = kLpNone;
        }
        // the given token of row row0 + (lane & 15) in this lane
        const int given = a.tgt && (lane & 15) < rows ? __ldg(a.tgt + row0 + (lane & 15)) : -1;
        bool ok = true;
        int it = 0;
        for (int w = blockIdx.x; w < a.tiles && ok; w += gridDim.x, ++it) {
            const int acc = it & 1;
            int up = 1;
            if (lane == 0) up = mbar_wait(tfull0 + 8 * acc, ((uint32_t)it >> 1) & 1u, abort_flag) ? 1 : 0;
            ok = __shfl_sync(0xffffffffu, up, 0) != 0;
            if (!ok) {
                if (lane == 0) {
                    *abort_flag = 1;
                    record_error(a.status, ATTT_ERR_TIMEOUT);
                }
                break;
            }
            (void)mbar_try_wait(tfull0 + 8 * acc, ((uint32_t)it >> 1) & 1u);  // per-thread acquire
            tc_fence_after();
            float v[16];
            tmem_ld_x16(tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * N + row0), v);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(tempty0 + 8 * acc);
            const int id = w * 128 + q * 32 + lane;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                if (4 * g >= rows) break;  // warp-uniform
                LpKeys n;
                unsigned mask[4];
                bool many = false;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int t = 4 * g + r;
                    const float z = id < a.V && t < rows ? v[t] : -INFINITY;
                    if (__shfl_sync(0xffffffffu, given, t) == id && id < a.V) a.ztgt[row0 + t] = z;
                    // the lane's running max moves to z, or z counts against it; -inf adds nothing,
                    // NaN reaches the sum
                    if (z != -INFINITY) {
                        const bool above = z > st[t].m;
                        const float d = (above ? st[t].m - z : z - st[t].m) * a.c2, e = ex2(d), dm = fmaxf(d, -1e4f);
                        if (above) {
                            st[t].t = e * fmaf(1.f + st[t].s, dm, st[t].t);
                            st[t].s = fmaf(st[t].s, e, e);
                            st[t].m = z;
                        } else {
                            st[t].t = fmaf(e, dm, st[t].t);
                            st[t].s += e;
                        }
                    }
                    __syncwarp();
                    if constexpr (TOP) {  // those above the least that counts
                        n.k[r] = z > -INFINITY ? lp_key(z, id) : kLpNone;
                        mask[r] = __ballot_sync(0xffffffffu,
                                                n.k[r] > __shfl_sync(0xffffffffu, top[g].k[r], a.topk - 1));
                        many |= __popc(mask[r]) > 2;
                    }
                }
                if constexpr (TOP) {
                    if (many) {
                        top[g] = lp_sort_in(top[g], n, lane);
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r) lp_insert(top[g].k[r], n.k[r], mask[r], lane);
                    }
                }
            }
        }
        // the four warps of a set through shared memory: every MMA has completed, and with it
        // every load into the ring
        LpPart *sp = reinterpret_cast<LpPart *>(smem) + set * 16 * 4;
        LpKey *sk = reinterpret_cast<LpKey *>(smem + 2048) + set * 16 * 4 * 32;
        // a lane's 16 sums over the warp: with every exchange half as many rows and twice as many
        // lanes in each sum, until lanes 2 t and 2 t + 1 hold row t's
#pragma unroll
        for (int o = 16, n = 8; n > 0; o >>= 1, n >>= 1) {
            const bool up = lane & o;
#pragma unroll
            for (int t = 0; t < n; ++t) {
                const LpPart mine = up ? st[t + n] : st[t];
                st[t] = (up ? st[t] : st[t + n]).shfl_xor(o);
                st[t].merge(mine, a.c2);
            }
        }
        st[0].merge(st[0].shfl_xor(1), a.c2);
        if ((lane & 1) == 0) sp[(lane >> 1) * 4 + q] = st[0];
        if constexpr (TOP) {
#pragma unroll
            for (int t = 0; t < 16; ++t)
                if (t < rows) sk[(t * 4 + q) * 32 + lane] = top[t / 4].k[t % 4];
        }
        named_barrier_sync(1u + set, 128);
        const int64_t plane = (int64_t)kLpUnits * a.L;
        if (q == 0 && lane < rows) {
            LpPart p = sp[lane * 4];
#pragma unroll
            for (int k = 1; k < 4; ++k) p.merge(sp[lane * 4 + k], a.c2);
            const int64_t o = (int64_t)blockIdx.x * a.L + row0 + lane;
            a.part[o] = p.m;
            a.part[plane + o] = p.s;
            a.part[2 * plane + o] = p.t;
        }
        if constexpr (TOP) {
            for (int t = q; t < rows; t += 4) {
                const int64_t o = (int64_t)blockIdx.x * a.L + row0 + t;
                LpKey x = sk[t * 4 * 32 + lane], y = sk[(t * 4 + 2) * 32 + lane];
                lp_merge(x, sk[(t * 4 + 1) * 32 + lane], lane);
                lp_merge(y, sk[(t * 4 + 3) * 32 + lane], lane);
                lp_merge(x, y, lane);
                a.top_v[o * 32 + lane] = lp_value(x);
                a.top_i[o * 32 + lane] = lp_id(x);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_dealloc(tmem_base, kCols);
}

// Merges a row's sets: WARPS warps per row, each every WARPS-th set, some at a time on
// their way, then the warps' in pairs (ties of alternatives go to the lowest id, sums are
// in a fixed order).  FEW: the sets of a call of few rows, one per CTA and each with 32
// alternatives, all on their way at once (13 rows through 33,364 x 3,368: 3 us of the call
// against the loops that other calls take).
template <bool TOP, int WARPS, bool FEW>
__global__ void __launch_bounds__(kLpWarps * 32) logprob_reduce_kernel(const LpReduceArgs a) {
    __shared__ LpPart s_part[kLpWarps];
    __shared__ LpKey s_top[TOP && WARPS > 1 ? kLpWarps : 1][32];
    griddep_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, w = warp % WARPS;
    const int j = blockIdx.x * (kLpWarps / WARPS) + warp / WARPS;
    const bool row = j < a.rows;
    const float c2 = a.inv_temp * kLog2e;
    LpPart p{-INFINITY, 0.f, 0.f};
    LpKey top = kLpNone;
    if constexpr (FEW) {
        constexpr int kEach = kLpUnits / WARPS;
        const int t = w + lane * WARPS;
        const int64_t o = (int64_t)t * a.rows + j;
        if (lane < kEach && t < a.nsets)
            p = LpPart{__ldcg(a.part + o), __ldcg(a.part + a.plane + o), __ldcg(a.part + 2 * a.plane + o)};
        if constexpr (TOP) {
            LpKey n[kEach];
#pragma unroll
            for (int k = 0; k < kEach; ++k) {
                const int t = w + k * WARPS;
                const int64_t o = ((int64_t)t * a.rows + j) * 32 + lane;
                const float v = t < a.nsets ? __ldcg(a.top_v + o) : -INFINITY;
                n[k] = lp_key(v, t < a.nsets ? __ldcg(a.top_i + o) : -1);
            }
#pragma unroll
            for (int h = 1; h < kEach; h *= 2)  // pairs of pairs: a level's merges do not wait for each other
#pragma unroll
                for (int k = 0; k + h < kEach; k += 2 * h) lp_merge(n[k], n[k + h], lane);
            top = n[0];
        }
    } else {
        const int first = j / a.tile_rows * a.tiles_n;
        const int units = run_unit(a.nwork, first + a.tiles_n - 1, a.units) - run_unit(a.nwork, first, a.units) + 1;
        const int nsets = row ? a.sets * units * (a.split ? 2 : 1) : 0;
        for (int t = w + lane * WARPS; t < nsets; t += 32 * WARPS) {
            const int64_t o = (int64_t)t * a.rows + j;
            p.merge(LpPart{__ldcg(a.part + o), __ldcg(a.part + a.plane + o), __ldcg(a.part + 2 * a.plane + o)}, c2);
        }
        if constexpr (TOP) {
            for (int t0 = w; t0 < nsets; t0 += 4 * WARPS) {
                LpKey n[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int t = t0 + k * WARPS;
                    const int64_t o = ((int64_t)t * a.rows + j) * a.top_ld + lane;
                    const bool in = lane < a.topk && t < nsets;
                    const float v = in ? __ldcg(a.top_v + o) : -INFINITY;
                    n[k] = lp_key(v, in ? __ldcg(a.top_i + o) : -1);
                }
                lp_merge(n[0], n[1], lane);
                lp_merge(n[2], n[3], lane);
                lp_merge(n[0], n[2], lane);
                lp_merge(top, n[0], lane);
            }
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) p.merge(p.shfl_xor(o), c2);
    if constexpr (WARPS > 1) {
        if (lane == 0) s_part[warp] = p;
        if constexpr (TOP) {
            // half of the warps that hold a list take the other half's
            for (int n = WARPS / 2; n > 0; n /= 2) {
                s_top[warp][lane] = top;
                __syncthreads();
                if (w < n) lp_merge(top, s_top[warp + n][lane], lane);
                __syncthreads();
            }
        } else {
            __syncthreads();
        }
        if (w > 0) return;
        p = lane < WARPS ? s_part[warp + lane] : LpPart{-INFINITY, 0.f, 0.f};
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) p.merge(p.shfl_xor(o), c2);
    }
    if (!row) return;
    const float ln = lp_log_sum(p);
    if (lane == 0) lp_row(a, j, p, ln);
    if constexpr (TOP) {
        if (lane < a.topk) {
            a.top_logp[(int64_t)j * a.topk + lane] = (lp_value(top) - p.m) * a.inv_temp - ln;
            a.top_id[(int64_t)j * a.topk + lane] = lp_id(top);
        }
    }
}

template <bool TOP, int WARPS, bool FEW>
static attt_status launch_reduce_as(const LpReduceArgs &a, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)cdiv(a.rows, kLpWarps / WARPS));
    cfg.blockDim = dim3(kLpWarps * 32);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, logprob_reduce_kernel<TOP, WARPS, FEW>, a) != cudaSuccess) return ATTT_ERR_CUDA;
    count_launch();
    return cudaGetLastError() == cudaSuccess ? ATTT_OK : ATTT_ERR_CUDA;
}

// The fewer rows, the more sets each has (and SMs to spare): a block per row, half of one,
// or a warp.  Hidden size 752 through 13,323, us a call with 16 / 8 / 1 warps per row: with 8
// alternatives 500 rows 41 / 41 / 70, 1,000 rows 60 / 53 / 63, 2,000 rows 94 / 76 / 72;
// without, 1,000 rows 28.8 / 27.4 / 26.1.  (171 rows x 1,424 through 12,055 with one: 22.6 / 32 / 70.)
template <bool TOP>
static attt_status launch_reduce(const LpReduceArgs &a, cudaStream_t stream) {
    if (a.tile_rows == 0) return launch_reduce_as<TOP, kLpWarps, true>(a, stream);
    if (a.rows <= 384) return launch_reduce_as<TOP, kLpWarps, false>(a, stream);
    if constexpr (TOP)
        if (a.rows <= 1536) return launch_reduce_as<TOP, kLpWarps / 2, false>(a, stream);
    return launch_reduce_as<TOP, 1, false>(a, stream);
}

template <bool TOP, int SETS>
static attt_status launch_few(const attt_bf16 *d_h, int64_t h_ld, const attt_bf16 *d_W, int64_t d, FewArgs f,
                              LpReduceArgs a, int dev, cudaStream_t stream) {
    CUtensorMap tw, th;
    if (!make_tmap_bf16(&tw, d_W, (uint64_t)d, (uint64_t)f.V, (uint64_t)d * 2, 64, 128) ||
        !make_tmap_bf16(&th, d_h, (uint64_t)d, (uint64_t)f.L, (uint64_t)h_ld * 2, 64, 16 * SETS))
        return ATTT_ERR_INVALID_ARG;
    auto kern = logprob_few_kernel<TOP, SETS>;
    f.kb = (int)cdiv(d, 64);
    f.tiles = (int)cdiv(f.V, 128);
    f.stages = kFewMaxStages;
    const size_t smem = 1024 + (size_t)f.stages * few_stage_bytes(SETS) + 8 * (2 * f.stages + 5) + 16;
    if (!set_smem_limit(reinterpret_cast<const void *>(kern), smem, dev)) return ATTT_ERR_CUDA;
    const int ctas = std::min({f.tiles, num_sms(dev), kLpUnits});
    kern<<<ctas, few_threads(SETS), smem, stream>>>(tw, th, f);
    count_launch();
    if (cudaGetLastError() != cudaSuccess) return ATTT_ERR_CUDA;
    a.nsets = ctas;
    return launch_reduce<TOP>(a, stream);
}

template <int EPI>
static attt_status launch_logits(const GemmProblem &p, const EpiParams &ep, int sets, int dev, cudaStream_t stream) {
    return sets == 2 ? launch_gemm<EPI, false, false, 2>(p, ep, dev, stream)
                     : launch_gemm<EPI, false, false, 1>(p, ep, dev, stream);
}

struct GradLayout {
    int64_t rows, ld;
    int regions;
    bool lo;  // G's rows, then those of what rounding to them took away
    __nv_bfloat16 *G;
    float *loss;
    float *split_ws;
    unsigned int *split_tick;
    size_t bytes;
};

static GradLayout grad_layout(void *ws, int64_t L, int64_t d, int64_t V) {
    GradLayout c{};
    c.ld = round_up(V, 64);
    c.rows = lp_block_rows(L, 2 * c.ld, kLpGBytes);
    const int64_t t2 = 2 * kMaxPieces * cdiv(c.rows, 256) * cdiv(d, 256);
    c.regions = (int)(t2 < kLpSplitRegions ? t2 : kLpSplitRegions);
    c.lo = L <= kLoRows;
    // the sum that joins G's two blocks reads partials: those of a row of whole tiles fit at least
    // (up to 256 accumulator rows of d columns and of what a tile is wider)
    if (c.lo) c.regions = (int)std::max<int64_t>(c.regions, 2 * (cdiv(d, 256) + 1));
    Carve cv{static_cast<char *>(ws), 0};
    c.G = cv.take<__nv_bfloat16>((size_t)((c.lo ? 2 : 1) * c.rows * c.ld));
    c.loss = cv.take<float>((size_t)c.rows);
    c.split_ws = cv.take<float>((size_t)c.regions * 128 * 256);
    c.split_tick = cv.take<unsigned int>((size_t)c.regions);
    c.bytes = (size_t)round_up((int64_t)cv.used, 256);
    return c;
}

// The sizes that both calls and their workspaces take.
static attt_status lp_sizes(int64_t L, int64_t d, int64_t V) {
    if (L < 1 || V < 1 || d < 8 || d % 8 != 0) return ATTT_ERR_INVALID_ARG;
    return L > (1ll << 30) || V > (1ll << 30) || d > (1ll << 20) ? ATTT_ERR_UNSUPPORTED : ATTT_OK;
}

// What both calls ask of their operands.
static attt_status lp_check(const attt_bf16 *d_h, int64_t h_ld, const attt_bf16 *d_W, int64_t L, int64_t d, int64_t V,
                            float inv_temp) {
    if (!d_h || !d_W || h_ld < d || h_ld % 8 != 0) return ATTT_ERR_INVALID_ARG;
    if (!(inv_temp > 0.f) || !(inv_temp <= 1e4f)) return ATTT_ERR_INVALID_ARG;
    const attt_status st = lp_sizes(L, d, V);
    if (st != ATTT_OK) return st;
    if (h_ld > (1ll << 36)) return ATTT_ERR_UNSUPPORTED;
    if (!aligned16(d_h) || !aligned16(d_W)) return ATTT_ERR_INVALID_ARG;
    return ATTT_OK;
}

}  // namespace attt

extern "C" {

size_t attt_logprob_workspace_bytes(int64_t L, int64_t d, int64_t V, int topk) {
    if (attt::lp_sizes(L, d, V) != ATTT_OK || topk < 0 || topk > attt::kLpTopMax || topk > V) return 0;
    return attt::lp_layout(nullptr, L, d, V, topk).bytes;
}

attt_status attt_logprob_forward(const attt_bf16 *d_h, int64_t h_ld, const attt_bf16 *d_W, const int32_t *d_tgt,
                                 int64_t L, int64_t d, int64_t V, float inv_temp, int topk, float *d_logp,
                                 float *d_entropy, float *d_lse, float *d_top_logp, int32_t *d_top_id, void *d_ws,
                                 size_t ws_bytes, attt_stream stream) {
    ATTT_NVTX_RANGE();
    using namespace attt;
    attt_status st = lp_check(d_h, h_ld, d_W, L, d, V, inv_temp);
    if (st != ATTT_OK) return st;
    if (topk < 0 || topk > kLpTopMax || topk > V || (d_tgt != nullptr) != (d_logp != nullptr) ||
        (topk > 0) != (d_top_logp != nullptr) || (topk > 0) != (d_top_id != nullptr))
        return ATTT_ERR_INVALID_ARG;
    if (!d_logp && !d_entropy && !d_lse && topk == 0) return ATTT_ERR_INVALID_ARG;
    if (!aligned_to(4, d_tgt, d_logp, d_entropy, d_lse, d_top_logp, d_top_id)) return ATTT_ERR_INVALID_ARG;
    if (!d_ws || !aligned256(d_ws) || ws_bytes < attt_logprob_workspace_bytes(L, d, V, topk))
        return ATTT_ERR_WORKSPACE;
    int dev;
    st = current_device(&dev);
    if (st != ATTT_OK) return st;
    int *status = device_status_word(dev);
    if (!status) return ATTT_ERR_CUDA;
    const LpLayout c = lp_layout(d_ws, L, d, V, topk);
    LpReduceArgs a{};
    a.part = c.part; a.ztgt = c.ztgt; a.top_v = c.top_v; a.top_i = c.top_i; a.plane = c.plane;
    a.rows = (int)L; a.V = (int)V; a.topk = topk; a.top_ld = (int)c.ld; a.inv_temp = inv_temp;
    a.tgt = d_tgt; a.logp = d_logp; a.entropy = d_entropy; a.lse = d_lse; a.top_logp = d_top_logp;
    a.top_id = d_top_id; a.status = status;
    if (L <= kFewRows) {
        FewArgs f{};
        f.L = (int)L; f.V = (int)V; f.topk = topk; f.c2 = inv_temp * kLog2e;
        f.tgt = d_tgt; f.ztgt = c.ztgt; f.part = c.part; f.top_v = c.top_v; f.top_i = c.top_i; f.status = status;
        if (topk > 0)
            return L <= 16 ? launch_few<true, 1>(d_h, h_ld, d_W, d, f, a, dev, stream)
                           : launch_few<true, 2>(d_h, h_ld, d_W, d, f, a, dev, stream);
        return L <= 16 ? launch_few<false, 1>(d_h, h_ld, d_W, d, f, a, dev, stream)
                       : launch_few<false, 2>(d_h, h_ld, d_W, d, f, a, dev, stream);
    }
    const int sms = num_sms(dev);
    const int64_t rows = lp_forward_rows(L, d);
    for (int64_t r0 = 0; r0 < L; r0 += rows) {
        const int64_t R = std::min(rows, L - r0);
        const TilePlan t = plan_tiles(R, V, cdiv(d, 64), sms, 0, false, false);
        GemmProblem p{};
        p.a = d_h + r0 * h_ld; p.a_rows_ld = h_ld; p.a_rows = R; p.a_k = d;
        p.b = d_W; p.b_rows_ld = d; p.b_rows = V; p.b_k = d;
        p.M = (int)R; p.N = (int)V; p.K = (int)d; p.BN = t.BN; p.pair = t.pair; p.tight = true;
        EpiParams ep{};
        ep.tgt = d_tgt ? d_tgt + r0 : nullptr; ep.ztgt = c.ztgt;
        ep.lp_part = c.part; ep.lp_plane = c.plane;
        ep.top_v = c.top_v; ep.top_i = c.top_i; ep.top_ld = (int)c.ld;
        ep.inv_temp = inv_temp;
        ep.lp_split = a.split = R > (t.pair ? 256 : 128) && 2 * d * V > kLpHeadBytes;
        a.rows = (int)R;
        a.sets = lp_sets(d);
        a.tile_rows = t.pair ? 256 : 128;
        a.tiles_n = (int)cdiv(V, t.BN);
        a.nwork = (int)cdiv(R, a.tile_rows) * a.tiles_n;
        a.units = std::min(a.nwork, t.pair ? sms / 2 : sms);  // as launch_gemm has it
        if (a.nwork > a.units * a.tiles_n) return ATTT_ERR_UNSUPPORTED;  // runs longer than a row (fewer SMs than 128)
        a.tgt = ep.tgt;
        a.logp = d_logp ? d_logp + r0 : nullptr;
        a.entropy = d_entropy ? d_entropy + r0 : nullptr;
        a.lse = d_lse ? d_lse + r0 : nullptr;
        if (topk > 0) {
            a.top_logp = d_top_logp + r0 * topk;
            a.top_id = d_top_id + r0 * topk;
        }
        st = topk == 0   ? launch_logits<EPI_LOGP>(p, ep, a.sets, dev, stream)
             : topk == 1 ? launch_logits<EPI_LOGP_TOP1>(p, ep, a.sets, dev, stream)
             : topk <= 8 ? launch_logits<EPI_LOGP_TOP8>(p, ep, a.sets, dev, stream)
                         : launch_logits<EPI_LOGP_TOP20>(p, ep, a.sets, dev, stream);
        if (st == ATTT_OK) st = topk > 0 ? launch_reduce<true>(a, stream) : launch_reduce<false>(a, stream);
        if (st != ATTT_OK) return st;
    }
    return ATTT_OK;
}

size_t attt_logprob_grad_workspace_bytes(int64_t L, int64_t d, int64_t V) {
    if (attt::lp_sizes(L, d, V) != ATTT_OK) return 0;
    return attt::grad_layout(nullptr, L, d, V).bytes;
}

attt_status attt_logprob_input_grad(const attt_bf16 *d_h, int64_t h_ld, const attt_bf16 *d_W, const int32_t *d_tgt,
                                    const float *d_lse, const float *d_entropy, const float *d_glogp,
                                    const float *d_gent, int64_t L, int64_t d, int64_t V, float inv_temp,
                                    attt_bf16 *d_dh, void *d_ws, size_t ws_bytes, attt_stream stream) {
    ATTT_NVTX_RANGE();
    using namespace attt;
    attt_status st = lp_check(d_h, h_ld, d_W, L, d, V, inv_temp);
    if (st != ATTT_OK) return st;
    if (!d_tgt || !d_lse || !d_glogp || (d_gent && !d_entropy) || !d_dh || !aligned16(d_dh)) return ATTT_ERR_INVALID_ARG;
    if (!aligned_to(4, d_tgt, d_lse, d_entropy, d_glogp, d_gent)) return ATTT_ERR_INVALID_ARG;
    if (!d_ws || !aligned256(d_ws) || ws_bytes < attt_logprob_grad_workspace_bytes(L, d, V)) return ATTT_ERR_WORKSPACE;
    int dev;
    st = current_device(&dev);
    if (st != ATTT_OK) return st;
    if (!device_status_word(dev)) return ATTT_ERR_CUDA;
    const GradLayout c = grad_layout(d_ws, L, d, V);
    const int sets = lp_sets(d);
    for (int64_t r0 = 0; r0 < L; r0 += c.rows) {
        const int64_t R = L - r0 < c.rows ? L - r0 : c.rows;
        const int64_t M = c.lo ? 2 * R : R;  // the sum of the pieces adds the two rows of each
        const TilePlan td = plan_tiles(M, d, c.ld / 64, num_sms(dev), c.regions, !c.lo, true);
        // whole tiles: the last wave's may be cut, with arrival counters that start at 0
        if (td.pieces == 1 && !c.lo &&
            cudaMemsetAsync(c.split_tick, 0, sizeof(unsigned int) * (size_t)c.regions, stream) != cudaSuccess)
            return ATTT_ERR_CUDA;
        {   // G from the logits
            const TilePlan t = plan_tiles(R, V, cdiv(d, 64), num_sms(dev), 0, false, false);
            GemmProblem p{};
            p.a = d_h + r0 * h_ld; p.a_rows_ld = h_ld; p.a_rows = R; p.a_k = d;
            p.b = d_W; p.b_rows_ld = d; p.b_rows = V; p.b_k = d;
            p.M = (int)R; p.N = (int)V; p.K = (int)d; p.BN = t.BN; p.pair = t.pair; p.tight = true;
            EpiParams ep{};
            ep.tgt = d_tgt + r0; ep.lse = d_lse + r0; ep.glogp = d_glogp + r0;
            ep.entropy = d_gent ? d_entropy + r0 : nullptr;
            ep.gent = d_gent ? d_gent + r0 : nullptr;
            ep.inv_temp = inv_temp; ep.V = (int)V;
            ep.G = c.G; ep.G_ld = c.ld;
            if (c.lo) ep.G_lo = c.G + R * c.ld;
            else ep.lp_loss = c.loss;
            st = launch_logits<EPI_LOGP_GRAD>(p, ep, sets, dev, stream);
            if (st != ATTT_OK) return st;
        }
        {   // dh = G W
            GemmProblem p{};
            p.a = c.G; p.a_rows_ld = c.ld; p.a_rows = M; p.a_k = c.ld;
            p.b = d_W; p.b_rows_ld = d; p.b_rows = d; p.b_k = V;
            p.M = (int)M; p.N = (int)d; p.K = (int)c.ld;
            p.fold = c.lo ? (int)R : 0;
            p.tight = true;
            p.pdl = true;
            p.split_ws = c.split_ws; p.split_tick = c.split_tick; p.split_regions = c.regions;
            EpiParams ep{};
            ep.out16 = reinterpret_cast<__nv_bfloat16 *>(d_dh) + r0 * d; ep.out_ld = d; ep.alpha = 1.0f;
            if (!c.lo) {
                ep.row_gamma = c.loss; ep.fix_tgt = d_tgt + r0;
                ep.fix_W = reinterpret_cast<const __nv_bfloat16 *>(d_W); ep.fix_ld = d; ep.fix_V = (int)V;
            }
            st = launch_planned<true, false, true>(p, ep, td, dev, stream);
            if (st != ATTT_OK) return st;
        }
    }
    return ATTT_OK;
}

}  // extern "C"

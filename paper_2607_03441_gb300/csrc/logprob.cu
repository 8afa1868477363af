// logprob.cu -- log probabilities of given tokens through the frozen LM head,
// with the entropy of every row's distribution and its most probable
// alternatives, and their gradient with respect to the hidden states; the
// [L, V] logits never reach HBM.
//
// With z = h W^T, T the temperature, p = softmax(z / T):
//   logp_j = z_{j,t_j} / T - lse_j,   lse_j = log sum_v exp(z_jv / T),
//   H_j = -sum_v p_jv log p_jv.
// Forward: one contraction over the whole vocabulary (2 L V d FLOPs).  Its epilogue
// reduces each row of a column set (a tile, or half of one) to its max, the sum
// of exponentials, that sum's first moment, and its few largest logits
// (tc_gemm.cuh, EPI_LOGP*); a second kernel merges a row's sets.
// Gradient: with given da_j = dL/dlogp_j and db_j = dL/dH_j,
//   dL/dz_jv = (da_j [v = t_j] - p_jv (da_j + db_j (log p_jv + H_j))) / T,
// formed from the logits in the epilogue of the same contraction (the
// softmax needs no second sweep: lse and H are the forward call's) as a bf16 block
// G, then dh = G W (4 L V d FLOPs: the logits are formed again).
// Rows are taken in blocks so that the workspace stays bounded.
// Bound: the tensor core from a few hundred rows on, the head's bytes below.
#include <algorithm>

#include "gemm_launch.cuh"

namespace attt {

constexpr int kLpTopMax = 20;
constexpr int kLpWarps = 16;
constexpr int kLpRows = 8;  // rows per reduction block: lane & 7
constexpr int kLpStreams = kLpWarps * 32 / kLpRows;
// Bounds of the forward workspace (largest logits of every column set and row) and
// of the gradient block, in bytes per row block.
constexpr int64_t kLpTopBytes = 512ll << 20;
constexpr int64_t kLpNarrowBytes = 64ll << 20;  // what narrower sets than a 256-column tile's may take
constexpr int64_t kLpGBytes = 2048ll << 20;
constexpr int kFewRows = 32;   // rows of a call that reads the head as the M operand, at most
constexpr int kFewSets = 160;  // and its CTAs
constexpr int kLpSplitRegions = 320;  // K pieces of the second contraction: 128 KB each

inline int lp_sets(int64_t d) { return cdiv(d, 64) <= kTwoSetBlocks ? 2 : 1; }
inline int64_t lp_top_ld(int topk) { return round_up(topk, 4); }
inline int64_t lp_set_bytes(int topk) { return 12 + 8 * lp_top_ld(topk); }  // of one row

// Rows of a block of `total` rows at `row_bytes` of workspace each: equal blocks, a
// multiple of 256.
inline int64_t lp_block_rows(int64_t total, int64_t row_bytes, int64_t bound) {
    int64_t most = bound / row_bytes / 256 * 256;
    if (most < 256) most = 256;
    if (total <= most) return total;
    return round_up(cdiv(total, cdiv(total, most)), 256);
}

struct LpLayout {
    int64_t rows, plane, ld;  // rows per block; elements of a plane [sets, rows]
    bool few;
    float *part, *ztgt, *top_v;
    int32_t *top_i;
    size_t bytes;
};

static LpLayout lp_layout(void *ws, int64_t L, int64_t d, int64_t V, int topk) {
    LpLayout c{};
    if (L <= kFewRows) {  // one set per CTA, 32 alternatives
        c.few = true;
        c.rows = L;
        c.ld = 32;
        c.plane = kFewSets * L;
        Carve cv{static_cast<char *>(ws), 0};
        c.part = cv.take<float>((size_t)(3 * c.plane));
        c.ztgt = cv.take<float>((size_t)L);
        c.top_v = cv.take<float>((size_t)(topk > 0 ? c.plane * c.ld : 0));
        c.top_i = cv.take<int32_t>((size_t)(topk > 0 ? c.plane * c.ld : 0));
        c.bytes = (size_t)round_up((int64_t)cv.used, 256);
        return c;
    }
    const int64_t wide = cdiv(V, 256) * lp_sets(d), per = lp_set_bytes(topk);
    c.rows = lp_block_rows(L, wide * per, kLpTopBytes);
    c.ld = lp_top_ld(topk);
    const int64_t narrow = cdiv(V, 64) * lp_sets(d) * c.rows, most = kLpNarrowBytes / per;
    c.plane = narrow < most ? narrow : most;
    if (c.plane < wide * c.rows) c.plane = wide * c.rows;
    Carve cv{static_cast<char *>(ws), 0};
    c.part = cv.take<float>((size_t)(3 * c.plane));
    c.ztgt = cv.take<float>((size_t)c.rows);
    c.top_v = cv.take<float>((size_t)(c.plane * c.ld));
    c.top_i = cv.take<int32_t>((size_t)(c.plane * c.ld));
    c.bytes = (size_t)round_up((int64_t)cv.used, 256);
    return c;
}

// (max, sum, moment) of some of a row's sets, as epilogue_logp forms them.  While
// the max is -inf the sum means nothing but that it may be NaN.
struct LpPart {
    float m, s, t;
    __device__ __forceinline__ void merge(const LpPart &o, float c2) {
        const float M = fmaxf(m, o.m);
        if (M == -INFINITY) {
            s += o.s;
            t += o.t;
            return;
        }
        const float a = (m - M) * c2, b = (o.m - M) * c2, fa = ex2(a), fb = ex2(b);
        t = fa * fmaf(s, fmaxf(a, -1e4f), t) + fb * fmaf(o.s, fmaxf(b, -1e4f), o.t);
        s = fa * s + fb * o.s;
        m = M;
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
    int nsets, rows, V, topk, top_ld;
    float inv_temp;
    const int32_t *tgt;  // outputs and tgt from the block's first row
    float *logp, *entropy, *lse, *top_logp;
    int32_t *top_id;
    int *status;
};

// A row's lse, entropy and log probability of its given token, from its (max, sum,
// moment) and ln = log(sum).
__device__ __forceinline__ void lp_row(const LpReduceArgs &a, int j, const LpPart &p, float ln) {
    if (a.lse) a.lse[j] = fmaf(p.m, a.inv_temp, ln);
    if (a.entropy) a.entropy[j] = ln - 0.69314718055994531f * (p.t / p.s);
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

// Merges the sets of 8 rows (lane & 7): 64 streams read every 64th set, four sets'
// loads in flight, then shuffles and shared memory, in a fixed order.  K > 0: every
// stream also keeps its K largest logits; their lists meet in shared memory, where
// one warp per row takes the best head of its 64 lists `topk` times, the lowest id
// among equal ones.
template <int K>
__global__ void __launch_bounds__(kLpWarps * 32) logprob_reduce_kernel(const LpReduceArgs a) {
    extern __shared__ float s_dyn[];
    __shared__ LpPart s_part[kLpWarps][kLpRows];
    __shared__ float s_max[kLpRows], s_ln[kLpRows];
    griddep_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rl = lane & (kLpRows - 1), sub = lane / kLpRows;
    const int j = blockIdx.x * kLpRows + rl;
    const int stream = warp * (32 / kLpRows) + sub;
    const float c2 = a.inv_temp * kLog2e;
    LpPart acc{-INFINITY, 0.f, 0.f};
    if (j < a.rows) {
        for (int t0 = stream; t0 < a.nsets; t0 += 4 * kLpStreams) {
            LpPart v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int t = t0 + k * kLpStreams;
                const int64_t o = (int64_t)t * a.rows + j;
                v[k] = t < a.nsets ? LpPart{__ldcg(a.part + o), __ldcg(a.part + a.plane + o),
                                            __ldcg(a.part + 2 * a.plane + o)}
                                   : LpPart{-INFINITY, 0.f, 0.f};
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) acc.merge(v[k], c2);
        }
    }
    for (int o = kLpRows; o < 32; o <<= 1) acc.merge(acc.shfl_xor(o), c2);
    if (sub == 0) s_part[warp][rl] = acc;
    if constexpr (K > 0) {
        TopList<K> top;
        top.clear();
        if (j < a.rows) {
            for (int t = stream; t < a.nsets; t += kLpStreams) {
                const int64_t o = ((int64_t)t * a.rows + j) * a.top_ld;
                float v[K];
#pragma unroll
                for (int q = 0; q < K; q += 4) {
                    const float4 f = q < a.top_ld ? __ldcg(reinterpret_cast<const float4 *>(a.top_v + o + q))
                                                  : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
                    v[q] = f.x; v[q + 1] = f.y; v[q + 2] = f.z; v[q + 3] = f.w;
                }
                if (v[0] > top.least()) {  // a stream's sets and a set's list come in order: ties keep the lower id
#pragma unroll
                    for (int q = 0; q < K; ++q)
                        if (v[q] > top.least()) top.insert(v[q], __ldcg(a.top_i + o + q));
                }
            }
        }
        float *sv = s_dyn;
        int *si = reinterpret_cast<int *>(s_dyn + kLpRows * kLpStreams * K);
#pragma unroll
        for (int q = 0; q < K; ++q) {
            sv[(rl * kLpStreams + stream) * K + q] = top.v[q];
            si[(rl * kLpStreams + stream) * K + q] = top.id[q];
        }
    }
    __syncthreads();
    if (warp == 0) {
        acc = LpPart{-INFINITY, 0.f, 0.f};
        for (int w = sub; w < kLpWarps; w += 32 / kLpRows) acc.merge(s_part[w][rl], c2);
        for (int o = kLpRows; o < 32; o <<= 1) acc.merge(acc.shfl_xor(o), c2);
        if (j < a.rows && sub == 0) {
            const float ln = logf(acc.s);
            s_max[rl] = acc.m;
            s_ln[rl] = ln;
            lp_row(a, j, acc, ln);
        }
    }
    if constexpr (K > 0) {
        __syncthreads();
        const int jr = blockIdx.x * kLpRows + warp;
        if (warp >= kLpRows || jr >= a.rows) return;
        const float *sv = s_dyn + warp * kLpStreams * K;
        const int *si = reinterpret_cast<const int *>(s_dyn + kLpRows * kLpStreams * K) + warp * kLpStreams * K;
        int h0 = 0, h1 = 0;  // heads of this lane's lists, lane and lane + 32
        for (int q = 0; q < a.topk; ++q) {
            float v = h0 < K ? sv[lane * K + h0] : -INFINITY;
            int id = h0 < K ? si[lane * K + h0] : -1;
            const float v1 = h1 < K ? sv[(lane + 32) * K + h1] : -INFINITY;
            const int id1 = h1 < K ? si[(lane + 32) * K + h1] : -1;
            const bool second = v1 > v || (v1 == v && (unsigned)id1 < (unsigned)id);  // -1: after every id
            if (second) {
                v = v1;
                id = id1;
            }
            float bv = v;
            unsigned bi = (unsigned)id;
            for (int o = 16; o > 0; o >>= 1) {
                const float ov = __shfl_xor_sync(0xffffffffu, bv, o);
                const unsigned oi = __shfl_xor_sync(0xffffffffu, bi, o);
                if (ov > bv || (ov == bv && oi < bi)) {
                    bv = ov;
                    bi = oi;
                }
            }
            if (bi == (unsigned)id && id >= 0) {
                if (second) ++h1;
                else ++h0;
            }
            if (lane == 0) {
                a.top_logp[(int64_t)jr * a.topk + q] = (bv - s_max[warp]) * a.inv_temp - s_ln[warp];
                a.top_id[(int64_t)jr * a.topk + q] = (int)bi;
            }
        }
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
// Through 152,064 x 3,584 with 5 alternatives one row takes 167 us (96% of the copy
// bandwidth; 228 with the row padded to 128 and the alternatives kept by its one lane),
// 16 rows through 152,064 x 5,120 with 20 take 255 (90%; 307).
// ---------------------------------------------------------------------------

constexpr int kFewMaxStages = 10;

// Whether logit a of id i comes before b of j: larger, or equal and of a lower id (ids
// as unsigned: -1, an empty place, comes last).
__device__ __forceinline__ bool lp_before(float a, int i, float b, int j) {
    return a > b || (a == b && (unsigned)i < (unsigned)j);
}

// One compare-exchange of a warp-wide sort: the lane keeps the earlier of its own and
// its partner's (lane ^ o) where `first`, else the later.
__device__ __forceinline__ void lp_exchange(float &v, int &id, int o, bool first) {
    const float ov = __shfl_xor_sync(0xffffffffu, v, o);
    const int oi = __shfl_xor_sync(0xffffffffu, id, o);
    if (lp_before(ov, oi, v, id) == first) {
        v = ov;
        id = oi;
    }
}

// Sorts the warp's 32 values, lane 0 the first.
__device__ __forceinline__ void lp_sort(float &v, int &id, int lane) {
#pragma unroll
    for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
        for (int o = k >> 1; o > 0; o >>= 1) lp_exchange(v, id, o, ((lane & o) == 0) == ((lane & k) == 0));
}

// (v, id): the first 32 of two sorted lists.
__device__ __forceinline__ void lp_merge(float &v, int &id, float ov, int oi, int lane) {
    ov = __shfl_xor_sync(0xffffffffu, ov, 31);
    oi = __shfl_xor_sync(0xffffffffu, oi, 31);
    if (lp_before(ov, oi, v, id)) {
        v = ov;
        id = oi;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) lp_exchange(v, id, o, (lane & o) == 0);
}

// A tile's 32 logits (-inf or NaN: none) into the list, of which the first k count.
__device__ __forceinline__ void lp_offer(float &lv, int &li, float v, int id, int k, int lane) {
    unsigned mask = __ballot_sync(0xffffffffu, v > __shfl_sync(0xffffffffu, lv, k - 1));
    if (__popc(mask) > 2) {
        float nv = v > -INFINITY ? v : -INFINITY;  // NaN: none
        int ni = v > -INFINITY ? id : -1;
        lp_sort(nv, ni, lane);
        lp_merge(lv, li, nv, ni, lane);
        return;
    }
    while (mask) {  // ids come in order, so that equal ones already there stay before
        const int from = __ffs(mask) - 1;
        mask &= mask - 1;
        const float nv = __shfl_sync(0xffffffffu, v, from);
        const int ni = __shfl_sync(0xffffffffu, id, from);
        const int at = __popc(__ballot_sync(0xffffffffu, lv >= nv));
        const float uv = __shfl_up_sync(0xffffffffu, lv, 1);
        const int ui = __shfl_up_sync(0xffffffffu, li, 1);
        if (lane > at) {
            lv = uv;
            li = ui;
        }
        if (lane == at) {
            lv = nv;
            li = ni;
        }
    }
}

struct FewArgs {
    int L, V, kb, stages, tiles, topk;
    float c2;  // log2 e / T
    const int32_t *tgt;
    float *ztgt;
    float *part;   // [CTAs][L] max, then sum, then moment, kFewSets * L apart
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
        float lv[TOP ? 16 : 1];
        int li[TOP ? 16 : 1];
#pragma unroll
        for (int t = 0; t < 16; ++t) {
            st[t] = LpPart{-INFINITY, 0.f, 0.f};
            if constexpr (TOP) {
                lv[t] = -INFINITY;
                li[t] = -1;
            }
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
            for (int t = 0; t < 16; ++t) {
                if (t >= rows) break;  // warp-uniform
                const float z = id < a.V ? v[t] : -INFINITY;
                if (__shfl_sync(0xffffffffu, given, t) == id && id < a.V) a.ztgt[row0 + t] = z;
                // the lane's running max moves to z, or z counts against it; -inf adds nothing, NaN
                // reaches the sum
                if (z != -INFINITY) {
                    const bool above = z > st[t].m;
                    const float d = (above ? st[t].m - z : z - st[t].m) * a.c2, e = ex2(d), dm = fmaxf(d, -1e4f);
                    if (above) {
                        st[t].t = e * fmaf(st[t].s, dm, st[t].t);
                        st[t].s = fmaf(st[t].s, e, 1.f);
                        st[t].m = z;
                    } else {
                        st[t].t = fmaf(e, dm, st[t].t);
                        st[t].s += e;
                    }
                }
                __syncwarp();
                if constexpr (TOP) lp_offer(lv[t], li[t], z, id, a.topk, lane);
            }
        }
        // the four warps of a set through shared memory: every MMA has completed, and with it
        // every load into the ring
        float *sp = reinterpret_cast<float *>(smem) + set * 16 * 4 * 3;
        float *sv = reinterpret_cast<float *>(smem) + SETS * 16 * 4 * 3 + set * 16 * 4 * 64;
#pragma unroll
        for (int t = 0; t < 16; ++t) {
            if (t >= rows) break;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) st[t].merge(st[t].shfl_xor(o), a.c2);
            if (lane == 0) {
                sp[(t * 4 + q) * 3] = st[t].m;
                sp[(t * 4 + q) * 3 + 1] = st[t].s;
                sp[(t * 4 + q) * 3 + 2] = st[t].t;
            }
            if constexpr (TOP) {
                sv[(t * 4 + q) * 64 + lane] = lv[t];
                reinterpret_cast<int *>(sv)[(t * 4 + q) * 64 + 32 + lane] = li[t];
            }
        }
        named_barrier_sync(1u + set, 128);
        const int64_t plane = (int64_t)kFewSets * a.L;
        for (int t = q; t < rows; t += 4) {
            const int64_t o = (int64_t)blockIdx.x * a.L + row0 + t;
            if (lane == 0) {
                LpPart p{-INFINITY, 0.f, 0.f};
                for (int k = 0; k < 4; ++k)
                    p.merge(LpPart{sp[(t * 4 + k) * 3], sp[(t * 4 + k) * 3 + 1], sp[(t * 4 + k) * 3 + 2]}, a.c2);
                a.part[o] = p.m;
                a.part[plane + o] = p.s;
                a.part[2 * plane + o] = p.t;
            }
            if constexpr (TOP) {
                float x = sv[t * 4 * 64 + lane];
                int i = reinterpret_cast<int *>(sv)[t * 4 * 64 + 32 + lane];
                for (int k = 1; k < 4; ++k)
                    lp_merge(x, i, sv[(t * 4 + k) * 64 + lane], reinterpret_cast<int *>(sv)[(t * 4 + k) * 64 + 32 + lane],
                             lane);
                a.top_v[o * 32 + lane] = x;
                a.top_i[o * 32 + lane] = i;
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_dealloc(tmem_base, kCols);
}

// The CTAs' results of row blockIdx.x: warps take every kLpWarps-th, all of a warp's loads
// on their way at once, then warp 0 takes the warps'.
template <bool TOP>
__global__ void __launch_bounds__(kLpWarps * 32)
    logprob_few_reduce_kernel(const LpReduceArgs a) {
    __shared__ LpPart s_part[kLpWarps];
    __shared__ float s_v[kLpWarps][32];
    __shared__ int s_i[kLpWarps][32];
    constexpr int kEach = kFewSets / kLpWarps;
    griddep_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, j = blockIdx.x;
    const float c2 = a.inv_temp * kLog2e;
    LpPart p{-INFINITY, 0.f, 0.f};
    {
        const int t = warp + lane * kLpWarps;  // one set per lane
        const int64_t o = (int64_t)t * a.rows + j;
        if (lane < kEach && t < a.nsets)
            p = LpPart{__ldcg(a.part + o), __ldcg(a.part + a.plane + o), __ldcg(a.part + 2 * a.plane + o)};
    }
    float v = -INFINITY;
    int id = -1;
    if constexpr (TOP) {
        float nv[kEach];
        int ni[kEach];
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int t = warp + k * kLpWarps;
            const int64_t o = ((int64_t)t * a.rows + j) * 32 + lane;
            nv[k] = t < a.nsets ? __ldcg(a.top_v + o) : -INFINITY;
            ni[k] = t < a.nsets ? __ldcg(a.top_i + o) : -1;
        }
#pragma unroll
        for (int k = 0; k < kEach; ++k) lp_merge(v, id, nv[k], ni[k], lane);
        s_v[warp][lane] = v;
        s_i[warp][lane] = id;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) p.merge(p.shfl_xor(o), c2);
    if (lane == 0) s_part[warp] = p;
    __syncthreads();
    if (warp > 0) return;
    p = lane < kLpWarps ? s_part[lane] : LpPart{-INFINITY, 0.f, 0.f};
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) p.merge(p.shfl_xor(o), c2);
    const float ln = logf(p.s);
    if (lane == 0) lp_row(a, j, p, ln);
    if constexpr (TOP) {
        for (int k = 1; k < kLpWarps; ++k) lp_merge(v, id, s_v[k][lane], s_i[k][lane], lane);
        if (lane < a.topk) {
            a.top_logp[(int64_t)j * a.topk + lane] = (v - p.m) * a.inv_temp - ln;
            a.top_id[(int64_t)j * a.topk + lane] = id;
        }
    }
}

template <int K>
static attt_status launch_reduce(const LpReduceArgs &a, int dev, cudaStream_t stream) {
    auto kern = logprob_reduce_kernel<K>;
    const size_t smem = (size_t)8 * kLpRows * kLpStreams * K;
    if (smem > 0 && !set_smem_limit(reinterpret_cast<const void *>(kern), smem, dev)) return ATTT_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)cdiv(a.rows, kLpRows));
    cfg.blockDim = dim3(kLpWarps * 32);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kern, a) != cudaSuccess) return ATTT_ERR_CUDA;
    count_launch();
    return cudaGetLastError() == cudaSuccess ? ATTT_OK : ATTT_ERR_CUDA;
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
    const int ctas = std::min({f.tiles, num_sms(dev), kFewSets});
    kern<<<ctas, few_threads(SETS), smem, stream>>>(tw, th, f);
    count_launch();
    if (cudaGetLastError() != cudaSuccess) return ATTT_ERR_CUDA;
    a.nsets = ctas;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)f.L);
    cfg.blockDim = dim3(kLpWarps * 32);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, logprob_few_reduce_kernel<TOP>, a) != cudaSuccess) return ATTT_ERR_CUDA;
    count_launch();
    return cudaGetLastError() == cudaSuccess ? ATTT_OK : ATTT_ERR_CUDA;
}

template <int EPI>
static attt_status launch_logits(const GemmProblem &p, const EpiParams &ep, int sets, int dev, cudaStream_t stream) {
    return sets == 2 ? launch_gemm<EPI, false, false, 2>(p, ep, dev, stream)
                     : launch_gemm<EPI, false, false, 1>(p, ep, dev, stream);
}

struct GradLayout {
    int64_t rows, ld;
    int regions;
    __nv_bfloat16 *G;
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
    Carve cv{static_cast<char *>(ws), 0};
    c.G = cv.take<__nv_bfloat16>((size_t)(c.rows * c.ld));
    c.split_ws = cv.take<float>((size_t)c.regions * 128 * 256);
    c.split_tick = cv.take<unsigned int>((size_t)c.regions);
    c.bytes = (size_t)round_up((int64_t)cv.used, 256);
    return c;
}

// What both calls ask of their operands.
static attt_status lp_check(const attt_bf16 *d_h, int64_t h_ld, const attt_bf16 *d_W, int64_t L, int64_t d, int64_t V,
                            float inv_temp) {
    if (!d_h || !d_W || L < 1 || V < 1 || d < 8 || d % 8 != 0 || h_ld < d || h_ld % 8 != 0) return ATTT_ERR_INVALID_ARG;
    if (!(inv_temp > 0.f) || !(inv_temp <= 1e4f)) return ATTT_ERR_INVALID_ARG;
    if (L > (1ll << 30) || V > (1ll << 30) || d > (1ll << 20) || h_ld > (1ll << 36)) return ATTT_ERR_UNSUPPORTED;
    if (!aligned16(d_h) || !aligned16(d_W)) return ATTT_ERR_INVALID_ARG;
    return ATTT_OK;
}

}  // namespace attt

extern "C" {

size_t attt_logprob_workspace_bytes(int64_t L, int64_t d, int64_t V, int topk) {
    if (L < 1 || V < 1 || d < 1 || topk < 0 || topk > attt::kLpTopMax) return 0;
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
    if (!d_ws || !aligned256(d_ws) || ws_bytes < attt_logprob_workspace_bytes(L, d, V, topk))
        return ATTT_ERR_WORKSPACE;
    int dev;
    st = current_device(&dev);
    if (st != ATTT_OK) return st;
    int *status = device_status_word(dev);
    if (!status) return ATTT_ERR_CUDA;
    const LpLayout c = lp_layout(d_ws, L, d, V, topk);
    if (c.few) {
        FewArgs f{};
        f.L = (int)L; f.V = (int)V; f.topk = topk; f.c2 = inv_temp * kLog2e;
        f.tgt = d_tgt; f.ztgt = c.ztgt; f.part = c.part; f.top_v = c.top_v; f.top_i = c.top_i; f.status = status;
        LpReduceArgs a{};
        a.part = c.part; a.ztgt = c.ztgt; a.top_v = c.top_v; a.top_i = c.top_i; a.plane = c.plane;
        a.rows = (int)L; a.V = (int)V; a.topk = topk; a.top_ld = (int)c.ld; a.inv_temp = inv_temp;
        a.tgt = d_tgt; a.logp = d_logp; a.entropy = d_entropy; a.lse = d_lse; a.top_logp = d_top_logp;
        a.top_id = d_top_id; a.status = status;
        if (topk > 0)
            return L <= 16 ? launch_few<true, 1>(d_h, h_ld, d_W, d, f, a, dev, stream)
                           : launch_few<true, 2>(d_h, h_ld, d_W, d, f, a, dev, stream);
        return L <= 16 ? launch_few<false, 1>(d_h, h_ld, d_W, d, f, a, dev, stream)
                       : launch_few<false, 2>(d_h, h_ld, d_W, d, f, a, dev, stream);
    }
    const int sets = lp_sets(d);
    for (int64_t r0 = 0; r0 < L; r0 += c.rows) {
        const int64_t R = L - r0 < c.rows ? L - r0 : c.rows;
        TilePlan t = plan_tiles(R, V, cdiv(d, 64), num_sms(dev), 0, false, false);
        while (t.BN < 256 && cdiv(V, t.BN) * sets * R > c.plane) t.BN += 64;
        GemmProblem p{};
        p.a = d_h + r0 * h_ld; p.a_rows_ld = h_ld; p.a_rows = R; p.a_k = d;
        p.b = d_W; p.b_rows_ld = d; p.b_rows = V; p.b_k = d;
        p.M = (int)R; p.N = (int)V; p.K = (int)d; p.BN = t.BN; p.pair = t.pair;
        EpiParams ep{};
        ep.tgt = d_tgt ? d_tgt + r0 : nullptr; ep.ztgt = c.ztgt;
        ep.lp_part = c.part; ep.lp_plane = c.plane;
        ep.top_v = c.top_v; ep.top_i = c.top_i; ep.top_ld = (int)c.ld;
        ep.inv_temp = inv_temp;
        st = topk == 0  ? launch_logits<EPI_LOGP>(p, ep, sets, dev, stream)
             : topk <= 8 ? launch_logits<EPI_LOGP_TOP8>(p, ep, sets, dev, stream)
                         : launch_logits<EPI_LOGP_TOP20>(p, ep, sets, dev, stream);
        if (st != ATTT_OK) return st;
        LpReduceArgs a{};
        a.part = c.part; a.ztgt = c.ztgt; a.top_v = c.top_v; a.top_i = c.top_i; a.plane = c.plane;
        a.nsets = (int)cdiv(V, t.BN / sets); a.rows = (int)R; a.V = (int)V; a.topk = topk; a.top_ld = (int)c.ld;
        a.inv_temp = inv_temp;
        a.tgt = ep.tgt;
        a.logp = d_logp ? d_logp + r0 : nullptr;
        a.entropy = d_entropy ? d_entropy + r0 : nullptr;
        a.lse = d_lse ? d_lse + r0 : nullptr;
        if (topk > 0) {
            a.top_logp = d_top_logp + r0 * topk;
            a.top_id = d_top_id + r0 * topk;
        }
        a.status = status;
        st = topk == 0  ? launch_reduce<0>(a, dev, stream)
             : topk <= 8 ? launch_reduce<8>(a, dev, stream)
                         : launch_reduce<20>(a, dev, stream);
        if (st != ATTT_OK) return st;
    }
    return ATTT_OK;
}

size_t attt_logprob_grad_workspace_bytes(int64_t L, int64_t d, int64_t V) {
    if (L < 1 || V < 1 || d < 1) return 0;
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
    if (!d_ws || !aligned256(d_ws) || ws_bytes < attt_logprob_grad_workspace_bytes(L, d, V)) return ATTT_ERR_WORKSPACE;
    int dev;
    st = current_device(&dev);
    if (st != ATTT_OK) return st;
    if (!device_status_word(dev)) return ATTT_ERR_CUDA;
    const GradLayout c = grad_layout(d_ws, L, d, V);
    const int sets = lp_sets(d);
    for (int64_t r0 = 0; r0 < L; r0 += c.rows) {
        const int64_t R = L - r0 < c.rows ? L - r0 : c.rows;
        const TilePlan td = plan_tiles(R, d, c.ld / 64, num_sms(dev), c.regions, true, true);
        // whole tiles: the last wave's may be cut, with arrival counters that start at 0
        if (td.pieces == 1 &&
            cudaMemsetAsync(c.split_tick, 0, sizeof(unsigned int) * (size_t)c.regions, stream) != cudaSuccess)
            return ATTT_ERR_CUDA;
        {   // G from the logits
            const TilePlan t = plan_tiles(R, V, cdiv(d, 64), num_sms(dev), 0, false, false);
            GemmProblem p{};
            p.a = d_h + r0 * h_ld; p.a_rows_ld = h_ld; p.a_rows = R; p.a_k = d;
            p.b = d_W; p.b_rows_ld = d; p.b_rows = V; p.b_k = d;
            p.M = (int)R; p.N = (int)V; p.K = (int)d; p.BN = t.BN; p.pair = t.pair;
            EpiParams ep{};
            ep.tgt = d_tgt + r0; ep.lse = d_lse + r0; ep.glogp = d_glogp + r0;
            ep.entropy = d_gent ? d_entropy + r0 : nullptr;
            ep.gent = d_gent ? d_gent + r0 : nullptr;
            ep.inv_temp = inv_temp; ep.V = (int)V;
            ep.G = c.G; ep.G_ld = c.ld;
            st = launch_logits<EPI_LOGP_GRAD>(p, ep, sets, dev, stream);
            if (st != ATTT_OK) return st;
        }
        {   // dh = G W
            GemmProblem p{};
            p.a = c.G; p.a_rows_ld = c.ld; p.a_rows = R; p.a_k = c.ld;
            p.b = d_W; p.b_rows_ld = d; p.b_rows = d; p.b_k = V;
            p.M = (int)R; p.N = (int)d; p.K = (int)c.ld;
            p.pdl = true;
            p.split_ws = c.split_ws; p.split_tick = c.split_tick; p.split_regions = c.regions;
            EpiParams ep{};
            ep.out16 = reinterpret_cast<__nv_bfloat16 *>(d_dh) + r0 * d; ep.out_ld = d; ep.alpha = 1.0f;
            st = launch_planned<true, false, true>(p, ep, td, dev, stream);
            if (st != ATTT_OK) return st;
        }
    }
    return ATTT_OK;
}

}  // extern "C"

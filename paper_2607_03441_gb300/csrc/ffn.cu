// ffn.cu -- the gated feed-forward block with an adapter on each of its three
// projections, forward and input gradient (kernels: tc_ffn.cuh).
//
//   g = x Wg + s (x Ag) Bg,  u = x Wu + s (x Au) Bu,  h = act(g) u,  y = h Wd + s (h Ad) Bd
//   dh = dy Wd^T + s (dy Bd^T) Ad^T,  dg = dh u act'(g),  du = dh act(g)
//   dx = dg Wg^T + s (dg Bg^T) Ag^T + du Wu^T + s (du Bu^T) Au^T
//
// Bound: tensor cores (6 L d f FLOPs either way) from some 300 rows on, below that the
// weights' bytes (6 d f).  Three contractions of a third of the work each way:
//   forward   [x | s x A] [W ; B] over gate and up columns side by side, whose epilogue
//             multiplies the factors: x is read once for both, g and u reach memory
//             only where the gradient will want them; then h Wd (tc_gemm.cuh);
//   backward  dy Wd^T, whose epilogue turns dh into dg and du without dh in memory; then
//             dg Wg^T + du Wu^T as one contraction over both K ranges.
// Adapters add a 64-deep K block or two, after a launch that forms the rank-r products.  A few rows take two
// launches that form them too (tc_ffn_few.cuh; which calls: ffn_few).
// Measured, 3,584 x 18,944, r 16: 2,048 rows forward 531 to 545 us (1,571 TFLOP/s; burst rate of a library's
// product 1,928, sustained 1,735); 8,192 rows at 5,120 x 27,648, r 64 backward 4,330 to 4,580 (1,540 to 1,630); 403
// rows at 4,096 x 14,336, r 32 forward 140 (512 rows of tiles, the products' launches 20); 1 row
// forward 69 (5.9 TB/s), 93 backward 97 (4.2 TB/s).
#include <algorithm>

#include "attt_host.h"
#include "tc_ffn.cuh"
#include "tc_ffn_few.cuh"

namespace attt {

// Partials of a contraction's K pieces, in 128 x 256 fp32 blocks.
constexpr int kFfnRegions = 160;

struct FfnLayout {
    int rpad, r8;
    __nv_bfloat16 *s2, *s1;   // [L, 2 rpad] (gate, up), [L, rpad] (down): rank-r products
    __nv_bfloat16 *pad[3];    // adapters' A with rows of r8, where r is not a multiple of 8
    float *split_ws;
    size_t bytes;
};

static FfnLayout ffn_layout(void *ws, int64_t L, int64_t d, int64_t f, int r) {
    FfnLayout c{};
    c.rpad = (int)round_up(r, 16);
    c.r8 = (int)round_up(r, 8);
    Carve cv{static_cast<char *>(ws), 0};
    c.s2 = cv.take<__nv_bfloat16>((size_t)L * 2 * c.rpad);
    c.s1 = cv.take<__nv_bfloat16>((size_t)L * c.rpad);
    for (int i = 0; i < 3; ++i) c.pad[i] = cv.take<__nv_bfloat16>(r % 8 ? (size_t)(i < 2 ? d : f) * c.r8 : 0);
    c.split_ws = cv.take<float>((size_t)kFfnRegions * 128 * 256);
    c.bytes = (size_t)round_up((int64_t)cv.used, 256);
    return c;
}

static attt_status ffn_sizes(int64_t L, int64_t d, int64_t f, int r) {
    if (L < 0 || d < 8 || f < 8 || d % 8 != 0 || f % 8 != 0 || r < 0 || r > 64) return ATTT_ERR_INVALID_ARG;
    if (L > (1ll << 30) || d > (1ll << 24) || f > (1ll << 24)) return ATTT_ERR_UNSUPPORTED;
    // tiles are counted in 32 bits
    if (cdiv(L, 128) * cdiv(std::max(d, f), 64) * kMaxPieces >= (1ll << 31)) return ATTT_ERR_UNSUPPORTED;
    return ATTT_OK;
}

// ---------------------------------------------------------------------------
// Small kernels
// ---------------------------------------------------------------------------

// A [n, r] with rows of r8 (zeros past r), for TMA, which reads rows of whole 16 bytes.
struct FfnPad {
    const __nv_bfloat16 *src[3];
    __nv_bfloat16 *dst[3];
    int64_t n[3];
    int r, r8;
};

__global__ void __launch_bounds__(256) ffn_pad_kernel(const FfnPad a) {
    griddep_launch_dependents();
    const int k = blockIdx.y;
    const __nv_bfloat16 *src = a.src[k];
    __nv_bfloat16 *dst = a.dst[k];
    if (!src) return;
    const int64_t total = a.n[k] * a.r8;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / a.r8;
        const int c = (int)(i - row * a.r8);
        dst[i] = c < a.r ? src[row * a.r + c] : __float2bfloat16_rn(0.f);
    }
}

// What an FFN_PART launch leaves, summed in piece order and finished as the whole tiles'
// epilogues do, four columns of a row per thread.
struct FfnReduce {
    const float *part;
    int M, N, BN, n_tile, pieces, rows, tiles_m, act;
    const __nv_bfloat16 *gate, *up;     // backward: the factors (out0 and out1 may be they)
    __nv_bfloat16 *out0, *out1, *out2;  // forward: h, g, u (g and u or neither); backward: dg, du
};

__device__ __forceinline__ float4 ffn_pieces(const FfnReduce &a, int64_t y, int col) {
    const float4 *src = reinterpret_cast<const float4 *>(a.part + y * a.BN + col);
    const int64_t step = (int64_t)a.rows * a.BN / 4;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int p = 0; p < a.pieces; ++p) {
        const float4 v = __ldcg(src + p * step);
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    return s;
}

__device__ __forceinline__ void ffn_put4(__nv_bfloat16 *p, const float (&v)[4]) {
    __nv_bfloat162 b[2] = {__floats2bfloat162_rn(v[0], v[1]), __floats2bfloat162_rn(v[2], v[3])};
    *reinterpret_cast<uint2 *>(p) = *reinterpret_cast<uint2 *>(b);
}

__device__ __forceinline__ void ffn_get4(const __nv_bfloat16 *p, float (&v)[4]) {
    const uint2 u = *reinterpret_cast<const uint2 *>(p);
    const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&u.x));
    const float2 b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&u.y));
    v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
}

template <bool GRAD>
__global__ void __launch_bounds__(256) ffn_reduce_kernel(const FfnReduce a) {
    griddep_launch_dependents();
    griddep_wait();
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int n4 = a.N / 4;
    if (i >= (int64_t)a.M * n4) return;
    const int row = (int)(i / n4), col = (int)(i - (int64_t)row * n4) * 4;
    const int tn = col / a.n_tile, c = col - tn * a.n_tile;
    const int64_t y = part_row(row / a.rows, tn, a.tiles_m, 0, a.pieces, a.rows) + row % a.rows;
    const int64_t o = (int64_t)row * a.N + col;
    const float4 s0 = ffn_pieces(a, y, c);
    const float v0[4] = {s0.x, s0.y, s0.z, s0.w};
    float r0[4], r1[4];
    if constexpr (GRAD) {
        float g[4], u[4];
        ffn_get4(a.gate + o, g);
        ffn_get4(a.up + o, u);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float f, slope;
            ffn_act(a.act, g[k], f, slope);
            r0[k] = v0[k] * u[k] * slope;
            r1[k] = v0[k] * f;
        }
        ffn_put4(a.out0 + o, r0);
        ffn_put4(a.out1 + o, r1);
    } else {
        const float4 s1 = ffn_pieces(a, y, a.BN / 2 + c);
        const float v1[4] = {s1.x, s1.y, s1.z, s1.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float f, slope;
            ffn_act(a.act, v0[k], f, slope);
            r0[k] = f * v1[k];
        }
        ffn_put4(a.out0 + o, r0);
        if (a.out1) {
            ffn_put4(a.out1 + o, v0);
            ffn_put4(a.out2 + o, v1);
        }
    }
}

static attt_status launch_pdl(const void *kern, dim3 grid, dim3 block, void **args, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelExC(&cfg, kern, args) != cudaSuccess) return ATTT_ERR_CUDA;
    count_launch();
    return cudaGetLastError() == cudaSuccess ? ATTT_OK : ATTT_ERR_CUDA;
}

// ---------------------------------------------------------------------------
// Contractions
// ---------------------------------------------------------------------------

// One operand pair of a contraction: A [M, K] (row pitch a_ld) with B: [N, K] K-major, or DUAL
// the gate's and the up's [K, N] (either may be nullptr: zeros).
struct FfnPair {
    const void *a;
    int64_t a_ld, K;
    const void *b, *b2;
    int64_t b_ld;
    int up_k;  // DUAL: column of A at which the up's K range begins (the gate's begins at 0)
    int64_t b_rows;  // rows of K that B has (DUAL)
};

struct FfnProblem {
    FfnPair pair[kFfnSegs];
    int npair;
    int M, N;
    int act;
    bool keep;
    const __nv_bfloat16 *gate, *up;
    __nv_bfloat16 *out[3];
    float *split_ws;
    bool pdl, operands_ready;
};

// The cut of least estimated time, as plan_tiles (gemm_launch.cuh), for the tiles that the
// block's kernels have (DUAL: 256 or 128 accumulator columns, in whole 64-column boxes of
// either half), with the bytes that have to come from HBM as a lower bound: few rows
// take that long however they are cut.
static TilePlan ffn_plan(int64_t M, int64_t N, int64_t kb, bool dual, double bytes, int sms) {
    TilePlan best{M > 128, 256, 1};
    double best_t = 1e30;
    // pairs only where both CTAs have rows: for fewer an empty half is filled with zeros and multiplied (forward at
    // 5,120 x 27,648: 9 rows 199 us, single CTAs 144; 128 rows 154, 156)
    for (int pair = M > 128 ? 1 : 0; pair >= 0; --pair) {
        const int64_t rows = pair ? 256 : 128, units = pair ? sms / 2 : sms;
        for (int BN = 256; BN >= 64; BN -= 64) {
            if (dual ? BN % 128 != 0 : pair && BN == 64) continue;
            const int n_tile = dual ? BN / 2 : BN;
            const int64_t tiles = cdiv(M, rows) * cdiv(N, n_tile);
            const double mma = pair && BN == 192 ? 0.29e-6 : 128.0 * BN * 128 / kSmFlops;
            const double feed = block_feed_seconds(pair, BN, false), block = mma > feed ? mma : feed;
            for (int64_t s = 1; s <= kMaxPieces; ++s) {
                if (s > 1 && (kb < 16 * s || tiles * s * (rows / 128) * BN > kFfnRegions * 256)) break;
                const double waves = (double)cdiv(tiles * s, units);
                const double extra = s > 1 ? kReduceFixed + kReduceByte * 4.0 * s * M * N * (dual ? 4 : 2) : 0.0;
                const double run = waves * cdiv(kb, s) * block, hbm = bytes / 6.7e12;
                const double t = (run > hbm ? run : hbm) + kTileFixed + BN * kTileColumn + extra;
                if (t < 0.98 * best_t) {
                    best_t = t;
                    best = TilePlan{pair != 0, BN, (int)s};
                }
            }
        }
    }
    return best;
}

template <int EPI, bool DUAL, bool PAIR, int SETS>
static attt_status ffn_launch(const FfnMaps &maps, const FfnArgs &p, size_t smem, int grid, bool pdl, int dev,
                              cudaStream_t stream) {
    auto kern = ffn_kernel<EPI, DUAL, PAIR, SETS>;
    if (!set_smem_limit(reinterpret_cast<const void *>(kern), smem, dev)) return ATTT_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)ffn_threads(SETS));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    unsigned na = 0;
    if (pdl) {
        attr[na].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[na].val.programmaticStreamSerializationAllowed = 1;
        ++na;
    }
    if (PAIR) {
        attr[na].id = cudaLaunchAttributeClusterDimension;
        attr[na].val.clusterDim.x = 2;
        attr[na].val.clusterDim.y = 1;
        attr[na].val.clusterDim.z = 1;
        ++na;
    }
    cfg.attrs = attr;
    cfg.numAttrs = na;
    if (cudaLaunchKernelEx(&cfg, kern, maps, p) != cudaSuccess) return ATTT_ERR_CUDA;
    count_launch();
    return cudaGetLastError() == cudaSuccess ? ATTT_OK : ATTT_ERR_CUDA;
}

template <int EPI, bool DUAL>
static attt_status ffn_launch_form(const FfnMaps &maps, const FfnArgs &p, size_t smem, int grid, bool pair, int sets,
                                   bool pdl, int dev, cudaStream_t stream) {
    if constexpr (EPI == FFN_GLU || EPI == FFN_GLU_GRAD)
        if (sets == 2)
            return pair ? ffn_launch<EPI, DUAL, true, 2>(maps, p, smem, grid, pdl, dev, stream)
                        : ffn_launch<EPI, DUAL, false, 2>(maps, p, smem, grid, pdl, dev, stream);
    return pair ? ffn_launch<EPI, DUAL, true, 1>(maps, p, smem, grid, pdl, dev, stream)
                : ffn_launch<EPI, DUAL, false, 1>(maps, p, smem, grid, pdl, dev, stream);
}

// Runs the contraction q with epilogue EPI, whole or in K pieces and a reduction.
template <int EPI, bool DUAL>
static attt_status ffn_contract(const FfnProblem &q, int dev, cudaStream_t stream) {
    int64_t kb = 0;
    double bytes = 0.0;
    for (int i = 0; i < q.npair; ++i) {
        kb += cdiv(q.pair[i].K, 64);
        bytes += 2.0 * q.pair[i].K * ((DUAL ? 2.0 : 1.0) * q.N + q.M);
    }
    if (kb > (1ll << 30)) return ATTT_ERR_UNSUPPORTED;
    const int sms = num_sms(dev);
    const TilePlan t = ffn_plan(q.M, q.N, kb, DUAL, bytes, sms);
    const int n_tile = DUAL ? t.BN / 2 : t.BN, rows = t.pair ? 256 : 128;
    const bool part = t.pieces > 1;
    const int sets = !part && EPI != FFN_OUT && kb <= kTwoSetBlocks ? 2 : 1;

    FfnMaps maps;
    FfnArgs p{};
    GemmArgs &g = p.g;
    // loads of a single row tile end with its last row (GemmProblem::tight)
    const uint32_t a_box = !t.pair && q.M < 128 ? (uint32_t)round_up(q.M, 8) : 128u;
    const uint32_t b_box = (uint32_t)(t.pair ? t.BN / 2 : t.BN);
    int na = 0, nb = 0, end = 0;
    for (int i = 0; i < q.npair; ++i) {
        const FfnPair &o = q.pair[i];
        FfnSeg &s = p.seg[p.nseg++];
        // pairs that follow one another may share A
        const bool same = i > 0 && o.a == q.pair[i - 1].a && o.a_ld == q.pair[i - 1].a_ld;
        if (!same) {
            if (na == 3) return ATTT_ERR_INVALID_ARG;
            if (!make_tmap_bf16(&maps.a[na++], o.a, (uint64_t)o.a_ld, (uint64_t)q.M, (uint64_t)o.a_ld * 2, 64, a_box))
                return ATTT_ERR_INVALID_ARG;
        }
        s.a = na - 1;
        end += (int)cdiv(o.K, 64);
        s.end = end;
        if (DUAL) {
            if (nb + 2 > 4) return ATTT_ERR_INVALID_ARG;
            const void *b[2] = {o.b ? o.b : o.b2, o.b2 ? o.b2 : o.b};
            for (int j = 0; j < 2; ++j)
                if (!make_tmap_bf16(&maps.b[nb + j], b[j], (uint64_t)q.N, (uint64_t)o.b_rows, (uint64_t)o.b_ld * 2, 64,
                                    64))
                    return ATTT_ERR_INVALID_ARG;
            // rows of K before a B's first and past its last are zeros; one that is missing lies past the end
            s.b = nb; s.b_k = o.b ? 0 : (int)o.b_rows;
            s.b2 = nb + 1; s.b2_k = o.b2 ? -o.up_k : (int)o.b_rows;
            nb += 2;
        } else {
            if (nb == 4) return ATTT_ERR_INVALID_ARG;
            if (!make_tmap_bf16(&maps.b[nb], o.b, (uint64_t)o.b_rows, (uint64_t)q.N, (uint64_t)o.b_ld * 2, 64, b_box))
                return ATTT_ERR_INVALID_ARG;
            s.b = nb++;
            s.a_k = o.up_k;
        }
    }
    for (; na < 3; ++na) maps.a[na] = maps.a[0];
    for (; nb < 4; ++nb) maps.b[nb] = maps.b[0];
    const int tiles_m = (int)cdiv(q.M, rows);
    if (part) {
        const int64_t n = (int64_t)tiles_m * cdiv(q.N, n_tile) * t.pieces * (t.pair ? 2 : 1);
        if (n * t.BN > (int64_t)kFfnRegions * 256) return ATTT_ERR_INVALID_ARG;
        if (!make_tmap_f32(&maps.c[0], q.split_ws, (uint64_t)t.BN, (uint64_t)n * 128, (uint64_t)t.BN * 4, 32, 32))
            return ATTT_ERR_INVALID_ARG;
        maps.c[1] = maps.c[2] = maps.c[0];
    } else {
        for (int i = 0; i < 3; ++i) {
            if (!q.out[i]) {
                maps.c[i] = maps.c[0];
                continue;
            }
            if (!make_tmap_bf16(&maps.c[i], q.out[i], (uint64_t)q.N, (uint64_t)q.M, (uint64_t)q.N * 2, 32, 32, 64))
                return ATTT_ERR_INVALID_ARG;
        }
    }

    g.M = q.M;
    g.N = q.N;
    g.BN = t.BN;
    g.e_stage_bytes = part ? kF32StageBytes : (uint32_t)sets * kEStageBytes;
    const int bn_cta = t.pair ? t.BN / 2 : t.BN;
    g.stages = gemm_stages(bn_cta, g.e_stage_bytes);
    g.tiles_m = (int)cdiv(q.M, 128);
    g.tiles_n = (int)cdiv(q.N, n_tile);
    g.kb_total = (int)kb;
    const int units = t.pair ? sms / 2 : sms, tiles = tiles_m * g.tiles_n;
    g.whole_tiles = part ? 0 : tiles;
    g.tail_s = t.pieces;
    g.tmem_cols = gemm_tmem_cols(t.BN);
    g.operands_ready = q.operands_ready ? 1 : 0;
    g.group_m = tile_group(q.M, rows, 2048 / rows, 128.0 * q.M * kb);
    g.a_bytes = a_box * 128u;
    g.status = device_status_word(dev);
    g.ep.alpha = 1.0f;
    p.act = q.act;
    p.keep = q.keep ? 1 : 0;
    p.gate = q.gate;
    p.up = q.up;
    const size_t smem = gemm_smem_bytes(bn_cta, g.stages, g.e_stage_bytes);
    const int nwork = tiles * (part ? t.pieces : 1);
    const int grid = t.pair ? 2 * std::min(nwork, units) : std::min(nwork, units);
    attt_status st = part ? ffn_launch_form<FFN_PART, DUAL>(maps, p, smem, grid, t.pair, sets, q.pdl, dev, stream)
                          : ffn_launch_form<EPI, DUAL>(maps, p, smem, grid, t.pair, sets, q.pdl, dev, stream);
    if (st != ATTT_OK || !part) return st;
    if constexpr (EPI == FFN_OUT) {
        SplitReduceArgs a{};
        a.part = q.split_ws;
        a.M = q.M; a.N = q.N; a.BN = t.BN; a.pieces = t.pieces; a.rows = rows; a.tiles_m = tiles_m;
        a.ld = q.N; a.alpha = 1.0f; a.out16 = q.out[0];
        return launch_split_reduce(a, stream);
    } else {
        FfnReduce a{};
        a.part = q.split_ws;
        a.M = q.M; a.N = q.N; a.BN = t.BN; a.n_tile = n_tile; a.pieces = t.pieces; a.rows = rows; a.tiles_m = tiles_m;
        a.act = q.act;
        a.gate = q.gate; a.up = q.up;
        a.out0 = q.out[0]; a.out1 = q.out[1]; a.out2 = q.out[2];
        void *args[] = {&a};
        const dim3 blocks((unsigned)cdiv((int64_t)q.M * (q.N / 4), 256));
        return launch_pdl(reinterpret_cast<const void *>(&ffn_reduce_kernel<EPI == FFN_GLU_GRAD>), blocks, dim3(256),
                          args, stream);
    }
}

// ---------------------------------------------------------------------------
// Few rows
// ---------------------------------------------------------------------------

// One contraction of a call: activations a[i] [M, K] against weights b (FEW_GLU: gate and up of one
// segment; FEW_DX: one of each segment) and up to two adapters.
struct FewProblem {
    const void *a[2], *b[2];
    int64_t K;  // of a segment
    int M, N;
    struct {
        const void *first;   // FEW_GLU, FEW_DOWN: A [K, r8]; else B [r, K]
        const void *second;  // B [r, N] or A [N, r]
        int slot;            // segment, or half of FEW_GLU
    } rank[2];
    int nrank, r, r8;
    float scale;
    bool pdl, weights_wait;
    int act;
    const __nv_bfloat16 *gate, *up;
    __nv_bfloat16 *out[3];
};

// The tile's columns, the CTAs per tile and per SM.  An SM takes a stage's bytes at some 65 a ns; a CTA
// begins and ends in some 5 us, 15 more for every wave after the first (with 5 the estimate took waves where two
// CTAs per SM, each with half of shared memory and of TMEM, were the faster: 1 row at 8,192 x 22,016
// forward 185 us, 163 so).  (Two per SM only for tiles of one CTA that
// are more than the SMs: a grid of fewer, or one that starts beside the previous one's end, is
// packed on half of the SMs: y of 64 rows at 5,120 x 27,648 61 -> 109 us.)
struct FewPlan {
    int n_tile, cluster, stages, per_sm;
};

static uint32_t few_w_bytes(int mode, int n_tile, int nrank, int rpad) {
    const int bn = mode == FEW_GLU ? 2 * n_tile : n_tile;
    return (uint32_t)bn * 128u + (uint32_t)nrank * (uint32_t)(mode == FEW_GLU || mode == FEW_DOWN ? few_rank_cols(rpad) : rpad) * 128u;
}

// Shared memory behind the ring: the rank-r products, the second matrices, barriers.
static uint32_t few_products(int M, int nrank, int rpad) { return (uint32_t)round_up(M, 16) * (nrank * rpad + 8) * 2u; }
static uint32_t few_second(int n_tile, int nrank, int rpad) { return (uint32_t)(nrank * n_tile * (rpad + 8)) * 2u; }
static uint32_t few_tail(int M, int n_tile, int nrank, int rpad) {
    return few_products(M, nrank, rpad) + few_second(n_tile, nrank, rpad) + 8u * (2 * kFewMaxStages + 1) + 16u;
}
static uint32_t few_sums(int mode, int M, int n_tile, int nrank, int rpad) {
    const int cols = (mode == FEW_GLU ? 2 * n_tile : n_tile) + nrank * rpad;
    return (uint32_t)(M * (cols + 4) * 4);
}

static FewPlan few_plan(int mode, int M, int64_t N, int64_t kb, int nrank, int rpad, double bytes, bool pdl, int dev) {
    FewPlan best{64, 1, 2, 1};
    double best_t = 1e30;
    const uint32_t a_alloc = (uint32_t)round_up(M, 8) * 128u;
    for (int per_sm = 1; per_sm <= 2; ++per_sm)
        for (int n_tile = 128; n_tile >= 64; n_tile /= 2) {
            // the second launch, and two CTAs per SM, with narrow tiles: 4 rows at 4,096 x 14,336 with r = 16 forward 88 us
            // (73 so), backward 94 (73); at 5,120 x 27,648 174 (167)
            if ((pdl || per_sm == 2) && n_tile == 64) continue;
            const int cols = (mode == FEW_GLU ? 2 * n_tile : n_tile) + nrank * rpad;
            if (cols * per_sm > 512) continue;
            const uint32_t w = few_w_bytes(mode, n_tile, nrank, rpad), total = per_sm == 2 ? 115200u : (uint32_t)kMaxSmem,
                           tail = few_tail(M, n_tile, nrank, rpad) + 2048u;
            if (tail + few_sums(mode, M, n_tile, nrank, rpad) > total || tail + 2 * (a_alloc + w) > total) continue;
            const int stages = (int)std::min<uint32_t>(kFewMaxStages, (total - tail) / (a_alloc + w));
            if (a_alloc + stages * w < 16384u) continue;
            const int64_t tiles = cdiv(N, n_tile);
            if (per_sm == 2 && tiles <= resident_clusters(1, dev)) continue;
            for (int c = 1; c <= (per_sm == 2 ? 1 : kFewMaxCluster) && c <= kb; ++c) {
                // clusters that start while the previous grid's CTAs leave are not packed as those of an idle
                // device: with all places needed some ran after the others (28 clusters of 5, 140 CTAs, dx of 93
                // rows at 3,584 x 18,944: 85 us, 62 with fewer)
                const int held = resident_clusters(c, dev), places = pdl && c > 1 ? std::max(1, held * 15 / 16) : held;
                const int64_t each = cdiv(tiles, places), waves = cdiv(each, per_sm);
                // and clusters in waves cost more than this estimate: 32 rows at 5,120 x 27,648 with r = 16 backward
                // 172 us (153 without), 4 rows at 5,120 x 13,824 with r = 64 forward 121 (100)
                if (c > 1 && each > 1) continue;
                const double run = (double)each * cdiv(kb, c) * (a_alloc + w) / 65e9, hbm = bytes / 6.7e12;
                const double end = M * (double)(mode == FEW_GLU ? 2 : 1) * n_tile * 8 / 100e9;
                const double t = (run > hbm ? run : hbm) + waves * (15.0e-6 + end) - 10.0e-6 + (c > 1 ? 1.0e-6 : 0.0);
                if (t < 0.98 * best_t) {
                    best_t = t;
                    best = FewPlan{n_tile, c, (int)std::min<int64_t>(stages, cdiv(kb, c)), per_sm};
                    if (best.stages < 2) best.stages = 2;
                }
            }
        }
    return best;
}

template <int MODE>
static attt_status few_contract(const FewProblem &q, int dev, cudaStream_t stream) {
    constexpr bool mn = MODE == FEW_GLU || MODE == FEW_DOWN;
    const int rpad = (int)round_up(q.r, 16), nseg = MODE == FEW_DX ? 2 : 1;
    const int64_t kbs = cdiv(q.K, 64), kb = kbs * nseg;
    if (kb > (1ll << 30)) return ATTT_ERR_UNSUPPORTED;
    const double bytes = 2.0 * q.K * nseg * (q.M + q.N * (MODE == FEW_GLU ? 2.0 : 1.0));
    const FewPlan t = few_plan(MODE, q.M, q.N, kb, q.nrank, rpad, bytes, q.pdl, dev);

    FewMaps maps;
    FewArgs p{};
    p.M = q.M; p.N = q.N; p.n_tile = t.n_tile;
    p.BN = MODE == FEW_GLU ? 2 * t.n_tile : t.n_tile;
    p.nseg = nseg;
    p.kb[0] = p.kb[1] = (int)kbs;
    p.kb_total = (int)kb;
    p.nrank = q.nrank; p.r = q.r; p.rpad = rpad;
    p.scale = q.scale;
    p.cluster = t.cluster; p.stages = t.stages;
    p.a_bytes = p.a_alloc = (uint32_t)round_up(q.M, 8) * 128u;
    p.b_bytes = (uint32_t)p.BN * 128u;
    p.r_cols = few_rank_cols(rpad);
    p.r_bytes = (uint32_t)(mn ? p.r_cols : rpad) * 128u;
    const uint32_t ring = (uint32_t)t.stages * (p.a_alloc + few_w_bytes(MODE, t.n_tile, q.nrank, rpad));
    p.ring_bytes = (uint32_t)round_up(std::max({ring, few_sums(MODE, q.M, t.n_tile, q.nrank, rpad), p.a_alloc + 16384u}), 1024);
    const int cols = p.BN + q.nrank * rpad;
    p.pitch = cols + 4;
    p.vpitch = q.nrank * rpad + 8;
    p.tmem_cols = 32;
    while ((int)p.tmem_cols < cols) p.tmem_cols <<= 1;
    p.weights_wait = q.weights_wait ? 1 : 0;
    p.act = q.act;
    p.keep = MODE == FEW_GLU && q.out[1] ? 1 : 0;
    p.gate = q.gate; p.up = q.up;
    for (int i = 0; i < 3; ++i) p.out[i] = q.out[i];
    p.status = device_status_word(dev);
    const uint32_t a_box = (uint32_t)round_up(q.M, 8);
    for (int i = 0; i < 2; ++i) {
        const bool seg = i < nseg;
        if (!seg) maps.a[i] = maps.a[0];
        else if (!make_tmap_bf16(&maps.a[i], q.a[i], (uint64_t)q.K, (uint64_t)q.M, (uint64_t)q.K * 2, 64, a_box))
            return ATTT_ERR_INVALID_ARG;
        const bool has = MODE == FEW_GLU || seg;
        if (!has) maps.b[i] = maps.b[0];
        else if (mn ? !make_tmap_bf16(&maps.b[i], q.b[i], (uint64_t)q.N, (uint64_t)q.K, (uint64_t)q.N * 2, 64, 64)
                    : !make_tmap_bf16(&maps.b[i], q.b[i], (uint64_t)q.K, (uint64_t)q.N, (uint64_t)q.K * 2, 64,
                                      (uint32_t)t.n_tile))
            return ATTT_ERR_INVALID_ARG;
        if (i >= q.nrank) {
            maps.r[i] = maps.b[0];
            continue;
        }
        if (mn ? !make_tmap_bf16(&maps.r[i], q.rank[i].first, (uint64_t)q.r8, (uint64_t)q.K, (uint64_t)q.r8 * 2,
                                 (uint32_t)p.r_cols, 64, 2 * p.r_cols)
               : !make_tmap_bf16(&maps.r[i], q.rank[i].first, (uint64_t)q.K, (uint64_t)q.r, (uint64_t)q.K * 2, 64,
                                 (uint32_t)rpad))
            return ATTT_ERR_INVALID_ARG;
        p.rank[i] = FewRank{MODE == FEW_DX ? q.rank[i].slot : 0, p.BN + i * rpad, MODE == FEW_GLU ? q.rank[i].slot : 0,
                            static_cast<const __nv_bfloat16 *>(q.rank[i].second), mn ? (int64_t)q.N : (int64_t)q.r};
    }
    p.second_at = p.ring_bytes + few_products(q.M, q.nrank, rpad);
    p.bars_at = p.second_at + few_second(t.n_tile, q.nrank, rpad);
    size_t smem = 1024 + (size_t)p.ring_bytes + few_tail(q.M, t.n_tile, q.nrank, rpad);
    if (t.per_sm == 1) smem = std::max<size_t>(smem, 118784);  // so that an SM takes one
    auto kern = ffn_few_kernel<MODE>;
    if (smem > kMaxSmem || !set_smem_limit(reinterpret_cast<const void *>(kern), smem, dev)) return ATTT_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(cdiv(q.N, t.n_tile) * t.cluster));
    cfg.blockDim = dim3(kFewThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    unsigned na = 0;
    if (q.pdl) {
        attr[na].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[na].val.programmaticStreamSerializationAllowed = 1;
        ++na;
    }
    if (t.cluster > 1) {
        attr[na].id = cudaLaunchAttributeClusterDimension;
        attr[na].val.clusterDim.x = (unsigned)t.cluster;
        attr[na].val.clusterDim.y = 1;
        attr[na].val.clusterDim.z = 1;
        ++na;
    }
    cfg.attrs = attr;
    cfg.numAttrs = na;
    if (cudaLaunchKernelEx(&cfg, kern, maps, p) != cudaSuccess) return ATTT_ERR_CUDA;
    count_launch();
    return cudaGetLastError() == cudaSuccess ? ATTT_OK : ATTT_ERR_CUDA;
}

// Which calls tc_ffn_few.cuh's kernels take.  Two launches and wider loads win where the weights'
// bytes and the launches are what a call costs; the chain of up to seven launches loads an
// adapter's columns once instead of once per cluster, and its tiles waste less on more rows.
// Times of the chain / of these kernels, us, replayed from a graph, weights not in L2 (f in tiles of 128: 148, 216, 64):
//   rows, r      3,584 x 18,944: forward, backward    5,120 x 27,648               2,048 x 8,192
//     8,  0      75.1 /  69.6   79.6 /  74.1   144.6 / 129.3  154.2 / 137.5    28.4 /  28.2   30.7 /  29.9
//    32,  0      75.9 /  72.5   80.7 /  76.7   146.7 / 132.4  154.9 / 141.7    29.1 /  30.0   31.4 /  32.5
//    64,  0      77.4 /  75.9   81.9 /  80.7   149.2 / 144.9  157.5 / 148.4    29.7 /  34.2   33.0 /  33.7
//    96,  0      79.6 /  79.8   85.6 /  84.5   152.8 / 151.9  159.2 / 156.2    30.2 /  39.5   33.9 /  38.3
//     8, 16      98.7 /  80.1  101.1 /  82.0   166.2 / 166.4  176.2 / 148.7    39.3 /  37.9   43.2 /  37.7
//    32, 16      99.6 /  82.5  103.9 /  84.3   168.7 / 169.6  176.7 / 153.0    39.5 /  40.8   43.6 /  39.5
//    64, 16     100.2 /  87.2  104.3 /  89.7   171.9 / 179.6  178.2 / 162.2    40.3 /  43.2   44.6 /  41.8
//    96, 16     102.0 /  91.6  109.0 /  95.5   174.5 / 189.7  181.8 / 172.1    41.5 /  49.8   45.7 /  47.8
//     8, 32      99.0 /  81.5  101.8 /  83.1   167.1 / 171.2  176.9 / 150.0    39.4 /  39.1   43.1 /  37.9
//    32, 32     100.5 /  84.0  103.2 /  86.4   169.0 / 174.7  177.2 / 155.1    40.0 /  42.6   44.3 /  40.9
//    64, 32     100.8 /  89.3  105.5 /  92.9   171.8 / 183.7  180.3 / 166.6    40.9 /  45.2   44.7 /  44.1
//    96, 32     102.6 /  97.1  109.0 / 100.0   174.8 / 204.2  181.9 / 190.9    42.2 /  53.9   46.0 /  51.6
//     8, 64     100.0 /  90.6  102.2 /  88.4   168.3 / 188.8  177.7 / 162.1    40.0 /  42.9   43.5 /  40.4
//    32, 64     101.2 /  91.1  104.2 /  92.6   170.1 / 195.3  177.7 / 167.4    40.7 /  47.0   44.6 /  44.5
//    64, 64     101.9 /  97.8  106.1 / 106.4   173.0 / 206.3  180.3 / 200.8    41.8 /  51.2   45.1 /  51.3
//    96, 64     103.7 / 120.3  109.5 / 122.2   176.4 / 265.2  182.4 / 228.5    42.7 /  64.9   46.1 /  63.2
// The limits go by d f, r, direction and whether f's tiles fit the SMs, not cell by cell, and an adapted forward call
// whose tiles do not fit takes the chain at any number of rows (166 to 173 us against 166 to 206 at 5,120 x 27,648).  Where the table's
// rows take the slower side by more than 2%: forward 3,584 x 18,944, 96 rows, r 16 (11%) and 32 (6%), 64 rows, r 64 (4%);
// 2,048 x 8,192, 8 rows, r 64 (7%); backward 2,048 x 8,192, 32 and 64 rows, r 16 (10%, 7%), 32 rows, r 32 (8%);
// 5,120 x 27,648, 96 rows, r 16 (6%).
static bool ffn_few(int64_t L, int64_t d, int64_t f, int r, bool back, int dev) {
    if (d * f <= 1ll << 24) return L <= 8;
    const bool fits = cdiv(f, 128) <= num_sms(dev);  // f's tiles on an SM each
    if (back) return L <= (r > 32 ? 32 : fits ? kFewRows : 64);
    return (fits || r == 0) && L <= (r > 32 ? 32 : 64);
}

// ---------------------------------------------------------------------------
// Arguments
// ---------------------------------------------------------------------------

struct FfnAdapters {
    const void *A[3], *B[3];  // nullptr: the projection has none
};

// Reads the host arrays of adapters (both NULL: none); false if one of a pair is missing.
static bool ffn_adapters(const attt_bf16 *const *d_A, const attt_bf16 *const *d_B, int r, FfnAdapters &ad) {
    ad = FfnAdapters{};
    if (!d_A != !d_B || (d_A != nullptr) != (r > 0)) return false;
    for (int i = 0; d_A && i < 3; ++i) {
        if (!d_A[i] != !d_B[i]) return false;
        if (!aligned16(d_A[i]) || !aligned16(d_B[i])) return false;
        ad.A[i] = d_A[i];
        ad.B[i] = d_B[i];
    }
    return true;
}

// What a call reads of the weights and adapters.
static void ffn_reads(const void *Wg, const void *Wu, const void *Wd, const FfnAdapters &ad, int64_t d, int64_t f, int r,
                      ByteRange (&in)[9]) {
    int n = 0;
    for (const void *w : {Wg, Wu, Wd}) in[n++] = ByteRange{w, 2 * d * f};
    for (int i = 0; i < 3; ++i) {
        in[n++] = ByteRange{ad.A[i], 2 * (i < 2 ? d : f) * r};
        in[n++] = ByteRange{ad.B[i], 2 * r * (i < 2 ? f : d)};
    }
}

// Whether a call's results share no byte with each other or with what it reads: out[0] is the
// last launch's, when `before` is read no more; out[j] may be same[j] itself.
template <int NO, int NB>
static bool ffn_apart(const ByteRange (&out)[NO], const void *const (&same)[NO], const ByteRange (&in)[9],
                      const ByteRange (&before)[NB]) {
    for (int j = 0; j < NO; ++j) {
        for (int k = 0; k < j; ++k)
            if (share_a_byte(out[j], out[k])) return false;
        for (const ByteRange &b : in)
            if (share_a_byte(out[j], b)) return false;
        for (const ByteRange &b : before)
            if (j > 0 && share_a_byte(out[j], b) && !(same[j] && same[j] == b.at && out[j].at == b.at)) return false;
    }
    return true;
}

// Copies of the adapters' A whose rows TMA cannot read; `mask`: of which projections.
// `launched`: whether that took a launch.
static attt_status ffn_pad_adapters(FfnAdapters &ad, int mask, const FfnLayout &c, int64_t d, int64_t f, int r, int dev,
                                    bool &launched, cudaStream_t stream) {
    if (r % 8 == 0) return ATTT_OK;
    FfnPad a{};
    a.r = r;
    a.r8 = c.r8;
    for (int i = 0; i < 3; ++i) {
        if (!(mask >> i & 1) || !ad.A[i]) continue;
        a.src[i] = static_cast<const __nv_bfloat16 *>(ad.A[i]);
        a.dst[i] = c.pad[i];
        a.n[i] = i < 2 ? d : f;
        ad.A[i] = c.pad[i];
        launched = true;
    }
    if (!launched) return ATTT_OK;
    ffn_pad_kernel<<<dim3((unsigned)std::min<int64_t>(cdiv(std::max(d, f) * c.r8, 256), num_sms(dev)), 3), 256, 0,
                     stream>>>(a);
    count_launch();
    return cudaGetLastError() == cudaSuccess ? ATTT_OK : ATTT_ERR_CUDA;
}

}  // namespace attt

extern "C" {

size_t attt_gated_ffn_workspace_bytes(int64_t L, int64_t d, int64_t f, int r) {
    if (attt::ffn_sizes(L, d, f, r) != ATTT_OK) return 0;
    return attt::ffn_layout(nullptr, L, d, f, r).bytes;
}

attt_status attt_gated_ffn_forward(const attt_bf16 *d_x, const attt_bf16 *d_Wg, const attt_bf16 *d_Wu,
                                   const attt_bf16 *d_Wd, const attt_bf16 *const *d_A, const attt_bf16 *const *d_B,
                                   int64_t L, int64_t d, int64_t f, int r, float scale, int act, attt_bf16 *d_y,
                                   attt_bf16 *d_h, attt_bf16 *d_g, attt_bf16 *d_u, void *d_ws, size_t ws_bytes,
                                   attt_stream stream) {
    ATTT_NVTX_RANGE();
    using namespace attt;
    attt_status st = ffn_sizes(L, d, f, r);
    if (st != ATTT_OK) return st;
    FfnAdapters ad;
    if (!d_Wg || !d_Wu || !d_Wd || (L > 0 && (!d_x || !d_y || !d_h)) || !d_g != !d_u) return ATTT_ERR_INVALID_ARG;
    if ((act != FFN_SILU && act != FFN_GELU_TANH) || !ffn_adapters(d_A, d_B, r, ad)) return ATTT_ERR_INVALID_ARG;
    if (!aligned_to(16, d_x, d_Wg, d_Wu, d_Wd, d_y, d_h, d_g, d_u)) return ATTT_ERR_INVALID_ARG;
    if (!d_ws || !aligned256(d_ws) || ws_bytes < attt_gated_ffn_workspace_bytes(L, d, f, r)) return ATTT_ERR_WORKSPACE;
    if (L == 0) return ATTT_OK;
    const FfnLayout c = ffn_layout(d_ws, L, d, f, r);
    {
        ByteRange in[9];
        ffn_reads(d_Wg, d_Wu, d_Wd, ad, d, f, r, in);
        const ByteRange out[5] = {{d_y, 2 * L * d}, {d_h, 2 * L * f}, {d_g, 2 * L * f}, {d_u, 2 * L * f},
                                  {d_ws, (int64_t)c.bytes}};
        const ByteRange before[1] = {{d_x, 2 * L * d}};
        const void *const same[5] = {};
        if (!ffn_apart(out, same, in, before)) return ATTT_ERR_INVALID_ARG;
    }
    int dev;
    st = current_device(&dev);
    if (st != ATTT_OK) return st;
    bool launched = false;  // whether this call has launched a kernel that the next one may depend on
    st = ffn_pad_adapters(ad, 7, c, d, f, r, dev, launched, stream);
    if (st != ATTT_OK) return st;

    if (ffn_few(L, d, f, r, false, dev)) {
        FewProblem q{};
        q.a[0] = d_x; q.b[0] = d_Wg; q.b[1] = d_Wu;
        q.K = d; q.M = (int)L; q.N = (int)f;
        q.r = r; q.r8 = c.r8; q.scale = scale;
        for (int i = 0; i < 2; ++i)
            if (ad.A[i]) {
                q.rank[q.nrank].first = ad.A[i];
                q.rank[q.nrank].second = ad.B[i];
                q.rank[q.nrank++].slot = i;
            }
        q.pdl = q.weights_wait = launched;
        q.act = act;
        q.out[0] = reinterpret_cast<__nv_bfloat16 *>(d_h);
        q.out[1] = reinterpret_cast<__nv_bfloat16 *>(d_g);
        q.out[2] = reinterpret_cast<__nv_bfloat16 *>(d_u);
        st = few_contract<FEW_GLU>(q, dev, stream);
        if (st != ATTT_OK) return st;
        FewProblem y{};
        y.a[0] = d_h; y.b[0] = d_Wd;
        y.K = f; y.M = (int)L; y.N = (int)d;
        y.r = r; y.r8 = c.r8; y.scale = scale;
        if (ad.A[2]) {
            y.rank[0].first = ad.A[2];
            y.rank[0].second = ad.B[2];
            y.nrank = 1;
        }
        y.pdl = true;
        y.weights_wait = launched;
        y.out[0] = reinterpret_cast<__nv_bfloat16 *>(d_y);
        return few_contract<FEW_DOWN>(y, dev, stream);
    }

    FfnProblem q{};
    q.M = (int)L; q.N = (int)f;
    q.act = act;
    q.keep = d_g != nullptr;
    q.out[0] = reinterpret_cast<__nv_bfloat16 *>(d_h);
    q.out[1] = reinterpret_cast<__nv_bfloat16 *>(d_g);
    q.out[2] = reinterpret_cast<__nv_bfloat16 *>(d_u);
    q.split_ws = c.split_ws;
    q.pair[q.npair++] = FfnPair{d_x, d, d, d_Wg, d_Wu, f, 0, d};
    if (ad.A[0] || ad.A[1]) {
        RankProduct list[2];
        int n = 0;
        for (int i = 0; i < 2; ++i)
            if (ad.A[i]) list[n++] = RankProduct{d_x, ad.A[i], d, true};
        st = rank_products(n, list, L, c.r8, c.rpad, scale, c.s2, launched, dev, stream);
        if (st != ATTT_OK) return st;
        q.operands_ready = !launched;  // x and the weights were there before that launch
        launched = true;
        q.pair[q.npair++] =
            FfnPair{c.s2, (int64_t)n * c.rpad, (int64_t)n * c.rpad, ad.B[0], ad.B[1], f, ad.B[0] ? c.rpad : 0, r};
    }
    q.pdl = launched;
    st = ffn_contract<FFN_GLU, true>(q, dev, stream);
    if (st != ATTT_OK) return st;

    if (ad.A[2]) {
        const RankProduct p{d_h, ad.A[2], f, true};
        st = rank_products(1, &p, L, c.r8, c.rpad, scale, c.s1, true, dev, stream);
        if (st != ATTT_OK) return st;
    }
    GemmProblem p{};
    p.a = d_h; p.a_rows_ld = f; p.a_rows = L; p.a_k = f;
    p.b = d_Wd; p.b_rows_ld = d; p.b_rows = d; p.b_k = f;
    if (ad.A[2]) {
        p.a2 = c.s1; p.a2_rows_ld = c.rpad; p.a2_rows = L; p.a2_k = c.rpad;
        p.b2 = ad.B[2]; p.b2_rows_ld = d; p.b2_rows = d; p.b2_k = r;
        p.K2 = c.rpad;
    }
    p.M = (int)L; p.N = (int)d; p.K = (int)f;
    p.pdl = true;
    p.tight = true;
    p.split_ws = c.split_ws; p.split_regions = kFfnRegions;
    EpiParams ep{};
    ep.out16 = reinterpret_cast<__nv_bfloat16 *>(d_y); ep.out_ld = d; ep.alpha = 1.0f;
    const TilePlan t = plan_tiles(L, d, cdiv(f, 64) + cdiv(p.K2, 64), num_sms(dev), kFfnRegions, false, true);
    return launch_planned<true, false, true>(p, ep, t, dev, stream);
}

attt_status attt_gated_ffn_backward(const attt_bf16 *d_dy, const attt_bf16 *d_Wg, const attt_bf16 *d_Wu,
                                    const attt_bf16 *d_Wd, const attt_bf16 *const *d_A, const attt_bf16 *const *d_B,
                                    const attt_bf16 *d_g, const attt_bf16 *d_u, int64_t L, int64_t d, int64_t f, int r,
                                    float scale, int act, attt_bf16 *d_dx, attt_bf16 *d_dg, attt_bf16 *d_du, void *d_ws,
                                    size_t ws_bytes, attt_stream stream) {
    ATTT_NVTX_RANGE();
    using namespace attt;
    attt_status st = ffn_sizes(L, d, f, r);
    if (st != ATTT_OK) return st;
    FfnAdapters ad;
    if (!d_Wg || !d_Wu || !d_Wd || (L > 0 && (!d_dy || !d_g || !d_u || !d_dg || !d_du))) return ATTT_ERR_INVALID_ARG;
    if ((act != FFN_SILU && act != FFN_GELU_TANH) || !ffn_adapters(d_A, d_B, r, ad)) return ATTT_ERR_INVALID_ARG;
    if (!aligned_to(16, d_dy, d_Wg, d_Wu, d_Wd, d_g, d_u, d_dx, d_dg, d_du)) return ATTT_ERR_INVALID_ARG;
    if (!d_ws || !aligned256(d_ws) || ws_bytes < attt_gated_ffn_workspace_bytes(L, d, f, r)) return ATTT_ERR_WORKSPACE;
    if (L == 0) return ATTT_OK;
    const FfnLayout c = ffn_layout(d_ws, L, d, f, r);
    {
        ByteRange in[9];
        ffn_reads(d_Wg, d_Wu, d_Wd, ad, d, f, r, in);
        const ByteRange out[4] = {{d_dx, 2 * L * d}, {d_dg, 2 * L * f}, {d_du, 2 * L * f}, {d_ws, (int64_t)c.bytes}};
        const ByteRange before[3] = {{d_dy, 2 * L * d}, {d_g, 2 * L * f}, {d_u, 2 * L * f}};
        const void *const same[4] = {nullptr, d_g, d_u, nullptr};
        if (!ffn_apart(out, same, in, before)) return ATTT_ERR_INVALID_ARG;
    }
    int dev;
    st = current_device(&dev);
    if (st != ATTT_OK) return st;
    if (ffn_few(L, d, f, r, true, dev)) {
        FewProblem q{};
        q.a[0] = d_dy; q.b[0] = d_Wd;
        q.K = d; q.M = (int)L; q.N = (int)f;
        q.r = r; q.scale = scale;
        if (ad.A[2]) {
            q.rank[0].first = ad.B[2];
            q.rank[0].second = ad.A[2];
            q.nrank = 1;
        }
        q.act = act;
        q.gate = reinterpret_cast<const __nv_bfloat16 *>(d_g);
        q.up = reinterpret_cast<const __nv_bfloat16 *>(d_u);
        q.out[0] = reinterpret_cast<__nv_bfloat16 *>(d_dg);
        q.out[1] = reinterpret_cast<__nv_bfloat16 *>(d_du);
        st = few_contract<FEW_GRAD>(q, dev, stream);
        if (st != ATTT_OK || !d_dx) return st;
        FewProblem x{};
        x.a[0] = d_dg; x.a[1] = d_du; x.b[0] = d_Wg; x.b[1] = d_Wu;
        x.K = f; x.M = (int)L; x.N = (int)d;
        x.r = r; x.scale = scale;
        for (int i = 0; i < 2; ++i)
            if (ad.A[i]) {
                x.rank[x.nrank].first = ad.B[i];
                x.rank[x.nrank].second = ad.A[i];
                x.rank[x.nrank++].slot = i;
            }
        x.pdl = true;
        x.out[0] = reinterpret_cast<__nv_bfloat16 *>(d_dx);
        return few_contract<FEW_DX>(x, dev, stream);
    }
    bool launched = false;
    st = ffn_pad_adapters(ad, d_dx ? 7 : 4, c, d, f, r, dev, launched, stream);
    if (st != ATTT_OK) return st;

    {   // dg, du of dh = dy Wd^T + s (dy Bd^T) Ad^T: Wd [f, d] and Ad [f, r] are read K-major
        FfnProblem q{};
        q.M = (int)L; q.N = (int)f;
        q.act = act;
        q.gate = reinterpret_cast<const __nv_bfloat16 *>(d_g);
        q.up = reinterpret_cast<const __nv_bfloat16 *>(d_u);
        q.out[0] = reinterpret_cast<__nv_bfloat16 *>(d_dg);
        q.out[1] = reinterpret_cast<__nv_bfloat16 *>(d_du);
        q.split_ws = c.split_ws;
        q.pair[q.npair++] = FfnPair{d_dy, d, d, d_Wd, nullptr, d, 0, d};
        if (ad.A[2]) {
            const RankProduct p{d_dy, ad.B[2], d, false};
            st = rank_products(1, &p, L, r, c.rpad, scale, c.s1, launched, dev, stream);
            if (st != ATTT_OK) return st;
            q.operands_ready = !launched;
            launched = true;
            q.pair[q.npair++] = FfnPair{c.s1, c.rpad, c.rpad, ad.A[2], nullptr, c.r8, 0, c.r8};
        }
        q.pdl = launched;
        st = ffn_contract<FFN_GLU_GRAD, false>(q, dev, stream);
        if (st != ATTT_OK || !d_dx) return st;
    }
    // dx = [dg | du | s dg Bg^T | s du Bu^T] [Wg^T ; Wu^T ; Ag^T ; Au^T], all read K-major
    FfnProblem q{};
    q.M = (int)L; q.N = (int)d;
    q.out[0] = reinterpret_cast<__nv_bfloat16 *>(d_dx);
    q.split_ws = c.split_ws;
    q.pdl = true;
    q.pair[q.npair++] = FfnPair{d_dg, f, f, d_Wg, nullptr, f, 0, f};
    q.pair[q.npair++] = FfnPair{d_du, f, f, d_Wu, nullptr, f, 0, f};
    RankProduct list[2];
    int n = 0;
    for (int i = 0; i < 2; ++i) n += ad.A[i] ? 1 : 0;
    for (int i = 0, k = 0; i < 2; ++i)
        if (ad.A[i]) {
            list[k] = RankProduct{i == 0 ? d_dg : d_du, ad.B[i], f, false};
            // columns past the product's own rpad meet the zeros past A's r8
            q.pair[q.npair++] =
                FfnPair{c.s2, (int64_t)n * c.rpad, c.rpad, ad.A[i], nullptr, c.r8, k * c.rpad, c.r8};
            ++k;
        }
    if (n > 0) {
        st = rank_products(n, list, L, r, c.rpad, scale, c.s2, true, dev, stream);
        if (st != ATTT_OK) return st;
    }
    return ffn_contract<FFN_OUT, false>(q, dev, stream);
}

}  // extern "C"

// rope.cu -- queries and keys between their projections and the attention: the
// norm of every head and the position rotation in one pass, and its gradient.
//
//   z = x rsqrt(mean(x^2) + eps) gamma     (a part with gamma; else z = x)
//   (a, b) of z's first `rot` values -> mscale (a cos - b sin, a sin + b cos), angle pos w_i
// Backward, dz = the rotation's transpose of dy, xh = x rstd, g = dz gamma:
//   dx = rstd (g - xh mean(g xh)),  dgamma = sum dz xh
//
// Bound: HBM bytes; below some hundred tokens a launch's latency.  A group of 2 to 32 lanes
// takes a head, a lane two 16-byte vectors of it: for the halves layout the two that
// turn together, so that the rotation needs no exchange and the norm one reduction over
// a few lanes.  The next head's vectors are loaded while one is worked on.  A block takes
// some tokens with all their heads, so that cosines are formed once per token.
// Angles: w_i is held in turns per position as a 64-bit fraction; pos w_i modulo 2^64
// is then the exact fraction of a turn whatever the position (fp32 products are off by
// 0.06 radians at position 10^6), and a quarter turn is taken off before it goes to fp32.
#include <algorithm>
#include <cmath>

#include "attt_common.cuh"
#include "attt_host.h"

namespace attt {

constexpr int kRopeThreads = 256;
constexpr int kRopeParts = 2;
constexpr int kRopeMaxD = 512;
constexpr int kRopeTable = 2048;  // cosines and sines that a block holds

struct RopeTensor {
    const void *x, *dy;
    void *y;  // forward: the result, backward: dx
    const float *gamma;
    int64_t x_ld, x_hs, dy_ld, dy_hs, y_ld, y_hs;
    int heads;
};

struct RopeArgs {
    RopeTensor part[kRopeParts];
    const int32_t *pos;
    const uint64_t *freq;
    int64_t T;
    int nparts, D, half, tokens;  // half: rot / 2; tokens: of a block at a time
    int block0[kRopeParts + 1];   // backward: first block of each part
    float eps, mscale;
    float *dgamma;                // backward: [blocks, D] partial sums, nullptr: not wanted
};

template <class T>
struct RopeVec {  // values of a 16-byte vector
    static constexpr int n = 16 / sizeof(T);
};

__device__ __forceinline__ void rope_get(const float *p, float (&v)[4]) {
    const float4 f = *reinterpret_cast<const float4 *>(p);
    v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
}
__device__ __forceinline__ void rope_get(const __nv_bfloat16 *p, float (&v)[8]) {
    const uint4 u = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void rope_get(const float *p, float (&v)[1]) { v[0] = *p; }
__device__ __forceinline__ void rope_get(const __nv_bfloat16 *p, float (&v)[1]) { v[0] = __bfloat162float(*p); }
__device__ __forceinline__ void rope_put(float *p, const float (&v)[4]) {
    *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void rope_put(__nv_bfloat16 *p, const float (&v)[8]) {
    __nv_bfloat162 b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    *reinterpret_cast<uint4 *>(p) = *reinterpret_cast<uint4 *>(b);
}
__device__ __forceinline__ void rope_put(float *p, const float (&v)[1]) { *p = v[0]; }
__device__ __forceinline__ void rope_put(__nv_bfloat16 *p, const float (&v)[1]) { *p = __float2bfloat16_rn(v[0]); }

// (cos, sin) of pos w, times mscale.  The nearest quarter turn comes off in integers, so
// that what is left keeps its relative precision.
__device__ __forceinline__ float2 rope_turn(int32_t pos, uint64_t w, float mscale) {
    const uint64_t turn = (uint64_t)(int64_t)pos * w;
    const uint32_t quarter = (uint32_t)((turn + (1ull << 61)) >> 62);
    const int64_t rest = (int64_t)(turn - ((uint64_t)quarter << 62));
    float s, c;
    sincospif((float)rest * 0x1p-63f, &s, &c);
    const float a = quarter & 1u ? -s : c, b = quarter & 1u ? c : s;
    const float sign = quarter & 2u ? -mscale : mscale;
    return make_float2(sign * a, sign * b);
}

// What a lane holds of a head: NS slots of V pairs.  Pair p < half turns: values p and p + half
// (halves) or 2 p and 2 p + 1 (neighbours); the others are 2 p and 2 p + 1 and do not.
// V > 1: the pairs of a slot are two vectors, at first() and second().
template <class T, int V, bool INTER>
struct RopeSlot {
    int pair;  // its first pair; at least D / 2: nothing
    __device__ __forceinline__ bool turns(int half) const { return pair < half; }
    __device__ __forceinline__ bool apart(int half) const { return !INTER && pair < half; }
    __device__ __forceinline__ int first(int half) const { return apart(half) ? pair : 2 * pair; }
    __device__ __forceinline__ int second(int half) const { return apart(half) ? pair + half : 2 * pair + V; }
    // the vectors' values as the two members of each pair, and back
    __device__ __forceinline__ void split(int half, float (&a)[V], float (&b)[V]) const {
        if constexpr (V > 1) {
            if (apart(half)) return;
            float v[2 * V];
#pragma unroll
            for (int i = 0; i < V; ++i) { v[i] = a[i]; v[V + i] = b[i]; }
#pragma unroll
            for (int i = 0; i < V; ++i) { a[i] = v[2 * i]; b[i] = v[2 * i + 1]; }
        }
    }
    __device__ __forceinline__ void join(int half, float (&a)[V], float (&b)[V]) const {
        if constexpr (V > 1) {
            if (apart(half)) return;
            float v[2 * V];
#pragma unroll
            for (int i = 0; i < V; ++i) { v[2 * i] = a[i]; v[2 * i + 1] = b[i]; }
#pragma unroll
            for (int i = 0; i < V; ++i) { a[i] = v[i]; b[i] = v[V + i]; }
        }
    }
};

template <int V, int NS>
struct RopeHead {
    float a[NS][V], b[NS][V];
};

template <class T, int V, int NS, bool INTER>
__device__ __forceinline__ void rope_load(const void *base, int64_t off, const RopeSlot<T, V, INTER> (&slot)[NS], int half,
                                          int pairs, RopeHead<V, NS> &h) {
    const T *p = static_cast<const T *>(base) + off;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        if (slot[s].pair < pairs) {
            rope_get(p + slot[s].first(half), h.a[s]);
            rope_get(p + slot[s].second(half), h.b[s]);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) h.a[s][i] = h.b[s][i] = 0.f;
        }
    }
}

// BACK: dx (and dgamma) from dy, else y from x.  V values per vector (1: any sizes and
// alignment), NS slots per lane, G lanes per head.
template <class T, int V, int NS, int G, bool INTER, bool BACK>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const __grid_constant__ RopeArgs p) {
    __shared__ float2 table[kRopeTable];
    __shared__ float red[BACK ? kRopeThreads / 32 * kRopeMaxD : 1];
    if (BACK) griddep_launch_dependents();
    constexpr int kGroups = kRopeThreads / G;
    const int lane = threadIdx.x % G, group = threadIdx.x / G;
    const int half = p.half, pairs = p.D / 2;
    RopeSlot<T, V, INTER> slot[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) slot[s].pair = (lane + s * G) * V;

    const int part0 = BACK && p.nparts > 1 && (int)blockIdx.x >= p.block0[1] ? 1 : 0;
    const int part1 = BACK ? part0 + 1 : p.nparts;
    const int block = BACK ? (int)blockIdx.x - p.block0[part0] : (int)blockIdx.x;
    const int blocks = BACK ? p.block0[part0 + 1] - p.block0[part0] : (int)gridDim.x;
    const float inv_d = 1.f / (float)p.D;
    float sum_a[NS][V], sum_b[NS][V];  // BACK: this lane's share of dgamma
    if constexpr (BACK) {
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int i = 0; i < V; ++i) sum_a[s][i] = sum_b[s][i] = 0.f;
    }

    for (int64_t t0 = (int64_t)block * p.tokens; t0 < p.T; t0 += (int64_t)blocks * p.tokens) {
        const int nt = (int)min((int64_t)p.tokens, p.T - t0);
        __syncthreads();  // the table is no longer read
        for (int i = threadIdx.x; i < nt * half; i += kRopeThreads) {
            const int t = i / half;
            table[i] = rope_turn(__ldg(p.pos + t0 + t), __ldg(p.freq + (i - t * half)), p.mscale);
        }
        __syncthreads();
        for (int part = part0; part < part1; ++part) {
            const RopeTensor &q = p.part[part];
            const bool norm = q.gamma != nullptr;
            float ga[NS][V], gb[NS][V];
            if (norm) {
#pragma unroll
                for (int s = 0; s < NS; ++s) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        ga[s][i] = slot[s].pair < pairs ? __ldg(q.gamma + slot[s].first(half) + i) : 0.f;
                        gb[s][i] = slot[s].pair < pairs ? __ldg(q.gamma + slot[s].second(half) + i) : 0.f;
                    }
                    slot[s].split(half, ga[s], gb[s]);
                }
            }
            const int n = nt * q.heads;
            RopeHead<V, NS> next, next_x;
            auto fetch = [&](int i) {
                const int t = i / q.heads, h = i - t * q.heads;
                if (BACK) rope_load<T, V, NS, INTER>(q.dy, (t0 + t) * q.dy_ld + h * q.dy_hs, slot, half, pairs, next);
                if (!BACK || norm)
                    rope_load<T, V, NS, INTER>(q.x, (t0 + t) * q.x_ld + h * q.x_hs, slot, half, pairs,
                                               BACK ? next_x : next);
            };
            if (group < n) fetch(group);
            // whole warps go round together (the reductions are theirs)
            for (int i0 = 0; i0 < n; i0 += kGroups) {
                const int i = i0 + group;
                const bool live = i < n;
                RopeHead<V, NS> z = next, x = next_x;
                if (i + kGroups < n) fetch(i + kGroups);
                const int t = i / q.heads, h = i - t * q.heads;
                const float2 *cs = table + t * half;
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    slot[s].split(half, z.a[s], z.b[s]);
                    if (BACK && norm) slot[s].split(half, x.a[s], x.b[s]);
                }
                if constexpr (!BACK) {
                    if (norm) {
                        float ss = 0.f;
#pragma unroll
                        for (int s = 0; s < NS; ++s)
#pragma unroll
                            for (int k = 0; k < V; ++k)
                                ss = fmaf(z.a[s][k], z.a[s][k], fmaf(z.b[s][k], z.b[s][k], ss));
#pragma unroll
                        for (int o = G / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
                        const float rstd = __frsqrt_rn(fmaf(ss, inv_d, p.eps));
#pragma unroll
                        for (int s = 0; s < NS; ++s)
#pragma unroll
                            for (int k = 0; k < V; ++k) {
                                z.a[s][k] *= rstd * ga[s][k];
                                z.b[s][k] *= rstd * gb[s][k];
                            }
                    }
                }
                if (live) {
#pragma unroll
                    for (int s = 0; s < NS; ++s)
                        if (slot[s].turns(half)) {
#pragma unroll
                            for (int k = 0; k < V; ++k) {
                                const float2 e = cs[slot[s].pair + k];
                                const float a = z.a[s][k], b = z.b[s][k], sn = BACK ? -e.y : e.y;
                                z.a[s][k] = fmaf(a, e.x, -(b * sn));
                                z.b[s][k] = fmaf(a, sn, b * e.x);
                            }
                        }
                }
                if constexpr (BACK) {
                    if (norm) {
                        float ss = 0.f, sg = 0.f;  // sums of x^2 and of g x
#pragma unroll
                        for (int s = 0; s < NS; ++s)
#pragma unroll
                            for (int k = 0; k < V; ++k) {
                                ss = fmaf(x.a[s][k], x.a[s][k], fmaf(x.b[s][k], x.b[s][k], ss));
                                sg = fmaf(z.a[s][k] * ga[s][k], x.a[s][k], fmaf(z.b[s][k] * gb[s][k], x.b[s][k], sg));
                            }
#pragma unroll
                        for (int o = G / 2; o > 0; o >>= 1) {
                            ss += __shfl_xor_sync(0xffffffffu, ss, o);
                            sg += __shfl_xor_sync(0xffffffffu, sg, o);
                        }
                        const float rstd = __frsqrt_rn(fmaf(ss, inv_d, p.eps)), m = sg * inv_d * rstd;
#pragma unroll
                        for (int s = 0; s < NS; ++s)
#pragma unroll
                            for (int k = 0; k < V; ++k) {
                                const float xa = x.a[s][k] * rstd, xb = x.b[s][k] * rstd;
                                if (live) {
                                    sum_a[s][k] = fmaf(z.a[s][k], xa, sum_a[s][k]);
                                    sum_b[s][k] = fmaf(z.b[s][k], xb, sum_b[s][k]);
                                }
                                z.a[s][k] = rstd * fmaf(-xa, m, z.a[s][k] * ga[s][k]);
                                z.b[s][k] = rstd * fmaf(-xb, m, z.b[s][k] * gb[s][k]);
                            }
                    }
                }
                if (live) {
                    T *y = static_cast<T *>(q.y) + (t0 + t) * q.y_ld + h * q.y_hs;
#pragma unroll
                    for (int s = 0; s < NS; ++s)
                        if (slot[s].pair < pairs) {
                            slot[s].join(half, z.a[s], z.b[s]);
                            rope_put(y + slot[s].first(half), z.a[s]);
                            rope_put(y + slot[s].second(half), z.b[s]);
                        }
                }
            }
        }
    }

    if constexpr (BACK) {
        if (!p.dgamma || !p.part[part0].gamma) return;
        // a warp's groups by exchanges, then the warps in order
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int o = 16; o >= G; o >>= 1) {
                    sum_a[s][k] += __shfl_xor_sync(0xffffffffu, sum_a[s][k], o);
                    sum_b[s][k] += __shfl_xor_sync(0xffffffffu, sum_b[s][k], o);
                }
        float *mine = red + threadIdx.x / 32 * p.D;
        if (threadIdx.x % 32 < G) {
#pragma unroll
            for (int s = 0; s < NS; ++s)
                if (slot[s].pair < pairs) {
                    slot[s].join(half, sum_a[s], sum_b[s]);
#pragma unroll
                    for (int k = 0; k < V; ++k) {
                        mine[slot[s].first(half) + k] = sum_a[s][k];
                        mine[slot[s].second(half) + k] = sum_b[s][k];
                    }
                }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < p.D; c += kRopeThreads) {
            float v = 0.f;
            for (int w = 0; w < kRopeThreads / 32; ++w) v += red[w * p.D + c];
            p.dgamma[(int64_t)blockIdx.x * p.D + c] = v;
        }
    }
}

// dgamma of each part from its blocks' sums, in their order: 8 strands of blocks per column.
struct RopeSum {
    const float *part;
    float *out[kRopeParts];
    int block0[kRopeParts + 1];
    int D;
};

__global__ void __launch_bounds__(256) rope_sum_kernel(const RopeSum a) {
    __shared__ float red[8][32];
    griddep_wait();
    const int q = blockIdx.y, c = blockIdx.x * 32 + threadIdx.x % 32, strand = threadIdx.x / 32;
    float v = 0.f;
    if (a.out[q] && c < a.D)
#pragma unroll 8
        for (int b = a.block0[q] + strand; b < a.block0[q + 1]; b += 8) v += __ldcg(a.part + (int64_t)b * a.D + c);
    red[strand][threadIdx.x % 32] = v;
    __syncthreads();
    if (strand == 0 && a.out[q] && c < a.D) {
        for (int s = 1; s < 8; ++s) v += red[s][threadIdx.x];
        a.out[q][c] = v;
    }
}

// ---------------------------------------------------------------------------

constexpr int kRopeMaxBlocks = 640;  // of the backward kernel, at most: four per SM

template <class T, bool INTER, bool BACK>
static const void *rope_pick(bool vec, int D) {
    constexpr int V = RopeVec<T>::n;
#define ATTT_ROPE(v, ns, g) reinterpret_cast<const void *>(&rope_kernel<T, v, ns, g, INTER, BACK>)
    if (vec) {
        const int slots = D / (2 * V);
        if (slots <= 4) return ATTT_ROPE(V, 1, 4);
        if (slots <= 8) return ATTT_ROPE(V, 1, 8);
        if (slots <= 16) return ATTT_ROPE(V, 1, 16);
        if (slots <= 32) return ATTT_ROPE(V, 1, 32);
        return ATTT_ROPE(V, 2, 32);
    }
    if (D <= 64) return ATTT_ROPE(1, 1, 32);
    if (D <= 128) return ATTT_ROPE(1, 2, 32);
    if (D <= 256) return ATTT_ROPE(1, 4, 32);
    return ATTT_ROPE(1, 8, 32);
#undef ATTT_ROPE
}

static bool rope_aligned(const void *p, int64_t ld, int64_t hs, size_t es) {
    return aligned16(p) && ld * (int64_t)es % 16 == 0 && hs * (int64_t)es % 16 == 0;
}

// Whether rows of D values at t ld + h hs are apart.
static bool rope_apart(int64_t T, int64_t heads, int64_t D, int64_t ld, int64_t hs) {
    if (T <= 1) return heads <= 1 || hs >= D;
    if (heads <= 1) return ld >= D;
    return (hs >= D && ld >= (heads - 1) * hs + D) || (ld >= D && hs >= (T - 1) * ld + D);
}

static attt_status rope_check(const attt_rope_part *parts, int nparts, const int32_t *d_pos, const uint64_t *d_freq,
                              int64_t T, int64_t D, int64_t rot, float eps, float mscale, int dtype, bool back) {
    if (!parts || nparts < 1 || nparts > kRopeParts || T < 0 || D < 2 || D % 2 != 0 || rot < 0 || rot > D ||
        rot % 2 != 0)
        return ATTT_ERR_INVALID_ARG;
    if (!(eps >= 0.f) || !std::isfinite(mscale) || (dtype != ATTT_BF16 && dtype != ATTT_F32)) return ATTT_ERR_INVALID_ARG;
    if ((rot > 0 && !d_freq) || (T > 0 && rot > 0 && !d_pos) || !aligned_to(4, d_pos) || !aligned_to(8, d_freq))
        return ATTT_ERR_INVALID_ARG;
    if (D > kRopeMaxD || T > (1ll << 30)) return ATTT_ERR_UNSUPPORTED;
    const size_t es = dtype == ATTT_BF16 ? 2 : 4;
    const int64_t most = 1ll << 36;
    for (int i = 0; i < nparts; ++i) {
        const attt_rope_part &q = parts[i];
        if (q.heads < 1 || !aligned_to(es, q.d_x, q.d_y, q.d_dy) || !aligned_to(4, q.d_gamma, q.d_dgamma))
            return ATTT_ERR_INVALID_ARG;
        if (q.heads > 1 << 16) return ATTT_ERR_UNSUPPORTED;
        if (T > 0 && (!q.d_y || (back && !q.d_dy) || ((!back || q.d_gamma) && !q.d_x))) return ATTT_ERR_INVALID_ARG;
        if (q.d_dgamma && !q.d_gamma) return ATTT_ERR_INVALID_ARG;
        for (int64_t v : {q.x_ld, q.x_hs, q.y_ld, q.y_hs, q.dy_ld, q.dy_hs})
            if (v < 0) return ATTT_ERR_INVALID_ARG;
            else if (v > most) return ATTT_ERR_UNSUPPORTED;
        if (!rope_apart(T, q.heads, D, q.y_ld, q.y_hs)) return ATTT_ERR_INVALID_ARG;
    }
    return ATTT_OK;
}

static attt_status rope_run(const attt_rope_part *parts, int nparts, const int32_t *d_pos, const uint64_t *d_freq,
                            int64_t T, int64_t D, int64_t rot, float eps, int interleaved, float mscale, int dtype,
                            bool back, float *ws, cudaStream_t stream) {
    int dev;
    attt_status st = current_device(&dev);
    if (st != ATTT_OK) return st;
    const size_t es = dtype == ATTT_BF16 ? 2 : 4;
    const int V = (int)(16 / es), sms = num_sms(dev);
    bool vec = D % (2 * V) == 0 && (interleaved ? rot % (2 * V) == 0 : (rot / 2) % V == 0);
    RopeArgs a{};
    int64_t heads = 0;
    bool sums = false;
    for (int i = 0; i < nparts; ++i) {
        const attt_rope_part &q = parts[i];
        a.part[i] = RopeTensor{q.d_x, q.d_dy, q.d_y, q.d_gamma, q.x_ld, q.x_hs, q.dy_ld, q.dy_hs, q.y_ld, q.y_hs,
                               q.heads};
        heads += q.heads;
        sums = sums || q.d_dgamma;
        vec = vec && rope_aligned(q.d_y, q.y_ld, q.y_hs, es);
        if (!back || q.d_gamma) vec = vec && rope_aligned(q.d_x, q.x_ld, q.x_hs, es);
        if (back) vec = vec && rope_aligned(q.d_dy, q.dy_ld, q.dy_hs, es);
    }
    a.pos = d_pos; a.freq = d_freq;
    a.T = T; a.nparts = nparts; a.D = (int)D; a.half = (int)(rot / 2);
    a.eps = eps; a.mscale = mscale;
    // tokens of a block at a time: some 128 heads, as many as its table holds, and no fewer blocks
    // than two per SM
    int64_t tokens = std::min<int64_t>(cdiv(128, heads), cdiv(T, 2 * sms));
    if (a.half > 0) tokens = std::min<int64_t>(tokens, kRopeTable / a.half);
    a.tokens = (int)std::max<int64_t>(tokens, 1);
    const int64_t tiles = cdiv(T, a.tokens);
    int blocks;
    if (!back) {
        blocks = (int)std::min<int64_t>(tiles, 1 << 30);
    } else {
        // every part has blocks of its own (their sums stay in registers), by its share of the heads
        const int all = std::min(4 * sms, kRopeMaxBlocks);
        for (int i = 0; i < nparts; ++i) {
            int64_t n = nparts == 1 ? all : std::max<int64_t>(1, all * parts[i].heads / heads);
            a.block0[i + 1] = a.block0[i] + (int)std::min<int64_t>(n, tiles);
        }
        blocks = a.block0[nparts];
        a.dgamma = sums ? ws : nullptr;
    }
    const void *kern;
    if (dtype == ATTT_BF16)
        kern = interleaved ? (back ? rope_pick<__nv_bfloat16, true, true>(vec, a.D)
                                   : rope_pick<__nv_bfloat16, true, false>(vec, a.D))
                           : (back ? rope_pick<__nv_bfloat16, false, true>(vec, a.D)
                                   : rope_pick<__nv_bfloat16, false, false>(vec, a.D));
    else
        kern = interleaved ? (back ? rope_pick<float, true, true>(vec, a.D) : rope_pick<float, true, false>(vec, a.D))
                           : (back ? rope_pick<float, false, true>(vec, a.D) : rope_pick<float, false, false>(vec, a.D));
    void *args[] = {&a};
    if (cudaLaunchKernel(kern, dim3((unsigned)blocks), dim3(kRopeThreads), args, 0, stream) != cudaSuccess)
        return ATTT_ERR_CUDA;
    count_launch();
    if (!back || !sums) return cudaGetLastError() == cudaSuccess ? ATTT_OK : ATTT_ERR_CUDA;
    RopeSum s{};
    s.part = ws;
    s.D = a.D;
    for (int i = 0; i < nparts; ++i) s.out[i] = parts[i].d_dgamma;
    for (int i = 0; i <= nparts; ++i) s.block0[i] = a.block0[i];
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)cdiv(D, 32), (unsigned)nparts);
    cfg.blockDim = dim3(256);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, rope_sum_kernel, s) != cudaSuccess) return ATTT_ERR_CUDA;
    count_launch();
    return cudaGetLastError() == cudaSuccess ? ATTT_OK : ATTT_ERR_CUDA;
}

}  // namespace attt

extern "C" {

attt_status attt_rope_frequencies(int64_t rot, double base, double factor, double context, double low, double high,
                                  uint64_t *host_freq) {
    if (rot < 2 || rot % 2 != 0 || rot > attt::kRopeMaxD || !host_freq) return ATTT_ERR_INVALID_ARG;
    if (!(base >= 1.0) || !std::isfinite(base) || !(factor >= 1.0) || !std::isfinite(factor) || !(context >= 0.0) ||
        !std::isfinite(context))
        return ATTT_ERR_INVALID_ARG;
    if (context > 0.0 && !(low >= 0.0 && high > low && std::isfinite(high))) return ATTT_ERR_INVALID_ARG;
    const double two_pi = 6.283185307179586476925;
    for (int64_t i = 0; i < rot / 2; ++i) {
        const double w = std::pow(base, -2.0 * (double)i / (double)rot);
        double keep = 0.0;  // the share of w that the stretched context leaves as it was
        if (context > 0.0) keep = std::min(1.0, std::max(0.0, (context * w / two_pi - low) / (high - low)));
        if (factor == 1.0) keep = 1.0;
        const double turns = (w * keep + w / factor * (1.0 - keep)) / two_pi;  // below 0.16
        host_freq[i] = (uint64_t)std::llround(turns * 9223372036854775808.0) * 2;
    }
    return ATTT_OK;
}

attt_status attt_rope_forward(const attt_rope_part *parts, int nparts, const int32_t *d_pos, const uint64_t *d_freq,
                              int64_t T, int64_t D, int64_t rot, float eps, int interleaved, float mscale, int dtype,
                              attt_stream stream) {
    ATTT_NVTX_RANGE();
    const attt_status st = attt::rope_check(parts, nparts, d_pos, d_freq, T, D, rot, eps, mscale, dtype, false);
    if (st != ATTT_OK || T == 0) return st;
    return attt::rope_run(parts, nparts, d_pos, d_freq, T, D, rot, eps, interleaved, mscale, dtype, false, nullptr,
                          stream);
}

size_t attt_rope_workspace_bytes(int64_t T, int64_t D) {
    if (T < 0 || T > (1ll << 30) || D < 2 || D % 2 != 0 || D > attt::kRopeMaxD) return 0;
    // a row per block; no part has more blocks than tokens, and a small part has one at least
    const int64_t rows = std::max<int64_t>(1, std::min<int64_t>(2 * T, attt::kRopeMaxBlocks + 1));
    return (size_t)attt::round_up(rows * D * (int64_t)sizeof(float), 256);
}

attt_status attt_rope_backward(const attt_rope_part *parts, int nparts, const int32_t *d_pos, const uint64_t *d_freq,
                               int64_t T, int64_t D, int64_t rot, float eps, int interleaved, float mscale, int dtype,
                               void *d_ws, size_t ws_bytes, attt_stream stream) {
    ATTT_NVTX_RANGE();
    using namespace attt;
    attt_status st = rope_check(parts, nparts, d_pos, d_freq, T, D, rot, eps, mscale, dtype, true);
    if (st != ATTT_OK) return st;
    bool sums = false;
    for (int i = 0; i < nparts; ++i) sums = sums || parts[i].d_dgamma;
    if (sums && (!d_ws || !aligned256(d_ws) || ws_bytes < attt_rope_workspace_bytes(T, D))) return ATTT_ERR_WORKSPACE;
    if (T > 0)
        return rope_run(parts, nparts, d_pos, d_freq, T, D, rot, eps, interleaved, mscale, dtype, true,
                        static_cast<float *>(d_ws), stream);
    if (!sums) return ATTT_OK;
    int dev;
    st = current_device(&dev);
    if (st != ATTT_OK) return st;
    for (int i = 0; i < nparts; ++i)
        if (parts[i].d_dgamma &&
            cudaMemsetAsync(parts[i].d_dgamma, 0, (size_t)D * sizeof(float), stream) != cudaSuccess)
            return ATTT_ERR_CUDA;
    return ATTT_OK;
}

}  // extern "C"

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
// a few lanes.  The vectors of the next heads stay in registers as loaded while some are
// worked on.  A block takes a run of tokens with all their heads and forms their cosines
// once, into a table whose order is that of the lanes' reads.
// Angles: w_i is held in turns per position as a 64-bit fraction; pos w_i modulo 2^64
// is then the exact fraction of a turn whatever the position (fp32 products are off by
// 0.06 radians at position 10^6), and a quarter turn is taken off before it goes to fp32.
// The inverse root of a head's mean is rsqrtf, 2 ulp: with the rounded root 2.3 M of 28.5 M instructions more.
// Measured: 8,192 tokens of 40 and 8 heads of 128, bf16 with norm, forward 35 to 38 us (5.3 to 5.7 TB/s, 79 to 85%
// of the copy rate: a chain of load, reduction over lanes, store per head is left), a pass among others 38.8; 2,048
// tokens of 28 and 4, backward with the norms' gradients 17.0 (floor 7.5: two launches, the table, the sums'
// way through memory are some 8 of it); 16 tokens forward 4.0.
#include <algorithm>
#include <cmath>

#include "attt_common.cuh"
#include "attt_host.h"

namespace attt {

constexpr int kRopeThreads = 256;
constexpr int kRopeParts = 2;
constexpr int kRopeMaxD = 512;
constexpr int kRopeTable = 2048;  // cosines and sines that a block holds
// Blocks per SM: what the registers of a thread's vectors leave room for.
constexpr int kRopeForward = 3, kRopeBack = 2;
constexpr int kRopeMaxBlocks = 160 * kRopeBack;  // of a part in the backward kernel, at most

struct RopeTensor {
    const void *x, *dy;
    void *y;  // forward: the result, backward: dx
    const float *gamma;
    int64_t x_ld, x_hs, dy_ld, dy_hs, y_ld, y_hs;
    int heads;
    uint32_t magic;  // of the division by heads (0: one head)
};

struct RopeArgs {
    RopeTensor part[kRopeParts];
    const int32_t *pos;
    const uint64_t *freq;
    int64_t T;
    int nparts, D, half;         // half: rot / 2
    int tokens;                  // that a table holds, at most
    int block0[kRopeParts + 1];  // backward: first block of each part
    float eps, mscale;
    float *dgamma;                // backward: [blocks, D] partial sums, nullptr: not wanted
};

// What a lane reads at once: a 16-byte vector or one value.
template <class T, int V>
struct RopeRead {
    using type = uint4;
};
template <class T>
struct RopeRead<T, 1> {
    using type = T;
};
template <class T>
struct RopeVec {  // values of a 16-byte vector
    static constexpr int n = 16 / sizeof(T);
};

__device__ __forceinline__ float rope_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float rope_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t rope_pack(float lo, float hi) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&b);
}

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
// (halves) or 2 p and 2 p + 1 (neighbours, INTER); the others do not.  V > 1: a slot is two vectors, at
// first() and second().
template <int V, bool INTER>
struct RopeSlot {
    int pair;  // its first pair; at least D / 2: nothing
    __device__ __forceinline__ bool turns(int half) const { return pair < half; }
    __device__ __forceinline__ bool apart(int half) const { return !INTER && pair < half; }
    __device__ __forceinline__ int first(int half) const { return apart(half) ? pair : 2 * pair; }
    __device__ __forceinline__ int second(int half) const { return apart(half) ? pair + half : 2 * pair + V; }
};

// The values of a slot's two vectors, in fp32, two to a register pair: a holds the first members
// of its pairs and b the second ones.  (Values that do not turn have no partner: without INTER
// they are a's and b's as they lie.)
template <class T, int V, bool INTER>
struct RopeValues {
    static constexpr int P = V > 1 ? V / 2 : 1;
    using R = typename RopeRead<T, V>::type;
    float2 a[P], b[P];

    __device__ __forceinline__ void unpack(const R &x, const R &y) {
        if constexpr (V == 1) {
            a[0] = make_float2((float)x, 0.f);
            b[0] = make_float2((float)y, 0.f);
        } else if constexpr (V == 8) {
            const uint32_t u[4] = {x.x, x.y, x.z, x.w}, v[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (INTER) {
                    const uint32_t w0 = i < 2 ? u[2 * i] : v[2 * i - 4], w1 = i < 2 ? u[2 * i + 1] : v[2 * i - 3];
                    a[i] = make_float2(rope_lo(w0), rope_lo(w1));
                    b[i] = make_float2(rope_hi(w0), rope_hi(w1));
                } else {
                    a[i] = make_float2(rope_lo(u[i]), rope_hi(u[i]));
                    b[i] = make_float2(rope_lo(v[i]), rope_hi(v[i]));
                }
            }
        } else {
            const float u[4] = {__uint_as_float(x.x), __uint_as_float(x.y), __uint_as_float(x.z), __uint_as_float(x.w)};
            const float v[4] = {__uint_as_float(y.x), __uint_as_float(y.y), __uint_as_float(y.z), __uint_as_float(y.w)};
            a[0] = INTER ? make_float2(u[0], u[2]) : make_float2(u[0], u[1]);
            b[0] = INTER ? make_float2(u[1], u[3]) : make_float2(v[0], v[1]);
            a[1] = INTER ? make_float2(v[0], v[2]) : make_float2(u[2], u[3]);
            b[1] = INTER ? make_float2(v[1], v[3]) : make_float2(v[2], v[3]);
        }
    }
    __device__ __forceinline__ void pack(R &x, R &y) const {
        if constexpr (V == 1) {
            x = (T)a[0].x;
            y = (T)b[0].x;
        } else if constexpr (V == 8) {
            uint32_t u[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (INTER) {
                    u[2 * i] = rope_pack(a[i].x, b[i].x);
                    u[2 * i + 1] = rope_pack(a[i].y, b[i].y);
                } else {
                    u[i] = rope_pack(a[i].x, a[i].y);
                    u[4 + i] = rope_pack(b[i].x, b[i].y);
                }
            }
            x = make_uint4(u[0], u[1], u[2], u[3]);
            y = make_uint4(u[4], u[5], u[6], u[7]);
        } else {
            float u[4], v[4];
            values(u, v);
            x = make_uint4(__float_as_uint(u[0]), __float_as_uint(u[1]), __float_as_uint(u[2]), __float_as_uint(u[3]));
            y = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        }
    }
    // the two vectors' values in their order, and back
    __device__ __forceinline__ void values(float (&u)[V], float (&v)[V]) const {
        if constexpr (V == 1) {
            u[0] = a[0].x;
            v[0] = b[0].x;
        } else {
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                if (INTER) {
                    float *w = i < V / 4 ? &u[4 * i] : &v[4 * i - V];
                    w[0] = a[i].x; w[1] = b[i].x; w[2] = a[i].y; w[3] = b[i].y;
                } else {
                    u[2 * i] = a[i].x; u[2 * i + 1] = a[i].y;
                    v[2 * i] = b[i].x; v[2 * i + 1] = b[i].y;
                }
            }
        }
    }
    __device__ __forceinline__ void from(const float (&u)[V], const float (&v)[V]) {
        if constexpr (V == 1) {
            a[0] = make_float2(u[0], 0.f);
            b[0] = make_float2(v[0], 0.f);
        } else {
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                if (INTER) {
                    const float *w = i < V / 4 ? &u[4 * i] : &v[4 * i - V];
                    a[i] = make_float2(w[0], w[2]);
                    b[i] = make_float2(w[1], w[3]);
                } else {
                    a[i] = make_float2(u[2 * i], u[2 * i + 1]);
                    b[i] = make_float2(v[2 * i], v[2 * i + 1]);
                }
            }
        }
    }
};

__device__ __forceinline__ float2 rope_mul(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 rope_fma(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }

// A lane's vectors of a head, as loaded.
template <class T, int V, int NS>
struct RopeHead {
    typename RopeRead<T, V>::type a[NS], b[NS];
};

template <class T, int V, int NS, bool INTER>
__device__ __forceinline__ void rope_load(const void *base, int64_t off, const RopeSlot<V, INTER> (&slot)[NS], int half,
                                          int pairs, RopeHead<T, V, NS> &h) {
    using R = typename RopeRead<T, V>::type;
    const T *p = static_cast<const T *>(base) + off;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        h.a[s] = h.b[s] = R{};
        if (slot[s].pair < pairs) {
            h.a[s] = *reinterpret_cast<const R *>(p + slot[s].first(half));
            h.b[s] = *reinterpret_cast<const R *>(p + slot[s].second(half));
        }
    }
}

// A token's table: cosine and sine of every pair, V > 1: of two neighbouring pairs as (cos, cos, sin, sin), those
// that the lanes read at once side by side.
template <int V>
__device__ __forceinline__ void rope_note(float *row, int i, int half, float2 e) {
    if (V == 1) {
        reinterpret_cast<float2 *>(row)[i] = e;
    } else {
        float *at = row + ((i % V) / 2 * (half / V) + i / V) * 4 + (i & 1);
        at[0] = e.x;
        at[2] = e.y;
    }
}

// BACK: dx (and dgamma) from dy, else y from x.  V values per vector (1: any sizes and
// alignment), NS slots per lane, G lanes per head.
template <class T, int V, int NS, int G, bool INTER, bool BACK>
__global__ void __launch_bounds__(kRopeThreads, NS > 1 && NS * V >= 8 ? 1 : BACK ? kRopeBack : kRopeForward)
    rope_kernel(const __grid_constant__ RopeArgs p) {
    __shared__ alignas(16) float table[2 * kRopeTable];
    __shared__ float red[BACK ? kRopeThreads / 32 * kRopeMaxD : 1];
    if (BACK) griddep_launch_dependents();
    constexpr int kGroups = kRopeThreads / G;
    // heads of a lane at a time: two where its registers hold them, one backward (2,048 tokens of 32
    // heads of 128: 17.6 us, two 19.6)
    constexpr int U = BACK || (NS > 1 && (V > 1 || NS >= 4)) ? 1 : 2;
    const int lane = threadIdx.x % G, group = threadIdx.x / G;
    const int half = p.half, pairs = p.D / 2;
    RopeSlot<V, INTER> slot[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) slot[s].pair = (lane + s * G) * V;

    const int part0 = BACK && p.nparts > 1 && (int)blockIdx.x >= p.block0[1] ? 1 : 0;
    const int part1 = BACK ? part0 + 1 : p.nparts;
    const int block = BACK ? (int)blockIdx.x - p.block0[part0] : (int)blockIdx.x;
    const int blocks = BACK ? p.block0[part0 + 1] - p.block0[part0] : (int)gridDim.x;
    const int64_t begin = p.T * block / blocks, end = p.T * (block + 1) / blocks;  // this block's tokens
    const float inv_d = 1.f / (float)p.D;
    using Values = RopeValues<T, V, INTER>;
    constexpr int P = Values::P;
    Values sum[NS];  // BACK: this lane's share of dgamma
    if constexpr (BACK) {
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int i = 0; i < P; ++i) sum[s].a[i] = sum[s].b[i] = make_float2(0.f, 0.f);
    }

    for (int64_t t0 = begin; t0 < end; t0 += p.tokens) {
        const int nt = (int)min((int64_t)p.tokens, end - t0);
        bool filled = false;
        for (int part = part0; part < part1; ++part) {
            const RopeTensor &q = p.part[part];
            const bool norm = q.gamma != nullptr;
            const int n = nt * q.heads;
            RopeHead<T, V, NS> next[U], next_x;
            auto fetch = [&](int i0) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int i = i0 + u * kGroups;
                    if (i < n) {
                        const int t = q.magic ? __umulhi((uint32_t)i, q.magic) : i, h = i - t * q.heads;
                        rope_load<T, V, NS, INTER>(BACK ? q.dy : q.x,
                                                   BACK ? (t0 + t) * q.dy_ld + h * q.dy_hs : (t0 + t) * q.x_ld + h * q.x_hs,
                                                   slot, half, pairs, next[u]);
                        if (BACK && norm)
                            rope_load<T, V, NS, INTER>(q.x, (t0 + t) * q.x_ld + h * q.x_hs, slot, half, pairs, next_x);
                    }
                }
            };
            fetch(group);
            if (!filled) {  // with the first loads under way
                __syncthreads();  // the table is no longer read
                for (int i = threadIdx.x; i < nt * half; i += kRopeThreads) {
                    const int t = i / half, k = i - t * half;
                    float2 e = rope_turn(__ldg(p.pos + t0 + t), __ldg(p.freq + k), p.mscale);
                    if (BACK) e.y = -e.y;
                    rope_note<V>(table + 2 * t * half, k, half, e);
                }
                __syncthreads();
                filled = true;
            }
            Values gamma[NS];
            if (norm) {
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    float u[V], v[V];
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        u[i] = slot[s].pair < pairs ? __ldg(q.gamma + slot[s].first(half) + i) : 0.f;
                        v[i] = slot[s].pair < pairs ? __ldg(q.gamma + slot[s].second(half) + i) : 0.f;
                    }
                    gamma[s].from(u, v);
                }
            }
            // whole warps go round together (the reductions are theirs)
            for (int i0 = 0; i0 < n; i0 += U * kGroups) {
                RopeHead<T, V, NS> head[U], head_x;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    head[u] = next[u];
                    if (BACK) head_x = next_x;
                }
                fetch(i0 + group + U * kGroups);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int i = i0 + group + u * kGroups;
                    const bool live = i < n;
                    const int t = q.magic ? __umulhi((uint32_t)i, q.magic) : i, h = i - t * q.heads;
                    Values z[NS];
#pragma unroll
                    for (int s = 0; s < NS; ++s) z[s].unpack(head[u].a[s], head[u].b[s]);
                    float2 rstd = make_float2(1.f, 1.f);
                    if (!BACK && norm) {
                        float2 ss = make_float2(0.f, 0.f);
#pragma unroll
                        for (int s = 0; s < NS; ++s)
#pragma unroll
                            for (int k = 0; k < P; ++k) {
                                ss = rope_fma(z[s].a[k], z[s].a[k], rope_fma(z[s].b[k], z[s].b[k], ss));
                                z[s].a[k] = rope_mul(z[s].a[k], gamma[s].a[k]);
                                z[s].b[k] = rope_mul(z[s].b[k], gamma[s].b[k]);
                            }
                        float sum2 = ss.x + ss.y;
#pragma unroll
                        for (int o = G / 2; o > 0; o >>= 1) sum2 += __shfl_xor_sync(0xffffffffu, sum2, o);
                        rstd.x = rstd.y = rsqrtf(fmaf(sum2, inv_d, p.eps));
                    }
                    if (live) {
#pragma unroll
                        for (int s = 0; s < NS; ++s)
                            if (slot[s].turns(half)) {
                                const float *cs = table + 2 * t * half + (V == 1 ? 2 : 4) * (slot[s].pair / V);
#pragma unroll
                                for (int k = 0; k < P; ++k) {
                                    float2 c, sn;
                                    if constexpr (V == 1) {
                                        const float2 f = *reinterpret_cast<const float2 *>(cs);
                                        c = make_float2(f.x, 0.f);
                                        sn = make_float2(f.y, 0.f);
                                    } else {
                                        const float4 f = *reinterpret_cast<const float4 *>(cs + 4 * k * (half / V));
                                        c = make_float2(f.x, f.y);
                                        sn = make_float2(f.z, f.w);
                                    }
                                    const float2 va = z[s].a[k], vb = z[s].b[k];
                                    // (a pair has no negation of its own; times -1 is one instruction, not two)
                                    z[s].a[k] = rope_fma(rope_mul(vb, sn), make_float2(-1.f, -1.f), rope_mul(va, c));
                                    z[s].b[k] = rope_fma(va, sn, rope_mul(vb, c));
                                }
                            }
                    }
                    if (!BACK && norm) {
#pragma unroll
                        for (int s = 0; s < NS; ++s)
#pragma unroll
                            for (int k = 0; k < P; ++k) {
                                z[s].a[k] = rope_mul(z[s].a[k], rstd);
                                z[s].b[k] = rope_mul(z[s].b[k], rstd);
                            }
                    }
                    if constexpr (BACK) {
                        if (norm) {
                            Values x[NS];
#pragma unroll
                            for (int s = 0; s < NS; ++s) x[s].unpack(head_x.a[s], head_x.b[s]);
                            float2 ss = make_float2(0.f, 0.f), sg = ss;  // sums of x^2 and of g x
#pragma unroll
                            for (int s = 0; s < NS; ++s)
#pragma unroll
                                for (int k = 0; k < P; ++k) {
                                    ss = rope_fma(x[s].a[k], x[s].a[k], rope_fma(x[s].b[k], x[s].b[k], ss));
                                    sg = rope_fma(rope_mul(z[s].a[k], gamma[s].a[k]), x[s].a[k], sg);
                                    sg = rope_fma(rope_mul(z[s].b[k], gamma[s].b[k]), x[s].b[k], sg);
                                }
                            float sum2 = ss.x + ss.y, sumg = sg.x + sg.y;
#pragma unroll
                            for (int o = G / 2; o > 0; o >>= 1) {
                                sum2 += __shfl_xor_sync(0xffffffffu, sum2, o);
                                sumg += __shfl_xor_sync(0xffffffffu, sumg, o);
                            }
                            rstd.x = rstd.y = rsqrtf(fmaf(sum2, inv_d, p.eps));
                            const float2 m = make_float2(-sumg * inv_d * rstd.x, -sumg * inv_d * rstd.x);
#pragma unroll
                            for (int s = 0; s < NS; ++s)
#pragma unroll
                                for (int k = 0; k < P; ++k) {
                                    const float2 ha = rope_mul(x[s].a[k], rstd), hb = rope_mul(x[s].b[k], rstd);
                                    if (live) {
                                        sum[s].a[k] = rope_fma(z[s].a[k], ha, sum[s].a[k]);
                                        sum[s].b[k] = rope_fma(z[s].b[k], hb, sum[s].b[k]);
                                    }
                                    z[s].a[k] = rope_mul(rstd, rope_fma(ha, m, rope_mul(z[s].a[k], gamma[s].a[k])));
                                    z[s].b[k] = rope_mul(rstd, rope_fma(hb, m, rope_mul(z[s].b[k], gamma[s].b[k])));
                                }
                        }
                    }
                    if (live) {
                        using R = typename RopeRead<T, V>::type;
                        T *y = static_cast<T *>(q.y) + (t0 + t) * q.y_ld + h * q.y_hs;
#pragma unroll
                        for (int s = 0; s < NS; ++s)
                            if (slot[s].pair < pairs) {
                                R u0, u1;
                                z[s].pack(u0, u1);
                                *reinterpret_cast<R *>(y + slot[s].first(half)) = u0;
                                *reinterpret_cast<R *>(y + slot[s].second(half)) = u1;
                            }
                    }
                }
            }
        }
    }

    if constexpr (BACK) {
        if (!p.dgamma || !p.part[part0].gamma) return;
        // a warp's groups by exchanges, then the warps in order
        float *mine = red + threadIdx.x / 32 * p.D;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            float u[V], v[V];
            sum[s].values(u, v);
#pragma unroll
            for (int k = 0; k < V; ++k) {
#pragma unroll
                for (int o = 16; o >= G; o >>= 1) {
                    u[k] += __shfl_xor_sync(0xffffffffu, u[k], o);
                    v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
                }
                if (threadIdx.x % 32 < G && slot[s].pair < pairs) {
                    mine[slot[s].first(half) + k] = u[k];
                    mine[slot[s].second(half) + k] = v[k];
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

// dgamma of each part from its blocks' sums: 32 strands of blocks per column, each in the
// blocks' order, then the strands in theirs.
struct RopeSum {
    const float *part;
    float *out[kRopeParts];
    int block0[kRopeParts + 1];
    int D;
};

__global__ void __launch_bounds__(1024) rope_sum_kernel(const RopeSum a) {
    __shared__ float red[32][33];
    griddep_wait();
    const int q = blockIdx.y, x = threadIdx.x % 32, c = blockIdx.x * 32 + x, strand = threadIdx.x / 32;
    if (!a.out[q]) return;
    float v = 0.f;
    if (c < a.D) {
        const int b0 = a.block0[q] + strand, b1 = a.block0[q + 1];
        float w[kRopeMaxBlocks / 32];  // all loads at once: their latency is what this kernel costs
#pragma unroll
        for (int k = 0; k < kRopeMaxBlocks / 32; ++k)
            w[k] = b0 + 32 * k < b1 ? __ldcg(a.part + (int64_t)(b0 + 32 * k) * a.D + c) : 0.f;
#pragma unroll
        for (int k = 0; k < kRopeMaxBlocks / 32; ++k) v += w[k];
    }
    red[strand][x] = v;
    __syncthreads();
    v = red[x][strand];  // a warp per column
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (x == 0 && blockIdx.x * 32 + strand < a.D) a.out[q][blockIdx.x * 32 + strand] = v;
}

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

// The bytes of a tensor's heads: `outer` runs `pitch` bytes apart, of `inner` rows `step` apart, from `at` on.
// Runs and rows follow one another without sharing bytes; heads that do share some (operands with
// strides of 0 or below D) are taken as one row from the first to the last byte.
struct RopeBytes {
    int64_t at, outer, pitch, inner, step, row;
    int64_t run() const { return (inner - 1) * step + row; }
    int64_t end() const { return at + (outer - 1) * pitch + run(); }
};

static RopeBytes rope_bytes(const void *p, int64_t T, int64_t heads, int64_t D, int64_t ld, int64_t hs, int64_t es) {
    const int64_t row = D * es, at = (int64_t)reinterpret_cast<uintptr_t>(p);
    if (T == 1 || ld == 0) T = 1, ld = 0;
    if (heads == 1 || hs == 0) heads = 1, hs = 0;
    ld *= es; hs *= es;
    if ((heads == 1 || hs >= row) && (T == 1 || ld >= (heads - 1) * hs + row)) return {at, T, ld, heads, hs, row};
    if (ld >= row && hs >= (T - 1) * ld + row) return {at, heads, hs, T, ld, row};
    return {at, 1, 0, 1, 0, (T - 1) * ld + (heads - 1) * hs + row};
}

// The two whole numbers c for which off - c pitch lies within a pitch of 0: the first of them.
static int64_t rope_floor(int64_t off, int64_t pitch) {
    return off >= 0 ? off / pitch : -((-off + pitch - 1) / pitch);
}

// Whether rows of a run of a and of one of b share a byte where b's begins `off` bytes behind a's.
static bool rope_runs_meet(const RopeBytes &a, const RopeBytes &b, int64_t off) {
    if (off >= a.run() || off + b.run() <= 0) return false;
    if (a.inner > 1 && b.inner > 1 && a.step == b.step) {  // row j of b by a's rows j + c, for every j
        const int64_t k = rope_floor(off, a.step);
        for (int64_t c = k; c <= k + 1; ++c)
            if (c < a.inner && c > -b.inner && off - c * a.step < a.row && off - c * a.step + b.row > 0) return true;
        return false;
    }
    for (int64_t j = 0; j < b.inner; ++j) {
        const int64_t x = off + j * b.step;  // b's row j; a's first row that ends behind its begin
        if (x + b.row <= 0 || x >= a.run()) continue;
        const int64_t i = x < a.row ? 0 : (x - a.row) / std::max<int64_t>(a.step, 1) + 1;
        if (i < a.inner && i * a.step < x + b.row) return true;
    }
    return false;
}

static bool rope_meet(const RopeBytes &a, const RopeBytes &b) {
    if (a.end() <= b.at || b.end() <= a.at) return false;
    // Runs of one pitch (q and k in the rows of one projection): run j of b by a's runs j + c, for every j.
    if (a.outer > 1 && b.outer > 1 && a.pitch == b.pitch) {
        const int64_t diff = b.at - a.at, k = rope_floor(diff, a.pitch);
        for (int64_t c = k; c <= k + 1; ++c)
            if (c < a.outer && c > -b.outer && rope_runs_meet(a, b, diff - c * a.pitch)) return true;
        return false;
    }
    const int64_t pitch = std::max<int64_t>(a.pitch, 1);
    for (int64_t j = 0; j < b.outer; ++j) {
        const int64_t x = b.at + j * b.pitch - a.at;
        if (x + b.run() <= 0) continue;
        for (int64_t i = x < a.run() ? 0 : (x - a.run()) / pitch + 1; i < a.outer && i * a.pitch < x + b.run(); ++i)
            if (rope_runs_meet(a, b, x - i * a.pitch)) return true;
    }
    return false;
}

// Whether no result shares a byte with the other one, or with an operand that is not the same
// heads: blocks and warps read and write at times of their own.
static bool rope_results_apart(const attt_rope_part *parts, int nparts, int64_t T, int64_t D, size_t es, bool back) {
    RopeBytes y[kRopeParts], in[kRopeParts][2];
    bool has[kRopeParts][2];
    for (int i = 0; i < nparts; ++i) {
        const attt_rope_part &q = parts[i];
        y[i] = rope_bytes(q.d_y, T, q.heads, D, q.y_ld, q.y_hs, es);
        has[i][0] = !back || q.d_gamma;
        has[i][1] = back;
        in[i][0] = rope_bytes(q.d_x, T, q.heads, D, q.x_ld, q.x_hs, es);
        in[i][1] = rope_bytes(q.d_dy, T, q.heads, D, q.dy_ld, q.dy_hs, es);
    }
    for (int i = 0; i < nparts; ++i) {
        for (int j = 0; j < nparts; ++j)
            for (int k = 0; k < 2; ++k) {
                if (!has[j][k]) continue;
                const RopeBytes &a = y[i], &b = in[j][k];
                const bool same = i == j && a.at == b.at && a.outer == b.outer && a.inner == b.inner &&
                                  a.pitch == b.pitch && a.step == b.step;
                if (!same && rope_meet(a, b)) return false;
            }
        if (i > 0 && rope_meet(y[0], y[i])) return false;
    }
    return !(nparts == 2 && share_a_byte({parts[0].d_dgamma, 4 * D}, {parts[1].d_dgamma, 4 * D}));
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
        for (int64_t ld : {q.x_ld, q.y_ld, q.dy_ld})  // farther than addresses reach
            if ((double)ld * (double)T > 0x1p48) return ATTT_ERR_UNSUPPORTED;
        if (!rope_apart(T, q.heads, D, q.y_ld, q.y_hs)) return ATTT_ERR_INVALID_ARG;
    }
    return T == 0 || rope_results_apart(parts, nparts, T, D, es, back) ? ATTT_OK : ATTT_ERR_INVALID_ARG;
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
    a.tokens = a.half > 0 ? std::max(1, kRopeTable / a.half) : 1 << 20;
    // a block for some 32 heads, as many as are resident together; a run of tokens each
    for (int i = 0; i < nparts; ++i) {
        const int64_t h = a.part[i].heads;
        a.part[i].magic = h > 1 ? (uint32_t)(((1ull << 32) + h - 1) / h) : 0;
        a.tokens = (int)std::min<int64_t>(a.tokens, std::max<int64_t>(1, 65536 / h));  // the division's range
    }
    int blocks;
    if (!back) {
        blocks = (int)std::min({T, cdiv(T * heads, 32), (int64_t)sms * kRopeForward});
    } else {
        // every part has blocks of its own (their sums stay in registers), by its share of the heads
        const int all = std::min(kRopeBack * sms, kRopeMaxBlocks);
        for (int i = 0; i < nparts; ++i) {
            const int64_t h = parts[i].heads;
            const int64_t n = nparts == 1 ? all : std::max<int64_t>(1, all * h / heads);
            a.block0[i + 1] = a.block0[i] + (int)std::min({T, cdiv(T * h, 32), n});
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
    cfg.blockDim = dim3(1024);
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

namespace attt {

// The table of attt_rope_frequencies, or of attt_rope_frequencies_by_index.
static attt_status rope_table(int64_t rot, double base, double factor, double context, double low, double high,
                              bool by_index, uint64_t *host_freq) {
    if (rot < 2 || rot % 2 != 0 || rot > kRopeMaxD || !host_freq) return ATTT_ERR_INVALID_ARG;
    if (!(base >= 1.0) || !std::isfinite(base) || !(factor >= 1.0) || !std::isfinite(factor) || !(context >= 0.0) ||
        !std::isfinite(context))
        return ATTT_ERR_INVALID_ARG;
    if (context > 0.0 && !(low >= 0.0 && high > low && std::isfinite(high))) return ATTT_ERR_INVALID_ARG;
    const double two_pi = 6.283185307179586476925;
    double i0 = 0.0, i1 = 0.0;  // by_index: w_i is kept up to i0, divided from i1 on
    if (by_index) {
        if (!(context > 0.0 && low > 0.0 && base > 1.0)) return ATTT_ERR_INVALID_ARG;
        // the (fractional) pair that turns n times over the context
        auto pair = [&](double n) { return (double)rot * std::log(context / (two_pi * n)) / (2.0 * std::log(base)); };
        i0 = std::max(0.0, std::floor(pair(high)));
        i1 = std::min((double)(rot - 1), std::ceil(pair(low)));
        if (!(i1 > i0)) return ATTT_ERR_INVALID_ARG;
    }
    for (int64_t i = 0; i < rot / 2; ++i) {
        const double w = std::pow(base, -2.0 * (double)i / (double)rot);
        double keep = 0.0;  // the share of w that the stretched context leaves as it was
        if (by_index) keep = std::min(1.0, std::max(0.0, (i1 - (double)i) / (i1 - i0)));
        else if (context > 0.0) keep = std::min(1.0, std::max(0.0, (context * w / two_pi - low) / (high - low)));
        if (factor == 1.0) keep = 1.0;
        const double turns = (w * keep + w / factor * (1.0 - keep)) / two_pi;  // below 0.16
        host_freq[i] = (uint64_t)std::llround(turns * 9223372036854775808.0) * 2;
    }
    return ATTT_OK;
}

}  // namespace attt

extern "C" {

attt_status attt_rope_frequencies(int64_t rot, double base, double factor, double context, double low, double high,
                                  uint64_t *host_freq) {
    return attt::rope_table(rot, base, factor, context, low, high, false, host_freq);
}

attt_status attt_rope_frequencies_by_index(int64_t rot, double base, double factor, double context, double low,
                                           double high, uint64_t *host_freq) {
    return attt::rope_table(rot, base, factor, context, low, high, true, host_freq);
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

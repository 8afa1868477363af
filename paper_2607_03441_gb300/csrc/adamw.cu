// adamw.cu -- the AdamW step of many tensors in one launch, with moments in 32 bits
// or in 8.
//
//   m <- b1 m + (1 - b1) g;  v <- b2 v + (1 - b2) g^2
//   p <- p (1 - lr wd) - (lr / (1 - b1^t)) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
// with every operation rounded on its own, as attt_lora_adamw_step: with moments in 32
// bits the two give the same bits (in 8 bits p's quotients are approximate, m and v are not).
//
// Moments in 8 bits: blocks of 256 values with one fp32 scale each.  A code is a number of 4
// exponent bits and k mantissa bits (exponent 0: without the leading one): 0 to 2 - 2^-k in
// 2^-14 steps of a relative 2^-k; m has a sign and k = 3, and in the place of v its root
// with k = 4 (the range of v would be twice as many powers of two).  The scale makes the
// block's largest value the largest code.  What a code cuts off rounds up with the probability
// of its size: with b2 = 0.999 a step without gradient takes 1/2000 of sqrt(v), a
// sixtieth of the distance to the next code or less, and rounding to nearest would never
// let it fall.  The random bits are a hash of (seed, tensor, index): a step can be repeated.
// A root above 0 is never stored as 0 but as the smallest code at least: beside values 2^18 times
// its size it would be 0 while its m still rounds up to a code now and then, and the step would divide
// that m by little more than sqrt(1 - b2) |g| (gradients of 1 and 2^-20 in a block: steps of 430 lr).
// The step itself uses the moments before they are rounded.
//
// Bound: HBM bytes, 30 a value (8 bits: 18 and 16 per block).  A warp takes a run of blocks of 256
// values, a lane two runs of four of each (16-byte vectors that lie side by side); largest values by
// one reduction over the warp.  The next block's lines are asked into L2 while one is worked on.
// Measured: 112 tensors, 5.0 M values, 32 bits 30.7 us (floor 22.4: 4.9 TB/s with a start and an
// end of some 4 us); 512 tensors, 134 M values, in 8 bits with the moments read back as fp32 662 us (floor 533:
// 5.3 TB/s, the hash and the codes' arithmetic beside the bytes).
#include <algorithm>
#include <cmath>
#include <cstring>
#include <memory>
#include <new>
#include <type_traits>
#include <utility>
#include <vector>

#include "attt_common.cuh"
#include "attt_host.h"

namespace attt {

constexpr int kAdamBlock = 256;  // values of a scale, and of a warp's step
constexpr int kAdamWarps = 4;
constexpr int kAdamStep8 = 5, kAdamStep32 = 5, kAdamRead = 10;  // blocks per SM
constexpr int kAdamAhead = 1;  // blocks of a warp that are asked for before their turn
constexpr float kAdamTiny = 0x1p-100f;  // blocks without a value of this size are 0

struct AdamTensor {
    float *p;
    const float *g;
    void *m, *v;  // fp32 or codes
    float *ms, *vs;
    __nv_bfloat16 *p16;
    int64_t n;
    int64_t block0;  // first of its blocks among all tensors'
    int vec;         // its vectors can be read whole
    uint32_t id;     // its number in the call, for the random bits
};

struct AdamArgs {
    const AdamTensor *tensors;
    const int64_t *first;  // first block of each
    int count;
    int64_t blocks;
    float decay, b1, one_b1, b2, one_b2, step_size, bc2_sqrt, inv_bc2, eps;
    uint32_t seed_lo, seed_hi;
    float *m32, *v32;  // adam_read_kernel
};

// A bijection of 32-bit numbers that spreads every bit over all: two multiplications by odd
// numbers (the digits of sqrt(2) and sqrt(3)), and halves folded onto each other.
__host__ __device__ __forceinline__ uint32_t adam_mix(uint32_t x) {
    x ^= x >> 16;
    x *= 0xB504F333u;
    x ^= x >> 15;
    x *= 0xDDB3D743u;
    return x ^ (x >> 16);
}

__device__ __forceinline__ float2 adam_two(float v) { return make_float2(v, v); }

// b x + c y with each product and the sum rounded on its own.  (Pairs, mul and add of f32x2, are
// contracted to one rounding less even as .rn: measured by scales a last bit off.)
__device__ __forceinline__ float adam_blend(float b, float x, float c, float y) {
    return __fadd_rn(__fmul_rn(b, x), __fmul_rn(c, y));
}

// Codes as fp32: their exponent and mantissa bits, at those of an fp32, are the code's value times
// 2^-112, exponent 0 among fp32's own numbers without a leading one.

// The value of byte j of w, a code (SIGN: with its sign in bit 7).
template <int K, bool SIGN>
__device__ __forceinline__ float adam_decode(uint32_t w, int j) {
    constexpr int up = 23 - K;
    const uint32_t c = (up >= 8 * j ? w << (up - 8 * j) : w >> (8 * j - up)) & ((16u << K) - 1u) << up;
    const uint32_t s = SIGN ? (w << (24 - 8 * j)) & 0x80000000u : 0u;
    return __uint_as_float(c | s) * 0x1p112f;
}

// The code of a in [0, 2 - 2^-K]; rnd: 23 - K random bits.
template <int K>
__device__ __forceinline__ uint32_t adam_encode(float a, uint32_t rnd) {
    return min((__float_as_uint(__fmul_rz(a, 0x1p-112f)) + rnd) >> (23 - K), (16u << K) - 1u);
}

// A block's scale and its inverse from the bits of its largest size (a NaN's are the largest).
template <int K>
__device__ __forceinline__ float adam_scale(uint32_t top_bits, float &inv) {
    const float top = __uint_as_float(top_bits);
    inv = 0.f;
    if (top_bits >= 0x7f800000u) return __uint_as_float(0x7fffffffu);
    if (!(top >= kAdamTiny)) return 0.f;
    const float s = __fmul_rn(top, (float)(1.0 / (2.0 - 1.0 / (1 << K))));
    inv = __fdiv_rn(1.f, s);
    return s;
}

// The tensor that has block b, the last one whose first block is not after it: 32 candidates at a
// time, one per lane (a search by halves is a chain of seven loads for 112 tensors, 4 us of a
// step of 33).
__device__ __forceinline__ int adam_find(const int64_t *first, int count, int64_t b, int lane) {
    int lo = 0, n = count;  // it is among [lo, lo + n)
    while (n > 1) {
        const int step = (n + 31) / 32, i = lane * step;
        const bool before = i < n && __ldg(first + lo + i) <= b;  // (lane 0's is)
        const int k = __popc(__ballot_sync(0xffffffffu, before)) - 1;
        lo += k * step;
        n = min(step, n - k * step);
    }
    return lo;
}

template <class T, int N>
struct alignas(sizeof(T) * N) AdamRun {
    T v[N];
};

// Four neighbouring values from i on.  Not WHOLE: value by value, those from n on as zeros.
template <bool WHOLE, class T>
__device__ __forceinline__ AdamRun<T, 4> adam_load(const T *p, int64_t i, int64_t n) {
    AdamRun<T, 4> r{};
    if constexpr (WHOLE) {
        r = *reinterpret_cast<const AdamRun<T, 4> *>(p + i);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + k < n) r.v[k] = p[i + k];
    }
    return r;
}
template <bool WHOLE, class T>
__device__ __forceinline__ void adam_store(T *p, int64_t i, int64_t n, const AdamRun<T, 4> &r) {
    if constexpr (WHOLE) {
        *reinterpret_cast<AdamRun<T, 4> *>(p + i) = r;
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + k < n) p[i + k] = r.v[k];
    }
}

__device__ __forceinline__ uint32_t adam_word(const AdamRun<uint8_t, 4> &r) { return *reinterpret_cast<const uint32_t *>(&r); }

// The step of one block of a tensor, its block `b`, by a warp.  key: BITS8, the random bits' of its first value.
template <bool BITS8, bool WHOLE>
__device__ __forceinline__ void adam_block(const AdamArgs &a, const AdamTensor &t, int64_t b, uint32_t key, int lane) {
    using State = typename std::conditional<BITS8, uint8_t, float>::type;
    const int64_t i0 = b * kAdamBlock + 4 * lane;
    AdamRun<float, 4> p[2], g[2];
    AdamRun<State, 4> m[2], v[2];
    AdamRun<__nv_bfloat16, 4> h[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int64_t i = i0 + 128 * j;
        p[j] = adam_load<WHOLE>(t.p, i, t.n);
        g[j] = adam_load<WHOLE>(t.g, i, t.n);
        m[j] = adam_load<WHOLE>(static_cast<const State *>(t.m), i, t.n);
        v[j] = adam_load<WHOLE>(static_cast<const State *>(t.v), i, t.n);
    }
    if constexpr (BITS8) {
        const float sm = t.ms[b], sv = t.vs[b];
        float2 mn[4], rn[4];
        uint32_t top_m = 0u, top_r = 0u;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t cm = adam_word(m[j]), cv = adam_word(v[j]);
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                const float2 m0 = __fmul2_rn(make_float2(adam_decode<3, true>(cm, e), adam_decode<3, true>(cm, e + 1)),
                                             adam_two(sm));
                const float2 r0 = __fmul2_rn(make_float2(adam_decode<4, false>(cv, e), adam_decode<4, false>(cv, e + 1)),
                                             adam_two(sv));
                const float2 gr = make_float2(g[j].v[e], g[j].v[e + 1]), v0 = __fmul2_rn(r0, r0), gg = __fmul2_rn(gr, gr);
                const float2 x = make_float2(adam_blend(a.b1, m0.x, a.one_b1, gr.x),
                                             adam_blend(a.b1, m0.y, a.one_b1, gr.y));
                const float2 y = make_float2(__fsqrt_rn(adam_blend(a.b2, v0.x, a.one_b2, gg.x)),
                                             __fsqrt_rn(adam_blend(a.b2, v0.y, a.one_b2, gg.y)));
                // m / denom by an approximate reciprocal: what it is off by, 2^-22, is of the
                // update and not of p, and a moment's own rounding is 2^-4
                const float2 denom = __ffma2_rn(y, adam_two(a.inv_bc2), adam_two(a.eps));
                const float2 pn = __ffma2_rn(__fmul2_rn(adam_two(a.step_size), x),
                                             make_float2(__fdividef(-1.f, denom.x), __fdividef(-1.f, denom.y)),
                                             __fmul2_rn(make_float2(p[j].v[e], p[j].v[e + 1]), adam_two(a.decay)));
                p[j].v[e] = pn.x;
                p[j].v[e + 1] = pn.y;
                mn[2 * j + e / 2] = x;
                rn[2 * j + e / 2] = y;
                top_m = max(top_m, max(__float_as_uint(x.x) & 0x7fffffffu, __float_as_uint(x.y) & 0x7fffffffu));
                top_r = max(top_r, max(__float_as_uint(y.x) & 0x7fffffffu, __float_as_uint(y.y) & 0x7fffffffu));
            }
        }
        top_m = __reduce_max_sync(0xffffffffu, top_m);
        top_r = __reduce_max_sync(0xffffffffu, top_r);
        float inv_m, inv_r;
        const float new_sm = adam_scale<3>(top_m, inv_m), new_sv = adam_scale<4>(top_r, inv_r);
        // (the scale of a block that is 0 or NaN has no inverse: its codes are 0)
        const bool has_m = inv_m > 0.f, has_r = inv_r > 0.f;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            uint32_t wm = 0u, wv = 0u;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t bits = adam_mix(key + (uint32_t)(4 * lane + 128 * j + e));
                const float x = e & 1 ? mn[2 * j + e / 2].y : mn[2 * j + e / 2].x;
                const float y = e & 1 ? rn[2 * j + e / 2].y : rn[2 * j + e / 2].x;
                const uint32_t cm = adam_encode<3>(__fmul_rn(fabsf(x), inv_m), bits << 4 & 0xffff0u);
                const uint32_t cv = adam_encode<4>(__fmul_rn(y, inv_r), bits >> 13 & 0x7fff8u);
                const uint32_t sign = __float_as_uint(x) >> 24 & 0x80u;
                wm |= (cm > 0u ? cm | sign : 0u) << (8 * e);
                wv |= cv << (8 * e);
            }
            // Roots above 0 with the code 0.  (The four codes together are asked for a 0 first: a comparison per
            // value takes a step over 512 tensors from 656 us to 668, this to 662.)
            if ((wv - 0x01010101u) & ~wv & 0x80808080u) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float y = e & 1 ? rn[2 * j + e / 2].y : rn[2 * j + e / 2].x;
                    if (y > 0.f && (wv >> (8 * e) & 0xffu) == 0u) wv |= 1u << (8 * e);
                }
            }
            *reinterpret_cast<uint32_t *>(&m[j]) = has_m ? wm : 0u;
            *reinterpret_cast<uint32_t *>(&v[j]) = has_r ? wv : 0u;
        }
        if (lane == 0) {
            t.ms[b] = new_sm;
            t.vs[b] = new_sv;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float gr = g[j].v[e];
                const float mn = adam_blend(a.b1, m[j].v[e], a.one_b1, gr);
                const float vn = adam_blend(a.b2, v[j].v[e], a.one_b2, __fmul_rn(gr, gr));
                const float denom = __fadd_rn(__fdiv_rn(__fsqrt_rn(vn), a.bc2_sqrt), a.eps);
                p[j].v[e] = __fsub_rn(__fmul_rn(p[j].v[e], a.decay), __fdiv_rn(__fmul_rn(a.step_size, mn), denom));
                m[j].v[e] = mn;
                v[j].v[e] = vn;
            }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int64_t i = i0 + 128 * j;
        adam_store<WHOLE>(t.p, i, t.n, p[j]);
        adam_store<WHOLE>(static_cast<State *>(t.m), i, t.n, m[j]);
        adam_store<WHOLE>(static_cast<State *>(t.v), i, t.n, v[j]);
        if (t.p16) {
#pragma unroll
            for (int e = 0; e < 4; e += 2)
                *reinterpret_cast<__nv_bfloat162 *>(&h[j].v[e]) = __floats2bfloat162_rn(p[j].v[e], p[j].v[e + 1]);
            adam_store<WHOLE>(t.p16, i, t.n, h[j]);
        }
    }
}

// Warp w of W takes blocks [blocks w / W, blocks (w + 1) / W), tensor by tensor.
template <bool BITS8>
__global__ void __launch_bounds__(32 * kAdamWarps, BITS8 ? kAdamStep8 : kAdamStep32)
    adam_step_kernel(const __grid_constant__ AdamArgs a) {
    const int lane = threadIdx.x & 31;
    const int64_t w = (int64_t)blockIdx.x * kAdamWarps + (threadIdx.x >> 5), W = (int64_t)gridDim.x * kAdamWarps;
    const int64_t last = a.blocks * (w + 1) / W;
    for (int64_t at = a.blocks * w / W; at < last;) {
        const AdamTensor t = a.tensors[adam_find(a.first, a.count, at, lane)];
        int64_t b = at - t.block0;
        const int64_t whole = t.vec ? t.n / kAdamBlock : 0, end = min(last - t.block0, (t.n + kAdamBlock - 1) / kAdamBlock);
        at = t.block0 + end;
        // BITS8: the hash of the seed with the tensor's number, and that with the index' upper half
        const uint32_t tensor = BITS8 ? adam_mix(a.seed_lo ^ adam_mix(a.seed_hi ^ adam_mix(t.id + 1u))) : 0u;
        auto key = [&](int64_t k) {
            return BITS8 ? adam_mix(tensor + (uint32_t)(k * kAdamBlock >> 32)) + (uint32_t)(k * kAdamBlock) : 0u;
        };
        // Each lane asks L2 for one 128-byte line of a later block: the loads of a block then wait for L2
        // instead of HBM, without registers for what is under way.
        constexpr int kState = BITS8 ? 2 : 8;  // lines of a block's m, and of its v
        const char *line = lane < 8    ? reinterpret_cast<const char *>(t.p) + 128 * lane
                           : lane < 16 ? reinterpret_cast<const char *>(t.g) + 128 * (lane - 8)
                           : lane < 16 + kState ? static_cast<const char *>(t.m) + 128 * (lane - 16)
                                                : static_cast<const char *>(t.v) + 128 * (lane - 16 - kState);
        const int pitch = lane < 16 ? 1024 : 128 * kState;
        for (; b < min(end, whole); ++b) {
            if (lane < 16 + 2 * kState && b + kAdamAhead < min(end, whole))
                asm volatile("prefetch.global.L2 [%0];" ::"l"(line + (b + kAdamAhead) * pitch));
            adam_block<BITS8, true>(a, t, b, key(b), lane);
        }
        for (; b < end; ++b) adam_block<BITS8, false>(a, t, b, key(b), lane);
    }
}

// The values that the moments stand for, fp32, every tensor from its first block on.
template <bool BITS8>
__global__ void __launch_bounds__(32 * kAdamWarps, kAdamRead) adam_read_kernel(const __grid_constant__ AdamArgs a) {
    using State = typename std::conditional<BITS8, uint8_t, float>::type;
    const int lane = threadIdx.x & 31;
    const int64_t w = (int64_t)blockIdx.x * kAdamWarps + (threadIdx.x >> 5), W = (int64_t)gridDim.x * kAdamWarps;
    const int64_t last = a.blocks * (w + 1) / W;
    for (int64_t at = a.blocks * w / W; at < last;) {
        const AdamTensor t = a.tensors[adam_find(a.first, a.count, at, lane)];
        const int64_t whole = t.vec ? t.n / kAdamBlock : 0, end = min(last - t.block0, (t.n + kAdamBlock - 1) / kAdamBlock);
        for (int64_t b = at - t.block0; b < end; ++b) {
            const float sm = BITS8 ? t.ms[b] : 0.f, sv = BITS8 ? t.vs[b] : 0.f;
            const int64_t i0 = b * kAdamBlock + 4 * lane;
            AdamRun<State, 4> ms[2], vs[2];
            const State *pm = static_cast<const State *>(t.m), *pv = static_cast<const State *>(t.v);
            if (b < whole) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    ms[j] = adam_load<true>(pm, i0 + 128 * j, t.n);
                    vs[j] = adam_load<true>(pv, i0 + 128 * j, t.n);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    ms[j] = adam_load<false>(pm, i0 + 128 * j, t.n);
                    vs[j] = adam_load<false>(pv, i0 + 128 * j, t.n);
                }
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float m[4], v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (BITS8) {
                        m[e] = __fmul_rn(adam_decode<3, true>(adam_word(ms[j]), e), sm);
                        const float r = __fmul_rn(adam_decode<4, false>(adam_word(vs[j]), e), sv);
                        v[e] = __fmul_rn(r, r);
                    } else {
                        m[e] = ms[j].v[e];
                        v[e] = vs[j].v[e];
                    }
                    // rows of whole blocks: what lies past a tensor's end is 0
                    if (i0 + 128 * j + e >= t.n) m[e] = v[e] = 0.f;
                }
                const int64_t o = t.block0 * kAdamBlock + i0 + 128 * j;
                if (a.m32) __stcs(reinterpret_cast<float4 *>(a.m32 + o), make_float4(m[0], m[1], m[2], m[3]));
                if (a.v32) __stcs(reinterpret_cast<float4 *>(a.v32 + o), make_float4(v[0], v[1], v[2], v[3]));
            }
        }
        at = t.block0 + end;
    }
}

}  // namespace attt

struct attt_adamw {
    int dev, count, bits;
    int64_t blocks;
    attt::AdamTensor *tensors;  // on the device, behind them the first block of each
};

namespace attt {

// Fills in the handle's part of a and returns the blocks of kAdamWarps warps: as many as the
// device holds at once, or a block of values per warp.
static unsigned adam_grid(const attt_adamw *h, AdamArgs &a, int per_sm) {
    a.tensors = h->tensors;
    a.first = reinterpret_cast<const int64_t *>(h->tensors + h->count);
    a.count = h->count;
    a.blocks = h->blocks;
    return (unsigned)std::min<int64_t>(cdiv(h->blocks, kAdamWarps), (int64_t)per_sm * num_sms(h->dev));
}

static attt_status adam_device(const attt_adamw *h) {
    int dev;
    const attt_status st = current_device(&dev);
    if (st != ATTT_OK) return st;
    return dev == h->dev ? ATTT_OK : ATTT_ERR_INVALID_ARG;
}

}  // namespace attt

extern "C" {

attt_status attt_adamw_create(int count, float *const *d_p, const float *const *d_g, void *const *d_m,
                              void *const *d_v, float *const *d_ms, float *const *d_vs, attt_bf16 *const *d_p16,
                              const int64_t *n, int state_bits, attt_adamw **out) {
    ATTT_NVTX_RANGE();
    using namespace attt;
    if (!out) return ATTT_ERR_INVALID_ARG;
    *out = nullptr;
    if (count < 1 || !d_p || !d_g || !d_m || !d_v || !n || (state_bits != 32 && state_bits != 8)) return ATTT_ERR_INVALID_ARG;
    const bool b8 = state_bits == 8;
    if (b8 != (d_ms != nullptr) || b8 != (d_vs != nullptr)) return ATTT_ERR_INVALID_ARG;
    if (count > 1 << 20) return ATTT_ERR_UNSUPPORTED;
    try {
        std::vector<AdamTensor> list;
        list.reserve((size_t)count);
        std::vector<std::pair<uintptr_t, uintptr_t>> written;  // what a step writes
        int64_t blocks = 0;
        for (int k = 0; k < count; ++k) {
            AdamTensor t{};
            t.n = n[k];
            if (t.n < 0) return ATTT_ERR_INVALID_ARG;
            if (t.n > (1ll << 40)) return ATTT_ERR_UNSUPPORTED;
            t.p = d_p[k];
            t.g = d_g[k];
            t.m = d_m[k];
            t.v = d_v[k];
            t.ms = b8 ? d_ms[k] : nullptr;
            t.vs = b8 ? d_vs[k] : nullptr;
            t.p16 = d_p16 ? reinterpret_cast<__nv_bfloat16 *>(d_p16[k]) : nullptr;
            t.block0 = blocks;
            t.id = (uint32_t)k;
            if (t.n > 0) {
                if (!t.p || !t.g || !t.m || !t.v || (b8 && (!t.ms || !t.vs))) return ATTT_ERR_INVALID_ARG;
                if (!aligned_to(4, t.p, t.g, t.ms, t.vs) || !aligned_to(2, t.p16)) return ATTT_ERR_INVALID_ARG;
                if (!b8 && !aligned_to(4, t.m, t.v)) return ATTT_ERR_INVALID_ARG;
                t.vec = aligned_to(16, t.p, t.g) && aligned_to(b8 ? 4 : 16, t.m, t.v) && aligned_to(8, t.p16);
                const int64_t nb = cdiv(t.n, kAdamBlock), e = b8 ? 1 : 4;
                auto add = [&](const void *a, int64_t bytes) {
                    if (a) written.emplace_back(reinterpret_cast<uintptr_t>(a), reinterpret_cast<uintptr_t>(a) + bytes);
                };
                add(t.p, 4 * t.n);
                add(t.m, e * t.n);
                add(t.v, e * t.n);
                add(t.ms, 4 * nb);
                add(t.vs, 4 * nb);
                add(t.p16, 2 * t.n);
                blocks += nb;
                list.push_back(t);
            }
        }
        // one step's warps write everything at once: no two arrays may share a byte, nor a gradient
        // lie in one
        std::sort(written.begin(), written.end());
        for (size_t i = 1; i < written.size(); ++i)
            if (written[i].first < written[i - 1].second) return ATTT_ERR_INVALID_ARG;
        for (const AdamTensor &t : list) {
            const auto g = reinterpret_cast<uintptr_t>(t.g);
            auto it = std::lower_bound(written.begin(), written.end(),
                                       std::make_pair(g + (uintptr_t)(4 * t.n), (uintptr_t)0));
            if (it != written.begin() && (it - 1)->second > g) return ATTT_ERR_INVALID_ARG;
        }
        if (blocks >= 1ll << 33) return ATTT_ERR_UNSUPPORTED;
        int dev;
        const attt_status st = current_device(&dev);
        if (st != ATTT_OK) return st;
        std::unique_ptr<attt_adamw> h(new attt_adamw{dev, (int)list.size(), state_bits, blocks, nullptr});
        if (!list.empty()) {
            const size_t table = list.size() * sizeof(AdamTensor), bytes = table + list.size() * sizeof(int64_t);
            std::vector<char> image(bytes);
            std::memcpy(image.data(), list.data(), table);
            for (size_t k = 0; k < list.size(); ++k)
                std::memcpy(image.data() + table + k * sizeof(int64_t), &list[k].block0, sizeof(int64_t));
            if (fault_take(FAULT_ALLOC) || cudaMalloc(&h->tensors, bytes) != cudaSuccess) {
                (void)cudaGetLastError();
                return ATTT_ERR_CUDA;
            }
            // (the copy of pageable memory may still be on its way, and a step's stream need not wait for it)
            if (cudaMemcpy(h->tensors, image.data(), bytes, cudaMemcpyHostToDevice) != cudaSuccess ||
                cudaStreamSynchronize(nullptr) != cudaSuccess) {
                (void)cudaGetLastError();
                cudaFree(h->tensors);
                return ATTT_ERR_CUDA;
            }
        }
        *out = h.release();
        return ATTT_OK;
    } catch (const std::bad_alloc &) {
        return ATTT_ERR_CUDA;
    }
}

attt_status attt_adamw_destroy(attt_adamw *h) {
    if (!h) return ATTT_OK;
    int cur = -1;
    (void)cudaGetDevice(&cur);
    bool ok = cur == h->dev || cudaSetDevice(h->dev) == cudaSuccess;
    if (ok && h->tensors) ok = cudaFree(h->tensors) == cudaSuccess;  // waits for the device
    if (cur >= 0 && cur != h->dev) (void)cudaSetDevice(cur);
    delete h;
    return ok ? ATTT_OK : ATTT_ERR_CUDA;
}

int64_t attt_adamw_state_values(const attt_adamw *h) { return h ? h->blocks * attt::kAdamBlock : 0; }

attt_status attt_adamw_step(attt_adamw *h, double lr, double beta1, double beta2, double eps, double weight_decay,
                            int64_t step, uint64_t seed, attt_stream stream) {
    ATTT_NVTX_RANGE();
    using namespace attt;
    if (!h || step < 1 || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !((float)eps > 0.f) ||
        !(weight_decay >= 0.0) || !std::isfinite(lr) || !std::isfinite(eps) || !std::isfinite(weight_decay))
        return ATTT_ERR_INVALID_ARG;
    // (8 bits: 1 / eps stays finite, so that a value without moments stays where it is)
    if (h->bits == 8 && eps < 1e-30) return ATTT_ERR_INVALID_ARG;
    const attt_status st = adam_device(h);
    if (st != ATTT_OK) return st;
    if (h->blocks == 0) return ATTT_OK;
    AdamArgs a{};
    const unsigned grid = adam_grid(h, a, h->bits == 8 ? kAdamStep8 : kAdamStep32);
    // the step's scalars in double, rounded once to fp32
    a.decay = (float)(1.0 - lr * weight_decay);
    a.b1 = (float)beta1;
    a.one_b1 = (float)(1.0 - beta1);
    a.b2 = (float)beta2;
    a.one_b2 = (float)(1.0 - beta2);
    a.step_size = (float)(lr / (1.0 - std::pow(beta1, (double)step)));
    a.bc2_sqrt = (float)std::sqrt(1.0 - std::pow(beta2, (double)step));
    a.inv_bc2 = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
    a.eps = (float)eps;
    a.seed_lo = (uint32_t)seed;
    a.seed_hi = (uint32_t)(seed >> 32);
    if (h->bits == 8) adam_step_kernel<true><<<grid, 32 * kAdamWarps, 0, stream>>>(a);
    else adam_step_kernel<false><<<grid, 32 * kAdamWarps, 0, stream>>>(a);
    count_launch();
    return cudaGetLastError() == cudaSuccess ? ATTT_OK : ATTT_ERR_CUDA;
}

attt_status attt_adamw_read_state(const attt_adamw *h, float *d_m32, float *d_v32, attt_stream stream) {
    ATTT_NVTX_RANGE();
    using namespace attt;
    if (!h || (!d_m32 && !d_v32) || !aligned_to(16, d_m32, d_v32)) return ATTT_ERR_INVALID_ARG;
    const int64_t bytes = h->blocks * kAdamBlock * (int64_t)sizeof(float);
    if (share_a_byte({d_m32, bytes}, {d_v32, bytes})) return ATTT_ERR_INVALID_ARG;
    const attt_status st = adam_device(h);
    if (st != ATTT_OK) return st;
    if (h->blocks == 0) return ATTT_OK;
    AdamArgs a{};
    const unsigned grid = adam_grid(h, a, kAdamRead);
    a.m32 = d_m32;
    a.v32 = d_v32;
    if (h->bits == 8) adam_read_kernel<true><<<grid, 32 * kAdamWarps, 0, stream>>>(a);
    else adam_read_kernel<false><<<grid, 32 * kAdamWarps, 0, stream>>>(a);
    count_launch();
    return cudaGetLastError() == cudaSuccess ? ATTT_OK : ATTT_ERR_CUDA;
}

}  // extern "C"

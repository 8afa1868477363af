// adamw.cu -- the AdamW step of many tensors in one launch, with moments in 32 bits
// or in 8.
//
//   m <- b1 m + (1 - b1) g;  v <- b2 v + (1 - b2) g^2
//   p <- p (1 - lr wd) - (lr / (1 - b1^t)) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
// with every operation rounded on its own, as attt_lora_adamw_step: with moments in 32
// bits the two give the same bits.
//
// Moments in 8 bits: blocks of 256 values with one fp32 scale each.  A code is a number of 4
// exponent bits and k mantissa bits (exponent 0: without the leading one): 0 to 2 - 2^-k in
// 2^-14 steps of a relative 2^-k; m has a sign and k = 3, and in the place of v its root
// with k = 4 (the range of v would be twice as many powers of two).  The scale makes the
// block's largest value the largest code.  What a code cuts off rounds up with the probability
// of its size: with b2 = 0.999 a step without gradient takes 1/2000 of sqrt(v), a
// sixtieth of the distance to the next code or less, and rounding to nearest would never
// let it fall.  The random bits are a hash of (seed, tensor, index): a step can be repeated.
// The step itself uses the moments before they are rounded.
//
// Bound: HBM bytes, 30 a value (8 bits: 18 and 16 per block).  A warp takes a block of 256 values,
// a lane two runs of four (16-byte vectors that lie side by side); largest values by one
// reduction over the warp.
#include <algorithm>
#include <cmath>
#include <new>
#include <type_traits>
#include <utility>
#include <vector>

#include "attt_common.cuh"
#include "attt_host.h"

namespace attt {

constexpr int kAdamBlock = 256;  // values of a scale, and of a warp's step
constexpr int kAdamWarps = 8;
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
    int count;
    int64_t blocks;
    int steps;  // of each warp
    float decay, b1, one_b1, b2, one_b2, step_size, bc2_sqrt, eps;
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

template <int K>
__device__ __forceinline__ float adam_decode(uint32_t code) {
    const uint32_t low = code & ((1u << K) - 1u), e = code >> K;
    return e > 0u ? __uint_as_float(((e + 112u) << 23) | (low << (23 - K))) : (float)low * (1.f / (float)(1 << (14 + K)));
}

// The code of a in [0, 2 - 2^-K]; rnd: 23 - K random bits.
template <int K>
__device__ __forceinline__ uint32_t adam_encode(float a, uint32_t rnd) {
    constexpr int cut = 23 - K;
    const uint32_t big = ((__float_as_uint(a) + rnd) >> cut) - (112u << K);
    const uint32_t small = ((uint32_t)(a * 0x1p37f) + rnd) >> cut;  // used below 2^-14: under 2^23
    return min(a >= 0x1p-14f ? big : small, (16u << K) - 1u);
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

// The tensor that has block b: the last one whose first block is not after it.
__device__ __forceinline__ int adam_find(const AdamTensor *t, int count, int64_t b) {
    int lo = 0, hi = count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (__ldg(&t[mid].block0) <= b) lo = mid;
        else hi = mid;
    }
    return lo;
}

template <class T, int N>
struct alignas(sizeof(T) * N) AdamRun {
    T v[N];
};

// Four neighbouring values from i on, those from n on as zeros.
template <class T>
__device__ __forceinline__ AdamRun<T, 4> adam_load(const T *p, int64_t i, int64_t n, bool whole) {
    if (whole) return *reinterpret_cast<const AdamRun<T, 4> *>(p + i);
    AdamRun<T, 4> r{};
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (i + k < n) r.v[k] = p[i + k];
    return r;
}
template <class T>
__device__ __forceinline__ void adam_store(T *p, int64_t i, int64_t n, bool whole, const AdamRun<T, 4> &r) {
    if (whole) {
        *reinterpret_cast<AdamRun<T, 4> *>(p + i) = r;
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (i + k < n) p[i + k] = r.v[k];
}

template <bool BITS8>
__global__ void __launch_bounds__(32 * kAdamWarps) adam_step_kernel(const __grid_constant__ AdamArgs a) {
    using State = typename std::conditional<BITS8, uint8_t, float>::type;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int64_t b = ((int64_t)blockIdx.x * a.steps) * kAdamWarps + warp;
    if (b >= a.blocks) return;
    int k = adam_find(a.tensors, a.count, b);
    AdamTensor t = a.tensors[k];
    int64_t end = k + 1 < a.count ? __ldg(&a.tensors[k + 1].block0) : a.blocks;
    for (int s = 0; s < a.steps && b < a.blocks; ++s, b += kAdamWarps) {
        if (b >= end) {  // the warp's next block is in a later tensor
            k = adam_find(a.tensors, a.count, b);
            t = a.tensors[k];
            end = k + 1 < a.count ? __ldg(&a.tensors[k + 1].block0) : a.blocks;
        }
        const int64_t i0 = (b - t.block0) * kAdamBlock;
        const bool whole = t.vec && i0 + kAdamBlock <= t.n;
        AdamRun<float, 4> p[2], g[2];
        AdamRun<State, 4> ms[2], vs[2];
        const State *tm = static_cast<const State *>(t.m), *tv = static_cast<const State *>(t.v);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int64_t i = i0 + 128 * j + 4 * lane;
            p[j] = adam_load(t.p, i, t.n, whole);
            g[j] = adam_load(t.g, i, t.n, whole);
            ms[j] = adam_load(tm, i, t.n, whole);
            vs[j] = adam_load(tv, i, t.n, whole);
        }
        float sm = 0.f, sv = 0.f;
        if (BITS8) {
            sm = t.ms[b - t.block0];
            sv = t.vs[b - t.block0];
        }
        float m[8], root[8];
        uint32_t top_m = 0u, top_r = 0u;
        AdamRun<__nv_bfloat16, 4> h[2];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float m0, v0;
                if constexpr (BITS8) {
                    const uint32_t cm = ms[j].v[e];
                    m0 = __fmul_rn(adam_decode<3>(cm & 127u), sm);
                    if (cm & 128u) m0 = -m0;
                    const float r = __fmul_rn(adam_decode<4>(vs[j].v[e]), sv);
                    v0 = __fmul_rn(r, r);
                } else {
                    m0 = ms[j].v[e];
                    v0 = vs[j].v[e];
                }
                const float gr = g[j].v[e];
                const float mn = __fadd_rn(__fmul_rn(a.b1, m0), __fmul_rn(a.one_b1, gr));
                const float vn = __fadd_rn(__fmul_rn(a.b2, v0), __fmul_rn(a.one_b2, __fmul_rn(gr, gr)));
                const float rn = __fsqrt_rn(vn);
                const float denom = __fadd_rn(__fdiv_rn(rn, a.bc2_sqrt), a.eps);
                const float pn = __fsub_rn(__fmul_rn(p[j].v[e], a.decay), __fdiv_rn(__fmul_rn(a.step_size, mn), denom));
                p[j].v[e] = pn;
                h[j].v[e] = __float2bfloat16_rn(pn);
                if constexpr (BITS8) {
                    m[4 * j + e] = mn;
                    root[4 * j + e] = rn;
                    top_m = max(top_m, __float_as_uint(mn) & 0x7fffffffu);
                    top_r = max(top_r, __float_as_uint(rn) & 0x7fffffffu);
                } else {
                    ms[j].v[e] = mn;
                    vs[j].v[e] = vn;
                }
            }
        if constexpr (BITS8) {
            top_m = __reduce_max_sync(0xffffffffu, top_m);
            top_r = __reduce_max_sync(0xffffffffu, top_r);
            float inv_m, inv_r;
            sm = adam_scale<3>(top_m, inv_m);
            sv = adam_scale<4>(top_r, inv_r);
            const uint32_t tensor = adam_mix(a.seed_lo ^ adam_mix(a.seed_hi ^ adam_mix(t.id + 1u)));
            const uint32_t key = adam_mix(tensor + (uint32_t)(i0 >> 32));
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t bits = adam_mix((uint32_t)i0 + (uint32_t)(128 * j + 4 * lane + e) + key);
                    const float mn = m[4 * j + e];
                    // a scale of 0 or NaN has inv 0 (and a NaN times it is not taken)
                    const float x = inv_m > 0.f ? __fmul_rn(fabsf(mn), inv_m) : 0.f;
                    const float y = inv_r > 0.f ? __fmul_rn(root[4 * j + e], inv_r) : 0.f;
                    const uint32_t cm = adam_encode<3>(x, (bits & 0xffffu) << 4);
                    ms[j].v[e] = (uint8_t)(cm | (mn < 0.f && cm > 0u ? 128u : 0u));
                    vs[j].v[e] = (uint8_t)adam_encode<4>(y, (bits >> 16) << 3);
                }
            if (lane == 0) {
                t.ms[b - t.block0] = sm;
                t.vs[b - t.block0] = sv;
            }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int64_t i = i0 + 128 * j + 4 * lane;
            adam_store(t.p, i, t.n, whole, p[j]);
            adam_store(static_cast<State *>(t.m), i, t.n, whole, ms[j]);
            adam_store(static_cast<State *>(t.v), i, t.n, whole, vs[j]);
            if (t.p16) adam_store(t.p16, i, t.n, whole, h[j]);
        }
    }
}

// The values that the moments stand for, fp32, every tensor from its first block on.
template <bool BITS8>
__global__ void __launch_bounds__(32 * kAdamWarps) adam_read_kernel(const __grid_constant__ AdamArgs a) {
    using State = typename std::conditional<BITS8, uint8_t, float>::type;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int64_t b = ((int64_t)blockIdx.x * a.steps) * kAdamWarps + warp;
    for (int s = 0; s < a.steps && b < a.blocks; ++s, b += kAdamWarps) {
        const AdamTensor t = a.tensors[adam_find(a.tensors, a.count, b)];
        const int64_t i0 = (b - t.block0) * kAdamBlock;
        const bool whole = t.vec && i0 + kAdamBlock <= t.n;
        const float sm = BITS8 ? t.ms[b - t.block0] : 0.f, sv = BITS8 ? t.vs[b - t.block0] : 0.f;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int64_t i = i0 + 128 * j + 4 * lane;
            const AdamRun<State, 4> ms = adam_load(static_cast<const State *>(t.m), i, t.n, whole);
            const AdamRun<State, 4> vs = adam_load(static_cast<const State *>(t.v), i, t.n, whole);
            AdamRun<float, 4> m, v;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (BITS8) {
                    const uint32_t c = ms.v[e];
                    const float x = __fmul_rn(adam_decode<3>(c & 127u), sm), r = __fmul_rn(adam_decode<4>(vs.v[e]), sv);
                    m.v[e] = c & 128u ? -x : x;
                    v.v[e] = __fmul_rn(r, r);
                } else {
                    m.v[e] = ms.v[e];
                    v.v[e] = vs.v[e];
                }
            }
            // rows of whole blocks: what lies past a tensor's end is 0
            const int64_t o = b * kAdamBlock + 128 * j + 4 * lane;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i + e >= t.n) m.v[e] = v.v[e] = 0.f;
            if (a.m32) *reinterpret_cast<AdamRun<float, 4> *>(a.m32 + o) = m;
            if (a.v32) *reinterpret_cast<AdamRun<float, 4> *>(a.v32 + o) = v;
        }
    }
}

}  // namespace attt

struct attt_adamw {
    int dev, count, bits;
    int64_t blocks;
    attt::AdamTensor *tensors;  // on the device
};

namespace attt {

// Blocks of kAdamWarps warps for the handle's blocks: up to 8 steps a warp, fewer where that
// would leave SMs without four blocks.
static unsigned adam_grid(const attt_adamw *h, AdamArgs &a) {
    const int64_t sets = cdiv(h->blocks, kAdamWarps), want = 4ll * num_sms(h->dev);
    int64_t steps = sets / want;
    a.steps = (int)(steps < 1 ? 1 : steps > 8 ? 8 : steps);
    a.tensors = h->tensors;
    a.count = h->count;
    a.blocks = h->blocks;
    return (unsigned)cdiv(sets, a.steps);
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
        attt_adamw *h = new attt_adamw{dev, (int)list.size(), state_bits, blocks, nullptr};
        if (!list.empty()) {
            const size_t bytes = list.size() * sizeof(AdamTensor);
            if (fault_take(FAULT_ALLOC) || cudaMalloc(&h->tensors, bytes) != cudaSuccess) {
                (void)cudaGetLastError();
                delete h;
                return ATTT_ERR_CUDA;
            }
            if (cudaMemcpy(h->tensors, list.data(), bytes, cudaMemcpyHostToDevice) != cudaSuccess) {
                (void)cudaGetLastError();
                cudaFree(h->tensors);
                delete h;
                return ATTT_ERR_CUDA;
            }
        }
        *out = h;
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
    const attt_status st = adam_device(h);
    if (st != ATTT_OK) return st;
    if (h->blocks == 0) return ATTT_OK;
    AdamArgs a{};
    const unsigned grid = adam_grid(h, a);
    // the step's scalars in double, rounded once to fp32
    a.decay = (float)(1.0 - lr * weight_decay);
    a.b1 = (float)beta1;
    a.one_b1 = (float)(1.0 - beta1);
    a.b2 = (float)beta2;
    a.one_b2 = (float)(1.0 - beta2);
    a.step_size = (float)(lr / (1.0 - std::pow(beta1, (double)step)));
    a.bc2_sqrt = (float)std::sqrt(1.0 - std::pow(beta2, (double)step));
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
    const attt_status st = adam_device(h);
    if (st != ATTT_OK) return st;
    if (h->blocks == 0) return ATTT_OK;
    AdamArgs a{};
    const unsigned grid = adam_grid(h, a);
    a.m32 = d_m32;
    a.v32 = d_v32;
    if (h->bits == 8) adam_read_kernel<true><<<grid, 32 * kAdamWarps, 0, stream>>>(a);
    else adam_read_kernel<false><<<grid, 32 * kAdamWarps, 0, stream>>>(a);
    count_launch();
    return cudaGetLastError() == cudaSuccess ? ATTT_OK : ATTT_ERR_CUDA;
}

}  // extern "C"

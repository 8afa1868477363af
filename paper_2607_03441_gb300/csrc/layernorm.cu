// layernorm.cu -- layer norm over the rows of a matrix, forward and backward,
// with the reduction of the weight's and the bias's gradient.
//
//   y_i = (x_i - mean) rstd gamma_i + beta_i,  rstd = 1 / sqrt(var + eps)
//   with g = dy gamma, xh = (x - mean) rstd:
//   dx = rstd (g - mean(g) - xh mean(g xh)),  dgamma = sum_rows dy xh,  dbeta = sum_rows dy
// A row stays in the registers of its warps between the reductions (mean, then the
// centred variance: no difference of large sums), so x and dy are read and y and
// dx written once; all sums are fp32.
//
// A persistent block per SM holds as many groups of warps as its threads allow; each
// group takes every (blocks x groups)-th row, or pair of rows, through a ring of its
// own in shared memory: one thread issues a row's bulk copies as soon as the group
// has read the row before it in that place (its first reduction says so), so the
// copies of several rows are in flight while one is worked on.  Rows that do not lie
// on 16-byte boundaries arrive in windows that do and are read value by value.
// The backward keeps the weight sums of a thread's columns in registers over all rows
// that its block takes; blocks leave one partial row each, and a second kernel adds
// those in a fixed order.
// Bound: HBM bytes for long texts, below a few hundred rows the chain of a launch, a
// load, two reductions and a store.  What stands between the kernels and the bytes is
// issue slots and waits: hence two values per instruction, few warps per row, and no
// branches between a thread's vectors.
// Figures (8,192 rows, both kernels of the backward): 5,120 bf16 32 us forward (77% of
// the copy bandwidth) and 47-50 backward (75-80%; 48 without the weights' sums); 5,001 bf16
// 43 and 81, 5,001 fp32 63 and 88, value by value from the window.  One block per row
// without the ring took 47 and 148, and value by value from global memory 176 and 310 at
// 5,001 bf16.
#include <algorithm>

#include "attt_common.cuh"
#include "attt_host.h"

namespace attt {

constexpr int kLnMaxBlocks = 160;  // partial rows of the weight gradients, at most
constexpr int kLnThreads = 512;  // of a block, at most: 128 registers, and no spills (which go to L2 here)
constexpr int kLnStages = 8;
constexpr int kLnRed = kLnThreads / 32;

// Two fp32 values in a register pair, added, multiplied and fused in one instruction.
using F2 = float2;
__device__ __forceinline__ F2 f2(float a, float b) { return make_float2(a, b); }
__device__ __forceinline__ F2 f2_add(F2 a, F2 b) { return __fadd2_rn(a, b); }
__device__ __forceinline__ F2 f2_mul(F2 a, F2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ F2 f2_fma(F2 a, F2 b, F2 c) { return __ffma2_rn(a, b, c); }
__device__ __forceinline__ float f2_sum(F2 a) { return a.x + a.y; }

__device__ __forceinline__ float ln_value(float v) { return v; }
__device__ __forceinline__ float ln_value(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void ln_put(float *p, float v) { *p = v; }
__device__ __forceinline__ void ln_put(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

// Four neighbouring values of a row: 16 bytes of fp32, 8 of bf16 (a warp's reads then
// lie side by side, as do those of its fp32 weights; 8 bf16 values a thread would read
// the weights 32 bytes apart, two bank conflicts each).
__device__ __forceinline__ void ln_load4(const float *p, F2 (&f)[2]) {
    const float4 v = *reinterpret_cast<const float4 *>(p);
    f[0] = f2(v.x, v.y);
    f[1] = f2(v.z, v.w);
}
__device__ __forceinline__ void ln_load4(const __nv_bfloat16 *p, F2 (&f)[2]) {
    const uint2 u = *reinterpret_cast<const uint2 *>(p);
    f[0] = f2(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u));
    f[1] = f2(__uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u));
}
__device__ __forceinline__ void ln_store4(float *p, const F2 (&f)[2]) {
    *reinterpret_cast<float4 *>(p) = make_float4(f[0].x, f[0].y, f[1].x, f[1].y);
}
__device__ __forceinline__ void ln_store4(__nv_bfloat16 *p, const F2 (&f)[2]) {
    __nv_bfloat162 o[2] = {__float22bfloat162_rn(f[0]), __float22bfloat162_rn(f[1])};
    *reinterpret_cast<uint2 *>(p) = *reinterpret_cast<uint2 *>(o);
}

// ---------------------------------------------------------------------------
// A thread's columns of a row
// ---------------------------------------------------------------------------

// A thread holds NV vectors of 4 values: neighbours (VEC), or 32 columns apart, so that
// the lanes of a warp read neighbours in either form.  All vectors but the last lie
// within the row for every thread (ln_ring sees to it).  What of the last one lies
// past the row reads the row's first value and counts 0 times: no branch between the
// vectors (branches and a loop over the warps' sums cost a third of the forward's
// instructions).
template <int NV, bool VEC>
struct LnLane {
    int t0, step;               // first column, distance of the vectors
    int last[VEC ? 1 : 4];      // columns of the last vector
    bool in[VEC ? 1 : 4];       // whether they lie within the row
    F2 count[VEC ? 1 : 2];      // 1 or 0 for each of them

    __device__ __forceinline__ LnLane(int wr, int lane, int warps, int d) {
        t0 = wr * 128 + (VEC ? 4 * lane : lane);
        step = warps * 128;
        float on[VEC ? 1 : 4];
#pragma unroll
        for (int j = 0; j < (VEC ? 1 : 4); ++j) {
            last[j] = t0 + (NV - 1) * step + 32 * j;
            in[j] = last[j] < d;
            if (!in[j]) last[j] = 0;
            on[j] = in[j] ? 1.f : 0.f;
        }
        if constexpr (VEC) {
            count[0] = f2(on[0], on[0]);
        } else {
            count[0] = f2(on[0], on[1]);
            count[1] = f2(on[2], on[3]);
        }
    }
    // Column of value j of vector k.
    __device__ __forceinline__ int at(int k, int j) const {
        if constexpr (VEC) return (k == NV - 1 ? last[0] : t0 + k * step) + j;
        else return k == NV - 1 ? last[j] : t0 + k * step + 32 * j;
    }
    __device__ __forceinline__ bool inside(int k, int j) const { return k < NV - 1 || in[VEC ? 0 : j]; }
    // Vector k times what it counts.
    __device__ __forceinline__ F2 counted(int k, int e, F2 v) const {
        return k == NV - 1 ? f2_mul(v, count[VEC ? 0 : e]) : v;
    }
    template <class T>
    __device__ __forceinline__ void load(const T *row, int k, F2 (&f)[2]) const {
        if constexpr (VEC) {
            ln_load4(row + at(k, 0), f);
        } else {
            f[0] = f2(ln_value(row[at(k, 0)]), ln_value(row[at(k, 1)]));
            f[1] = f2(ln_value(row[at(k, 2)]), ln_value(row[at(k, 3)]));
        }
    }
    template <class T>
    __device__ __forceinline__ void store(T *row, int k, const F2 (&f)[2]) const {
        if constexpr (VEC) {
            if (inside(k, 0)) ln_store4(row + at(k, 0), f);
        } else {
            if (inside(k, 0)) ln_put(row + at(k, 0), f[0].x);
            if (inside(k, 1)) ln_put(row + at(k, 1), f[0].y);
            if (inside(k, 2)) ln_put(row + at(k, 2), f[1].x);
            if (inside(k, 3)) ln_put(row + at(k, 3), f[1].y);
        }
    }
};

// ---------------------------------------------------------------------------
// Sums over a row's warps
// ---------------------------------------------------------------------------

// The sum of the `warps` values that a row's warps left in red (a multiple of 4 floats, 0
// past them): all read them as vectors, which takes less than a second round of shuffles.
__device__ __forceinline__ float ln_gather(const float *red, int warps) {
    F2 t[2] = {f2(0.f, 0.f), f2(0.f, 0.f)};
#pragma unroll
    for (int w = 0; w < kLnRed; w += 4)
        if (w < warps) {
            F2 q[2];
            ln_load4(red + w, q);
            t[0] = f2_add(t[0], q[0]);
            t[1] = f2_add(t[1], q[1]);
        }
    return f2_sum(f2_add(t[0], t[1]));
}

// Sums of one or two values over a row's warps, in every thread; `red`: N ld floats that
// no other call of this row's warps still reads (a row's calls alternate between two).
// Two values: each half of a warp's lanes takes one.
template <int N>
__device__ __forceinline__ void ln_sums(const F2 (&part)[N], float (&out)[N], int warps, int wr, int lane, int bar,
                                        float *red, int ld) {
    static_assert(N == 1 || N == 2, "");
    const bool up = N == 2 && lane >= 16;
    float v = f2_sum(part[0]);
    if constexpr (N == 2) {
        const float b = f2_sum(part[1]), other = __shfl_xor_sync(0xffffffffu, up ? v : b, 16);
        v = (up ? b : v) + other;
    } else {
        v += __shfl_xor_sync(0xffffffffu, v, 16);
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (warps == 1) {
#pragma unroll
        for (int n = 0; n < N; ++n) out[n] = __shfl_sync(0xffffffffu, v, 16 * n);
        __syncwarp();
        return;
    }
    if ((lane & (N == 2 ? 15 : 31)) == 0) red[(up ? ld : 0) + wr] = v;
    named_barrier_sync(1u + bar, 32u * warps);
#pragma unroll
    for (int n = 0; n < N; ++n) out[n] = ln_gather(red + n * ld, warps);
}

// ---------------------------------------------------------------------------
// The ring
// ---------------------------------------------------------------------------

struct LnShape {
    int64_t L, x_ld, y_ld, g_ld;  // y_ld: of y or dx; g_ld: of dy
    int d;
    int warps;   // of a row
    int red_ld;  // floats between a row's sums, a multiple of 4
    float inv_d, eps;
};

struct LnRing {
    int stages, groups;
    uint32_t place_bytes;   // of one row
    uint32_t weight_bytes;  // gamma in shared memory, fp32
};

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
                 "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}

// A group's ring: `stages` barriers, places of ROWS rows each.  Shared memory: gamma (or
// nothing), the groups' places, their barriers.
template <class T, int ROWS, bool VEC>
struct LnGroup {
    uint8_t *place0;
    uint32_t bar0, place_bytes, row_bytes;
    int stages, stage;
    uint32_t phase;

    __device__ __forceinline__ LnGroup(const LnRing &r, uint8_t *smem, int grp, int d) {
        place0 = smem + r.weight_bytes + (uint32_t)grp * r.stages * ROWS * r.place_bytes;
        bar0 = smem_u32(smem) + r.weight_bytes + (uint32_t)r.groups * r.stages * ROWS * r.place_bytes +
               8u * grp * r.stages;
        place_bytes = r.place_bytes;
        row_bytes = (uint32_t)(d * sizeof(T));
        stages = r.stages;
        stage = 0;
        phase = 0;
    }
    // The current place's r-th row; `src`: where it came from.
    __device__ __forceinline__ const T *row(int r, const T *src) const {
        const uint8_t *p = place0 + (uint32_t)(stage * ROWS + r) * place_bytes;
        if constexpr (!VEC) p += reinterpret_cast<uintptr_t>(src) & 15u;
        return reinterpret_cast<const T *>(p);
    }
    // One thread: the copies of place st's rows; src(r): where the r-th starts, [from(r),
    // to(r)): the matrix that it belongs to.  Rows that lie on 16-byte boundaries come
    // as they are.  Others come in the window of whole 16 bytes around them, which holds
    // nothing but the matrix (other rows' values, or what lies between rows) unless it
    // reaches past the matrix's ends: then its inner part, and the rest value by value.
    template <class Src, class From, class To>
    __device__ __forceinline__ void issue(int st, Src &&src, From &&from, To &&to) const {
        const uint32_t bar = bar0 + 8u * st;
        uint8_t *const p0 = place0 + (uint32_t)st * ROWS * place_bytes;
        if constexpr (VEC) {
            mbar_arrive_expect_tx(bar, ROWS * row_bytes);
#pragma unroll
            for (int r = 0; r < ROWS; ++r) bulk_load(smem_u32(p0) + r * place_bytes, src(r), row_bytes, bar);
        } else {
            uintptr_t lo[ROWS];
            uint32_t bytes[ROWS], skip[ROWS], all = 0;
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const T *s = src(r);
                const uintptr_t a = reinterpret_cast<uintptr_t>(s), e = a + row_bytes, base = a & ~uintptr_t(15);
                uintptr_t hi = (e + 15) & ~uintptr_t(15);
                lo[r] = base;
                if (base < reinterpret_cast<uintptr_t>(from(r)) || hi > reinterpret_cast<uintptr_t>(to(r))) {
                    lo[r] = (a + 15) & ~uintptr_t(15);
                    hi = e & ~uintptr_t(15);
                    if (hi < lo[r]) hi = lo[r];
                    const int n = (int)(row_bytes / sizeof(T)), n0 = (int)((lo[r] - a) / sizeof(T)),
                              n1 = hi > lo[r] ? (int)((hi - a) / sizeof(T)) : 0;
                    T *d = reinterpret_cast<T *>(p0 + r * place_bytes + (a - base));
                    for (int i = 0; i < n; ++i) {
                        if (i == n0 && n1 > n0) i = n1;
                        if (i < n) d[i] = s[i];
                    }
                    fence_proxy_async_smem();
                }
                skip[r] = (uint32_t)(lo[r] - base);
                bytes[r] = (uint32_t)(hi - lo[r]);
                all += bytes[r];
            }
            mbar_arrive_expect_tx(bar, all);
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
                if (bytes[r] > 0)
                    bulk_load(smem_u32(p0) + r * place_bytes + skip[r], reinterpret_cast<const void *>(lo[r]), bytes[r],
                              bar);
        }
    }
    // Whether the current place's rows have landed.  A wait that runs out is recorded; the
    // leader then lets what it has issued (units unit, unit + stride, .. < ahead) land,
    // bounded too, and issues no more.  Everybody goes on to the last unit without
    // waiting again, on garbage, so that the group's barriers stay matched.
    __device__ __forceinline__ bool wait(volatile int *abort_flag, int *status, bool leader, int64_t unit,
                                         int64_t &ahead, int64_t stride, int64_t units) const {
        if (mbar_wait(bar0 + 8u * stage, phase, abort_flag)) return true;
        *abort_flag = 1;
        record_error(status, ATTT_ERR_TIMEOUT);
        if (leader) {
            volatile int no_abort = 0;
            int st = stage;
            uint32_t ph = phase;
            for (; unit < ahead; unit += stride) {
                (void)mbar_wait(bar0 + 8u * st, ph, &no_abort);
                if (++st == stages) {
                    st = 0;
                    ph ^= 1u;
                }
            }
            ahead = units;
        }
        return false;
    }
    __device__ __forceinline__ void next() {
        if (++stage == stages) {
            stage = 0;
            phase ^= 1u;
        }
    }
};

// The barriers of all groups, and zeros into the sums' places.
__device__ __forceinline__ void ln_init(uint32_t bar0, int bars, float *red, int reds, int *abort_flag) {
    for (int i = threadIdx.x; i < reds; i += blockDim.x) red[i] = 0.f;
    if (threadIdx.x == 0) {
        for (int i = 0; i < bars; ++i) mbar_init(bar0 + 8u * i, 1);
        *abort_flag = 0;
        fence_mbar_init();
    }
    __syncthreads();
}

// ROWS rows at a time (rows ROWS u .., u = the group's number, + the number of groups,
// ..), NV vectors of each per thread: two rows share the reductions' barriers and fill
// each other's waits.  gamma and beta are in registers where KEEP, else they come from
// global memory for every row (rows longer than the registers of a block hold).
template <class T, bool VEC, int NV, bool KEEP, int ROWS>
__global__ void __launch_bounds__(kLnThreads, 1)
    ln_forward_kernel(const T *__restrict__ x, const float *__restrict__ gamma, const float *__restrict__ beta,
                      T *__restrict__ y, float *__restrict__ mean, float *__restrict__ rstd, const LnShape s,
                      const LnRing ring, int *status) {
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(16) float red[2][ROWS * kLnRed * 4];
    __shared__ int abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int grp = warp / s.warps, wr = warp - grp * s.warps;
    const LnLane<NV, VEC> l(wr, lane, s.warps, s.d);
    LnGroup<T, ROWS, VEC> g(ring, smem, grp, s.d);
    ln_init(g.bar0 - 8u * grp * ring.stages, ring.groups * ring.stages, &red[0][0], 2 * ROWS * kLnRed * 4, &abort_flag);
    const int64_t stride = (int64_t)gridDim.x * ring.groups, units = (s.L + ROWS - 1) / ROWS;
    int64_t unit = (int64_t)blockIdx.x * ring.groups + grp, ahead = unit;
    const bool leader = wr == 0 && lane == 0;
    bool ok = true;
    auto row_of = [&](int64_t u, int r) { return min(ROWS * u + r, s.L - 1); };  // past L: the last again
    auto issue = [&](int st, int64_t u) {
        g.issue(st, [&](int r) { return x + row_of(u, r) * s.x_ld; }, [&](int) { return x; },
                [&](int) { return x + (s.L - 1) * s.x_ld + s.d; });
    };
    if (leader)
        for (int st = 0; st < ring.stages && ahead < units; ++st, ahead += stride) issue(st, ahead);
    F2 w[KEEP ? NV : 1][2], b[KEEP ? NV : 1][2];
    auto weights = [&](int k, F2(&wv)[2], F2(&bv)[2]) {
        l.load(gamma, k, wv);
        bv[0] = bv[1] = f2(0.f, 0.f);
        if (beta) l.load(beta, k, bv);
    };
    if constexpr (KEEP) {
#pragma unroll
        for (int k = 0; k < NV; ++k) weights(k, w[k], b[k]);
    }
    float *const red0 = red[0] + ROWS * grp * s.red_ld, *const red1 = red[1] + ROWS * grp * s.red_ld;
    T *yr = y + ROWS * unit * s.y_ld;
    for (; unit < units; unit += stride, yr += ROWS * stride * s.y_ld) {
        if (ok) ok = g.wait(&abort_flag, status, leader, unit, ahead, stride, units);
        F2 v[ROWS][NV][2], part[ROWS];
        float mu[ROWS], rs[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const T *row = g.row(r, x + row_of(unit, r) * s.x_ld);
            part[r] = f2(0.f, 0.f);
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                l.load(row, k, v[r][k]);
#pragma unroll
                for (int e = 0; e < 2; ++e) part[r] = f2_add(part[r], l.counted(k, e, v[r][k][e]));
            }
        }
        ln_sums<ROWS>(part, mu, s.warps, wr, lane, grp, red0, s.red_ld);
        if (leader && ahead < units) {
            issue(g.stage, ahead);
            ahead += stride;
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            mu[r] *= s.inv_d;
            const F2 nm = f2(-mu[r], -mu[r]);
            part[r] = f2(0.f, 0.f);
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    v[r][k][e] = f2_add(v[r][k][e], nm);
                    part[r] = f2_fma(l.counted(k, e, v[r][k][e]), v[r][k][e], part[r]);
                }
        }
        ln_sums<ROWS>(part, rs, s.warps, wr, lane, grp, red1, s.red_ld);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            rs[r] = rsqrtf(fmaf(rs[r], s.inv_d, s.eps));
            if (r > 0 && ROWS * unit + r >= s.L) break;
            const F2 r2 = f2(rs[r], rs[r]);
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int kw = KEEP ? k : 0;
                if constexpr (!KEEP) weights(k, w[0], b[0]);
#pragma unroll
                for (int e = 0; e < 2; ++e) v[r][k][e] = f2_fma(f2_mul(v[r][k][e], r2), w[kw][e], b[kw][e]);
                l.store(yr + r * s.y_ld, k, v[r][k]);
            }
            if (leader) {
                if (mean) mean[ROWS * unit + r] = mu[r];
                if (rstd) rstd[ROWS * unit + r] = rs[r];
            }
        }
        g.next();
    }
}

// Row by row; `part`: two partial rows (dgamma, dbeta) per block, [gridDim.x][2][d].
// gamma is in shared memory, the statistics of a warp's next 32 rows in its lanes.
template <class T, bool VEC, int NV>
__global__ void __launch_bounds__(kLnThreads, 1)
    ln_backward_kernel(const T *__restrict__ dy, const T *__restrict__ x, const float *__restrict__ gamma,
                       const float *__restrict__ mean, const float *__restrict__ rstd, T *__restrict__ dx,
                       float *__restrict__ part, const LnShape s, const LnRing ring, int *status) {
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(16) float red[2][2 * kLnRed * 4];
    __shared__ int abort_flag;
    griddep_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int grp = warp / s.warps, wr = warp - grp * s.warps;
    const LnLane<NV, VEC> l(wr, lane, s.warps, s.d);
    LnGroup<T, 2, VEC> g(ring, smem, grp, s.d);
    float *const sw = reinterpret_cast<float *>(smem);
    ln_init(g.bar0 - 8u * grp * ring.stages, ring.groups * ring.stages, &red[0][0], 4 * kLnRed * 4, &abort_flag);
    const int64_t stride = (int64_t)gridDim.x * ring.groups;
    int64_t row = (int64_t)blockIdx.x * ring.groups + grp, ahead = row;
    const bool leader = wr == 0 && lane == 0;
    auto issue = [&](int st, int64_t u) {
        g.issue(st, [&](int r) { return r == 0 ? x + u * s.x_ld : dy + u * s.g_ld; },
                [&](int r) { return r == 0 ? x : dy; },
                [&](int r) { return r == 0 ? x + (s.L - 1) * s.x_ld + s.d : dy + (s.L - 1) * s.g_ld + s.d; });
    };
    if (leader)
        for (int st = 0; st < ring.stages && ahead < s.L; ++st, ahead += stride) issue(st, ahead);
    for (int i = threadIdx.x; i < s.d; i += blockDim.x) sw[i] = __ldg(gamma + i);
    __syncthreads();
    F2 ag[NV][2], ab[NV][2];
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 2; ++e) ag[k][e] = ab[k][e] = f2(0.f, 0.f);
    bool ok = true;
    T *dxr = dx + row * s.y_ld;
    float mus = 0.f, rss = 0.f;
    for (int it = 0; row < s.L; ++it, row += stride, dxr += stride * s.y_ld) {
        if ((it & 31) == 0) {
            const int64_t r = row + lane * stride;
            mus = r < s.L ? __ldg(mean + r) : 0.f;
            rss = r < s.L ? __ldg(rstd + r) : 0.f;
        }
        const float mu = __shfl_sync(0xffffffffu, mus, it & 31), rs = __shfl_sync(0xffffffffu, rss, it & 31);
        if (ok) ok = g.wait(&abort_flag, status, leader, row, ahead, stride, s.L);
        const T *px = g.row(0, x + row * s.x_ld), *pg = g.row(1, dy + row * s.g_ld);
        const F2 nm = f2(-mu, -mu), r2 = f2(rs, rs);
        F2 xv[NV][2], gv[NV][2];
        F2 sums[2] = {f2(0.f, 0.f), f2(0.f, 0.f)};
        float c[2];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            F2 w[2];
            l.load(sw, k, w);
            l.load(px, k, xv[k]);
            l.load(pg, k, gv[k]);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                xv[k][e] = f2_mul(f2_add(xv[k][e], nm), r2);
                ag[k][e] = f2_fma(gv[k][e], xv[k][e], ag[k][e]);  // past the row: never stored
                ab[k][e] = f2_add(ab[k][e], gv[k][e]);
                gv[k][e] = f2_mul(gv[k][e], w[e]);
                const F2 t = l.counted(k, e, gv[k][e]);
                sums[0] = f2_add(sums[0], t);
                sums[1] = f2_fma(t, xv[k][e], sums[1]);
            }
        }
        ln_sums<2>(sums, c, s.warps, wr, lane, grp, red[it & 1] + 2 * grp * s.red_ld, s.red_ld);
        if (leader && ahead < s.L) {
            issue(g.stage, ahead);
            ahead += stride;
        }
        const float c1 = -c[0] * s.inv_d, c2 = -c[1] * s.inv_d;
        const F2 n1 = f2(c1, c1), n2 = f2(c2, c2);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
#pragma unroll
            for (int e = 0; e < 2; ++e) gv[k][e] = f2_mul(f2_add(gv[k][e], f2_fma(xv[k][e], n2, n1)), r2);
            l.store(dxr, k, gv[k]);
        }
        g.next();
    }
    // the groups' sums in group order (over gamma and the ring, which have been read), then
    // the block's partial rows
    __syncthreads();
    float *out = part + (int64_t)blockIdx.x * 2 * s.d;
    for (int q = 0; q < ring.groups; ++q) {
        if (q == grp) {
            float *const to = q == ring.groups - 1 ? out : sw;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                if (q > 0) {
                    F2 og[2], ob[2];
                    l.load(sw, k, og);
                    l.load(sw + s.d, k, ob);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        ag[k][e] = f2_add(og[e], ag[k][e]);
                        ab[k][e] = f2_add(ob[e], ab[k][e]);
                    }
                }
                l.store(to, k, ag[k]);
                l.store(to + s.d, k, ab[k]);
            }
        }
        if (ring.groups > 1) __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// Rows that no ring holds (d from about 16,000, backward 8,000, on): a block per row at
// a time, value by value, from L2 after the first read; the backward's sums stay in
// the block's partial rows.  2,048 rows x 20,480: bf16 67 us forward and 241 backward, fp32
// 94 and 259 (bytes: 25, 37, 49 and 74).
// ---------------------------------------------------------------------------

constexpr int kLnWide = 1024;

template <class T>
__global__ void __launch_bounds__(kLnWide)
    ln_forward_wide_kernel(const T *__restrict__ x, const float *__restrict__ gamma, const float *__restrict__ beta,
                           T *__restrict__ y, float *__restrict__ mean, float *__restrict__ rstd, const LnShape s) {
    __shared__ float red[2][32];
    const int wr = threadIdx.x >> 5, lane = threadIdx.x & 31;
    auto total = [&](float v, float *r) {
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (lane == 0) r[wr] = v;
        __syncthreads();
        v = r[lane];
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    };
    for (int64_t row = blockIdx.x; row < s.L; row += gridDim.x) {
        const T *xr = x + row * s.x_ld;
        float sum = 0.f, sq = 0.f;
        for (int c = threadIdx.x; c < s.d; c += kLnWide) sum += ln_value(xr[c]);
        const float mu = total(sum, red[0]) * s.inv_d;
        for (int c = threadIdx.x; c < s.d; c += kLnWide) {
            const float t = ln_value(xr[c]) - mu;
            sq = fmaf(t, t, sq);
        }
        const float rs = rsqrtf(fmaf(total(sq, red[1]), s.inv_d, s.eps));
        for (int c = threadIdx.x; c < s.d; c += kLnWide)
            ln_put(y + row * s.y_ld + c, fmaf((ln_value(xr[c]) - mu) * rs, __ldg(gamma + c), beta ? __ldg(beta + c) : 0.f));
        if (threadIdx.x == 0) {
            if (mean) mean[row] = mu;
            if (rstd) rstd[row] = rs;
        }
    }
}

template <class T>
__global__ void __launch_bounds__(kLnWide)
    ln_backward_wide_kernel(const T *__restrict__ dy, const T *__restrict__ x, const float *__restrict__ gamma,
                            const float *__restrict__ mean, const float *__restrict__ rstd, T *__restrict__ dx,
                            float *__restrict__ part, const LnShape s) {
    __shared__ float red[2][2][32];
    griddep_launch_dependents();
    const int wr = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float *out = part + (int64_t)blockIdx.x * 2 * s.d;
    for (int c = threadIdx.x; c < s.d; c += kLnWide) out[c] = out[s.d + c] = 0.f;
    int par = 0;
    for (int64_t row = blockIdx.x; row < s.L; row += gridDim.x, par ^= 1) {
        const T *xr = x + row * s.x_ld, *gr = dy + row * s.g_ld;
        const float mu = __ldg(mean + row), rs = __ldg(rstd + row);
        float a = 0.f, b = 0.f;
        for (int c = threadIdx.x; c < s.d; c += kLnWide) {
            const float xh = (ln_value(xr[c]) - mu) * rs, g = ln_value(gr[c]), t = g * __ldg(gamma + c);
            out[c] = fmaf(g, xh, out[c]);
            out[s.d + c] += g;
            a += t;
            b = fmaf(t, xh, b);
        }
        for (int o = 16; o > 0; o >>= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, o);
            b += __shfl_xor_sync(0xffffffffu, b, o);
        }
        if (lane == 0) {
            red[par][0][wr] = a;
            red[par][1][wr] = b;
        }
        __syncthreads();
        a = red[par][0][lane];
        b = red[par][1][lane];
        for (int o = 16; o > 0; o >>= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, o);
            b += __shfl_xor_sync(0xffffffffu, b, o);
        }
        const float c1 = a * s.inv_d, c2 = b * s.inv_d;
        for (int c = threadIdx.x; c < s.d; c += kLnWide) {
            const float xh = (ln_value(xr[c]) - mu) * rs;
            ln_put(dx + row * s.y_ld + c, rs * (ln_value(gr[c]) * __ldg(gamma + c) - fmaf(xh, c2, c1)));
        }
    }
}

// dgamma (blockIdx.y 0) and dbeta: 32 columns per block, its 16 warps each every 16th
// partial row, then the warps' sums in order.
constexpr int kLnSumWarps = 16;
__global__ void __launch_bounds__(32 * kLnSumWarps)
    ln_weight_sum_kernel(const float *__restrict__ part, int nparts, int d, float *dgamma, float *dbeta) {
    __shared__ float s_w[kLnSumWarps][32];
    griddep_wait();
    float *out = blockIdx.y == 0 ? dgamma : dbeta;
    if (!out) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int c = blockIdx.x * 32 + lane;
    float sum = 0.f;
    if (c < d) {
        const float *p = part + (int64_t)blockIdx.y * d + c;
        float v[kLnMaxBlocks / kLnSumWarps];  // all on their way at once
#pragma unroll
        for (int k = 0; k < kLnMaxBlocks / kLnSumWarps; ++k) {
            const int q = warp + k * kLnSumWarps;
            v[k] = q < nparts ? __ldcg(p + (int64_t)q * 2 * d) : 0.f;
        }
#pragma unroll
        for (int k = 0; k < kLnMaxBlocks / kLnSumWarps; ++k) sum += v[k];
    }
    s_w[warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && c < d) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < kLnSumWarps; ++w) t += s_w[w][lane];
        out[c] = t;
    }
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------

// How a call is cut; false where a row does not fit.  `rows` rows per place of the ring,
// `units` of them; most: vectors per thread.  The fewest warps per row that hold it:
// what a row costs beside its values, it costs per warp.
struct LnPlan {
    LnRing ring;
    int nv;
    unsigned blocks;
    size_t smem;
};

static bool ln_ring(LnShape *s, size_t esize, bool vec, int rows, bool gamma, int64_t units, int most, int sms,
                    LnPlan *p) {
    const int64_t warps = cdiv(s->d, 128 * most);
    if (32 * warps > kLnThreads) return false;
    p->nv = (int)cdiv(s->d, 128 * warps);
    LnRing &r = p->ring;
    r.place_bytes = (uint32_t)round_up(s->d * (int64_t)esize, 16) + (vec ? 0u : 16u);
    r.weight_bytes = gamma ? (uint32_t)round_up(4 * (int64_t)s->d, 16) : 0u;
    // a barrier of its own for each group: 15 beside the block's
    int64_t groups = warps == 1 ? kLnRed : std::min<int64_t>(kLnRed / warps, 15);
    groups = std::max<int64_t>(1, std::min<int64_t>(groups, cdiv(units, sms)));
    // places of two x rows leave L1 the rest: 34.0 us with 216 KB, 31.9 with 150, 40.8 with
    // 118 (8,192 x 5,120 bf16); the backward's take all (46.2 against 47.2)
    const int64_t room = (rows == 2 && !gamma ? 150 : 216) * 1024 - r.weight_bytes;
    const int64_t place = (int64_t)rows * r.place_bytes + 8;
    while (groups > 1 && room / (groups * place) < 3) --groups;
    r.groups = (int)groups;
    r.stages = (int)std::min<int64_t>({kLnStages, room / (groups * place), cdiv(units, groups * sms)});
    if (r.stages < 1) return false;
    s->warps = (int)warps;
    s->red_ld = (int)round_up(warps, 4);
    p->smem = r.weight_bytes + (size_t)groups * r.stages * place;
    if (gamma && groups > 1) p->smem = std::max(p->smem, 8 * (size_t)s->d);
    p->blocks = (unsigned)std::min<int64_t>(std::min(sms, kLnMaxBlocks), cdiv(units, groups));
    return true;
}

template <class T, bool VEC, int NV, bool KEEP, int ROWS>
static attt_status ln_forward_launch(const T *x, const float *gamma, const float *beta, T *y, float *mean, float *rstd,
                                     const LnShape &s, const LnPlan &p, int dev, cudaStream_t stream) {
    auto kern = ln_forward_kernel<T, VEC, NV, KEEP, ROWS>;
    int *status = device_status_word(dev);
    if (!status || !set_smem_limit(reinterpret_cast<const void *>(kern), p.smem, dev)) return ATTT_ERR_CUDA;
    kern<<<p.blocks, 32 * s.warps * p.ring.groups, p.smem, stream>>>(x, gamma, beta, y, mean, rstd, s, p.ring, status);
    count_launch();
    return cudaGetLastError() == cudaSuccess ? ATTT_OK : ATTT_ERR_CUDA;
}

template <class T, bool VEC>
static attt_status ln_forward_run(const T *x, const float *gamma, const float *beta, T *y, float *mean, float *rstd,
                                  LnShape s, int dev, cudaStream_t stream) {
    const int sms = num_sms(dev);
    LnPlan p{};
    // two rows at a time once every SM has several
    if (s.L >= 8 * (int64_t)sms && ln_ring(&s, sizeof(T), VEC, 2, false, cdiv(s.L, 2), 5, sms, &p) &&
        p.ring.stages >= 2) {
        switch (p.nv) {
            case 1: return ln_forward_launch<T, VEC, 1, true, 2>(x, gamma, beta, y, mean, rstd, s, p, dev, stream);
            case 2: return ln_forward_launch<T, VEC, 2, true, 2>(x, gamma, beta, y, mean, rstd, s, p, dev, stream);
            case 3: return ln_forward_launch<T, VEC, 3, true, 2>(x, gamma, beta, y, mean, rstd, s, p, dev, stream);
            case 4: return ln_forward_launch<T, VEC, 4, true, 2>(x, gamma, beta, y, mean, rstd, s, p, dev, stream);
            default: return ln_forward_launch<T, VEC, 5, true, 2>(x, gamma, beta, y, mean, rstd, s, p, dev, stream);
        }
    }
    // few rows: up to two vectors per thread, for the shorter chain
    if (ln_ring(&s, sizeof(T), VEC, 1, false, s.L, 2, sms, &p))
        return p.nv == 1 ? ln_forward_launch<T, VEC, 1, true, 1>(x, gamma, beta, y, mean, rstd, s, p, dev, stream)
                         : ln_forward_launch<T, VEC, 2, true, 1>(x, gamma, beta, y, mean, rstd, s, p, dev, stream);
    // longer rows (over 4,096 values) than that: always 5, and over 10,240 always 8
    if (ln_ring(&s, sizeof(T), VEC, 1, false, s.L, 5, sms, &p) && p.nv == 5)
        return ln_forward_launch<T, VEC, 5, true, 1>(x, gamma, beta, y, mean, rstd, s, p, dev, stream);
    if (ln_ring(&s, sizeof(T), VEC, 1, false, s.L, 8, sms, &p) && p.nv == 8)
        return ln_forward_launch<T, VEC, 8, false, 1>(x, gamma, beta, y, mean, rstd, s, p, dev, stream);
    ln_forward_wide_kernel<T><<<(unsigned)std::min<int64_t>(s.L, 2 * sms), kLnWide, 0, stream>>>(x, gamma, beta, y,
                                                                                                mean, rstd, s);
    count_launch();
    return cudaGetLastError() == cudaSuccess ? ATTT_OK : ATTT_ERR_CUDA;
}

template <class T, bool VEC, int NV>
static attt_status ln_backward_launch(const T *dy, const T *x, const float *gamma, const float *mean, const float *rstd,
                                      T *dx, float *part, const LnShape &s, const LnPlan &p, int dev,
                                      cudaStream_t stream) {
    auto kern = ln_backward_kernel<T, VEC, NV>;
    int *status = device_status_word(dev);
    if (!status || !set_smem_limit(reinterpret_cast<const void *>(kern), p.smem, dev)) return ATTT_ERR_CUDA;
    kern<<<p.blocks, 32 * s.warps * p.ring.groups, p.smem, stream>>>(dy, x, gamma, mean, rstd, dx, part, s, p.ring,
                                                                     status);
    count_launch();
    return cudaGetLastError() == cudaSuccess ? ATTT_OK : ATTT_ERR_CUDA;
}

// The rows' pass; *nparts: its partial rows.
template <class T, bool VEC>
static attt_status ln_backward_rows(const T *dy, const T *x, const float *gamma, const float *mean, const float *rstd,
                                    T *dx, float *part, LnShape s, int dev, cudaStream_t stream, int64_t *nparts) {
    const int sms = num_sms(dev);
    LnPlan p{};
    // 5 vectors of bf16 take all 128 registers, of fp32 or value by value more
    const int most = VEC && sizeof(T) == 2 ? 5 : 4;
    if (ln_ring(&s, sizeof(T), VEC, 2, true, s.L, s.L < 2 * (int64_t)sms ? 2 : most, sms, &p) ||
        ln_ring(&s, sizeof(T), VEC, 2, true, s.L, most, sms, &p)) {
        *nparts = p.blocks;
        switch (p.nv) {
            case 1: return ln_backward_launch<T, VEC, 1>(dy, x, gamma, mean, rstd, dx, part, s, p, dev, stream);
            case 2: return ln_backward_launch<T, VEC, 2>(dy, x, gamma, mean, rstd, dx, part, s, p, dev, stream);
            case 3: return ln_backward_launch<T, VEC, 3>(dy, x, gamma, mean, rstd, dx, part, s, p, dev, stream);
            case 4: return ln_backward_launch<T, VEC, 4>(dy, x, gamma, mean, rstd, dx, part, s, p, dev, stream);
        }
        if constexpr (VEC && sizeof(T) == 2)
            return ln_backward_launch<T, VEC, 5>(dy, x, gamma, mean, rstd, dx, part, s, p, dev, stream);
        return ATTT_ERR_UNSUPPORTED;  // most 4
    }
    *nparts = std::min<int64_t>({s.L, sms, kLnMaxBlocks});
    ln_backward_wide_kernel<T><<<(unsigned)*nparts, kLnWide, 0, stream>>>(dy, x, gamma, mean, rstd, dx, part, s);
    count_launch();
    return cudaGetLastError() == cudaSuccess ? ATTT_OK : ATTT_ERR_CUDA;
}

template <class T, bool VEC>
static attt_status ln_backward_run(const T *dy, const T *x, const float *gamma, const float *mean, const float *rstd,
                                   T *dx, float *dgamma, float *dbeta, float *part, const LnShape &s, int dev,
                                   cudaStream_t stream) {
    int64_t nparts = 0;
    if (s.L > 0) {
        const attt_status st = ln_backward_rows<T, VEC>(dy, x, gamma, mean, rstd, dx, part, s, dev, stream, &nparts);
        if (st != ATTT_OK) return st;
    }
    if (!dgamma && !dbeta) return ATTT_OK;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)cdiv(s.d, 32), 2);
    cfg.blockDim = dim3(32 * kLnSumWarps);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, ln_weight_sum_kernel, (const float *)part, (int)nparts, s.d, dgamma, dbeta) !=
        cudaSuccess)
        return ATTT_ERR_CUDA;
    count_launch();
    return cudaGetLastError() == cudaSuccess ? ATTT_OK : ATTT_ERR_CUDA;
}

static attt_status ln_sizes(int64_t L, int64_t d) {
    if (L < 0 || d < 1) return ATTT_ERR_INVALID_ARG;
    return L > (1ll << 31) - 1 || d > (1ll << 24) ? ATTT_ERR_UNSUPPORTED : ATTT_OK;
}
static bool ln_type(int dtype) { return dtype == ATTT_BF16 || dtype == ATTT_F32; }

// Whether rows from p, `ld` elements apart, lie on 16-byte boundaries from end to end.
static bool ln_vector(const void *p, int64_t ld, int64_t d, size_t esize) {
    return aligned16(p) && ld * esize % 16 == 0 && d * esize % 16 == 0;
}

}  // namespace attt

extern "C" {

attt_status attt_layer_norm_forward(const void *d_x, int64_t x_ld, const float *d_gamma, const float *d_beta,
                                    int64_t L, int64_t d, float eps, int dtype, void *d_y, int64_t y_ld, float *d_mean,
                                    float *d_rstd, attt_stream stream) {
    ATTT_NVTX_RANGE();
    using namespace attt;
    if (!ln_type(dtype) || !(eps >= 0.f) || x_ld < d || y_ld < d) return ATTT_ERR_INVALID_ARG;
    if (!d_gamma || (L > 0 && (!d_x || !d_y))) return ATTT_ERR_INVALID_ARG;
    const size_t es = dtype == ATTT_BF16 ? 2 : 4;
    if (!aligned_to(es, d_x, d_y) || !aligned_to(4, d_gamma, d_beta, d_mean, d_rstd)) return ATTT_ERR_INVALID_ARG;
    attt_status st = ln_sizes(L, d);
    if (st != ATTT_OK) return st;
    if (x_ld > (1ll << 36) || y_ld > (1ll << 36)) return ATTT_ERR_UNSUPPORTED;
    if (L == 0) return ATTT_OK;
    int dev;
    st = current_device(&dev);
    if (st != ATTT_OK) return st;
    LnShape s{};
    s.L = L; s.d = (int)d; s.x_ld = x_ld; s.y_ld = y_ld; s.eps = eps; s.inv_d = 1.f / (float)d;
    const bool vec = ln_vector(d_x, x_ld, d, es) && ln_vector(d_y, y_ld, d, es) && aligned16(d_gamma) &&
                     (!d_beta || aligned16(d_beta));
    if (dtype == ATTT_BF16) {
        const auto *x = static_cast<const __nv_bfloat16 *>(d_x);
        auto *y = static_cast<__nv_bfloat16 *>(d_y);
        return vec ? ln_forward_run<__nv_bfloat16, true>(x, d_gamma, d_beta, y, d_mean, d_rstd, s, dev, stream)
                   : ln_forward_run<__nv_bfloat16, false>(x, d_gamma, d_beta, y, d_mean, d_rstd, s, dev, stream);
    }
    const auto *x = static_cast<const float *>(d_x);
    auto *y = static_cast<float *>(d_y);
    return vec ? ln_forward_run<float, true>(x, d_gamma, d_beta, y, d_mean, d_rstd, s, dev, stream)
               : ln_forward_run<float, false>(x, d_gamma, d_beta, y, d_mean, d_rstd, s, dev, stream);
}

size_t attt_layer_norm_workspace_bytes(int64_t L, int64_t d) {
    if (attt::ln_sizes(L, d) != ATTT_OK) return 0;
    const int64_t rows = std::max<int64_t>(1, std::min<int64_t>(L, attt::kLnMaxBlocks));
    return (size_t)attt::round_up(rows * 2 * d * (int64_t)sizeof(float), 256);
}

attt_status attt_layer_norm_backward(const void *d_dy, int64_t dy_ld, const void *d_x, int64_t x_ld,
                                     const float *d_gamma, const float *d_mean, const float *d_rstd, int64_t L,
                                     int64_t d, int dtype, void *d_dx, int64_t dx_ld, float *d_dgamma, float *d_dbeta,
                                     void *d_ws, size_t ws_bytes, attt_stream stream) {
    ATTT_NVTX_RANGE();
    using namespace attt;
    if (!ln_type(dtype) || dy_ld < d || x_ld < d || dx_ld < d) return ATTT_ERR_INVALID_ARG;
    if (!d_gamma || (L > 0 && (!d_dy || !d_x || !d_mean || !d_rstd || !d_dx))) return ATTT_ERR_INVALID_ARG;
    const size_t es = dtype == ATTT_BF16 ? 2 : 4;
    if (!aligned_to(es, d_dy, d_x, d_dx) || !aligned_to(4, d_gamma, d_mean, d_rstd, d_dgamma, d_dbeta))
        return ATTT_ERR_INVALID_ARG;
    attt_status st = ln_sizes(L, d);
    if (st != ATTT_OK) return st;
    if (dy_ld > (1ll << 36) || x_ld > (1ll << 36) || dx_ld > (1ll << 36)) return ATTT_ERR_UNSUPPORTED;
    if (!d_ws || !aligned256(d_ws) || ws_bytes < attt_layer_norm_workspace_bytes(L, d)) return ATTT_ERR_WORKSPACE;
    int dev;
    st = current_device(&dev);
    if (st != ATTT_OK) return st;
    LnShape s{};
    s.L = L; s.d = (int)d; s.x_ld = x_ld; s.y_ld = dx_ld; s.g_ld = dy_ld; s.inv_d = 1.f / (float)d;
    const bool vec = ln_vector(d_x, x_ld, d, es) && ln_vector(d_dy, dy_ld, d, es) && ln_vector(d_dx, dx_ld, d, es);
    float *part = static_cast<float *>(d_ws);
    if (dtype == ATTT_BF16) {
        const auto *x = static_cast<const __nv_bfloat16 *>(d_x), *dy = static_cast<const __nv_bfloat16 *>(d_dy);
        auto *dx = static_cast<__nv_bfloat16 *>(d_dx);
        return vec ? ln_backward_run<__nv_bfloat16, true>(dy, x, d_gamma, d_mean, d_rstd, dx, d_dgamma, d_dbeta, part,
                                                          s, dev, stream)
                   : ln_backward_run<__nv_bfloat16, false>(dy, x, d_gamma, d_mean, d_rstd, dx, d_dgamma, d_dbeta, part,
                                                           s, dev, stream);
    }
    const auto *x = static_cast<const float *>(d_x), *dy = static_cast<const float *>(d_dy);
    auto *dx = static_cast<float *>(d_dx);
    return vec ? ln_backward_run<float, true>(dy, x, d_gamma, d_mean, d_rstd, dx, d_dgamma, d_dbeta, part, s, dev,
                                              stream)
               : ln_backward_run<float, false>(dy, x, d_gamma, d_mean, d_rstd, dx, d_dgamma, d_dbeta, part, s, dev,
                                               stream);
}

}  // extern "C"

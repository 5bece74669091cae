// Injection between two norms, forward and backward: the injection rule h' = h + g m (paper Sec. 2.2) with a norm on the memory
// vector, a learned gate (the paper: "scalar, vector, or learned function") and the norm that the next block starts with.
//
//   a = 1 / sqrt(mean(m^2) + eps)    y = w_post a m          s = gate or sigmoid(gate), 1 without a gate
//   u = h + lam s y                  b = 1 / sqrt(mean(u^2) + eps)        n = w_next b u
// With U, N the gradients that arrive at u and n, and t = w_next N:
//   dh = U + b t - b^3 u mean(u t)                           dw_next = sum over rows of N b u
//   ds = lam y dh  (summed over the columns for a scalar gate, times s (1 - s) for a sigmoid)
//   x = lam s w_post dh              dm = a x - a^3 m mean(m x)            dw_post = sum over rows of lam s dh a m
//
// HBM bounds both, and nearly as much the issue slots: 32,768 x 1,024 bf16 with a vector gate take 57 us forward (5.9 TB/s of the operands'
// bytes, 73 % of the slots) and 107 us backward (5.0 TB/s).  A row is held in the registers of `row_threads` threads, eight columns each, so every operand is read once and every
// intermediate stays on the chip; backward makes a, y, u and b again rather than reading them.  Several rows share a block, and a
// block walks rows with the next row's loads under way.  u is rounded once for the output, n and the gradients come from it as it was
// before.  The weights' gradients are summed over a block's rows in registers, over its groups in shared memory, and over the blocks
// by a second kernel: no atomics, the order depends on the sizes alone.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "../../include/tfe.h"
#include "tfe_internal.h"
#include "tfe_rows.cuh"

namespace {

using tfe_rows::Elem;

constexpr int kCols = 8, kPairs = kCols / 2;    // columns of a thread, taken in pairs: an instruction for two
constexpr int kBlock = 512;                     // threads of a block that holds several rows, at most
constexpr int kMaxBlocks = 592;                 // whatever the device has: bounds the partial sums of the backward pass

struct NormParams {
    int32_t Q, d;
    int32_t row_threads, groups;                // threads of a row, rows of a block at a time
    const void *h, *m, *gate; int64_t ld_h, ld_m, ld_gate;
    int32_t gate_kind, sigmoid, weights_f32;
    const void *w_post, *w_next;
    float lam, eps;
    void *out, *normed; int64_t ld_out, ld_normed;
    const void *g_out, *g_normed; int64_t ld_g_out, ld_g_normed;
    void *g_h, *g_m, *g_gate; int64_t ld_g_h, ld_g_m, ld_g_gate;
    float *part;                                // [blocks][2][d]: sums for w_post and w_next
};

// A thread's eight columns of a row as they were read: 8 t .. 8 t + 7 for thread t (kVector: 16-byte vectors), or t, t + row_threads, ...;
// beyond the row zeros, or with vectors the row's first columns (a thread is in the row with all of its columns or with none, and those
// that are not add nothing to a sum: see RowSum).
template <typename T, bool kVector>
struct Eight {
    static constexpr int kWords = (int)sizeof(T) * 2;
    uint32_t w[kWords];

    __device__ __forceinline__ void load(const void *base, int64_t ld, int64_t row, int32_t d, int t, int threads)
    {
        const T *at = static_cast<const T *>(base) + row * ld;
        if constexpr (kVector) {
            const int32_t c = kCols * t < d ? kCols * t : 0;
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i) {
                const uint4 v = tfe_rows::load_stream(reinterpret_cast<const uint4 *>(at + c) + i);
                w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int e = 0; e < kCols; ++e) {
                const int32_t c = t + e * threads;
                const bool in = c < d;
                if constexpr (sizeof(T) == 4) {
                    w[e] = in ? __float_as_uint(at[c]) : 0u;
                } else {
                    const uint32_t x = in ? (uint32_t)__bfloat16_as_ushort(at[c]) : 0u;
                    w[e / 2] = e & 1 ? w[e / 2] | (x << 16) : x;
                }
            }
        }
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0;
    }
    __device__ __forceinline__ float2 two(int i) const      // elements 2 i and 2 i + 1
    {
        if constexpr (sizeof(T) == 4) return make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
        else return make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
    }
};

template <typename T, bool kVector>
__device__ __forceinline__ void store(void *base, int64_t ld, int64_t row, int32_t d, int t, int threads, const float2 (&x)[kPairs])
{
    T *at = static_cast<T *>(base) + row * ld;
    if constexpr (kVector) {
        if (kCols * t >= d) return;
        uint4 *to = reinterpret_cast<uint4 *>(at + kCols * t);
        constexpr int E = Elem<T>::kPerVec;
#pragma unroll
        for (int i = 0; i < kCols / E; ++i) {
            float part[E];
#pragma unroll
            for (int e = 0; e < E; ++e) part[e] = e & 1 ? x[(i * E + e) / 2].y : x[(i * E + e) / 2].x;
            __stcs(to + i, Elem<T>::pack(part));
        }
    } else {
#pragma unroll
        for (int e = 0; e < kCols; ++e)
            if (t + e * threads < d) Elem<T>::put(at + t + e * threads, e & 1 ? x[e / 2].y : x[e / 2].x);
    }
}

template <bool kVector>
__device__ __forceinline__ int32_t column(int e, int t, int threads) { return kVector ? kCols * t + e : t + e * threads; }

template <bool kVector>
__device__ __forceinline__ void load_weight(const void *w, bool f32, int32_t d, int t, int threads, float2 (&x)[kPairs])
{
#pragma unroll
    for (int e = 0; e < kCols; ++e) {
        const int32_t c = column<kVector>(e, t, threads);
        const float v = c >= d ? 0.f : f32 ? static_cast<const float *>(w)[c] : __bfloat162float(static_cast<const __nv_bfloat16 *>(w)[c]);
        (e & 1 ? x[e / 2].y : x[e / 2].x) = v;
    }
}

// Sums over the threads of a row.  Each use needs a slot of its own until every thread has passed the next one's barrier: two in turn.
struct RowSum {
    float2 *slots;                              // [2][32] of this row's group
    int warps, warp, barrier, threads;
    bool in;                                    // this thread's columns are in the row
    int turn, span;                             // span: half the warps, rounded up to a power of two; 0 for one warp

    __device__ __forceinline__ RowSum(float2 *slots_, int group, int row_threads, int t, bool in_)
        : slots(slots_), warps(row_threads / 32), warp(t / 32), barrier(group + 1), threads(row_threads), in(in_), turn(0), span(0)
    {
        for (int w = 1; w < warps; w *= 2) span = w;
        if (t < 32) slots[t] = slots[32 + t] = make_float2(0.f, 0.f);
        asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(threads) : "memory");
    }

    __device__ __forceinline__ float2 shared(float2 x)
    {
        if (warps == 1) return x;
        float2 *s = slots + 32 * turn;          // (one layout for one sum and for two: what lies beyond the warps stays zero)
        turn ^= 1;
        if ((threadIdx.x & 31) == 0) s[warp] = x;
        asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(threads) : "memory");
        return s[threadIdx.x & (2 * span - 1)];
    }
    // one sum, or two
    __device__ __forceinline__ float operator()(float x)
    {
        x = in ? x : 0.f;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
        x = shared(make_float2(x, 0.f)).x;
        for (int o = span; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
        return x;
    }
    __device__ __forceinline__ float2 operator()(float x, float y)
    {
        x = in ? x : 0.f;
        y = in ? y : 0.f;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
            y += __shfl_xor_sync(0xFFFFFFFFu, y, o);
        }
        float2 two = shared(make_float2(x, y));
        for (int o = span; o > 0; o >>= 1) {
            two.x += __shfl_xor_sync(0xFFFFFFFFu, two.x, o);
            two.y += __shfl_xor_sync(0xFFFFFFFFu, two.y, o);
        }
        return two;
    }
};

// The approximate root, reciprocal and exponential are off by 2^-22 at most, which is less than the sums before them; the exact ones are
// sequences of instructions, and issue slots are what bounds these kernels next to HBM.
__device__ __forceinline__ float inverse_root(float square, float inv_d, float eps)
{
    float y;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(fmaf(square, inv_d, eps)));
    return y;
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 mul(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 fma(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }
__device__ __forceinline__ float join(float2 a) { return a.x + a.y; }
// s = 1 / (1 + e) of a gate x, e = exp(-x)
template <typename T>
__device__ __forceinline__ float sigmoid(float x, float &e)
{
    if constexpr (sizeof(T) == 4) {             // (an exponent of 15 alone costs the fast one 1e-6)
        e = expf(-x);
        return __fdividef(1.f, 1.f + e);
    }
    float y;
    e = tfe_rows::exp2_approx(x * -1.4426950408889634f);
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(1.f + e));
    return y;
}
// 1 - s for its derivative: as e s, since the subtraction loses every digit of an open gate (from x = 17 on it gives 0).  Where e is
// beyond fp32 s is 0, and so is the derivative.  16-bit rows hold it for a vector gate from the sigmoid on, fp32 rows make the sigmoid of
// -x where it is needed: gradients of 32,768 x 1,024 take 107 and 182 us so (111 and 208 the other way round).
__device__ __forceinline__ float shut(float e, float s) { return fminf(e, 0x1p126f) * s; }
template <typename T> constexpr bool kHoldShut = sizeof(T) == 2;

// A row's operands, and what both directions make of them first.
template <typename T, bool kVector>
struct Row {
    Eight<T, kVector> h, m, gate;
    float scalar;

    __device__ __forceinline__ void load(const NormParams &p, int64_t row, int t)
    {
        h.load(p.h, p.ld_h, row, p.d, t, p.row_threads);
        m.load(p.m, p.ld_m, row, p.d, t, p.row_threads);
        if (p.gate_kind == TFE_GATE_VECTOR) gate.load(p.gate, p.ld_gate, row, p.d, t, p.row_threads);
        scalar = p.gate_kind == TFE_GATE_SCALAR ? static_cast<const float *>(p.gate)[row] : 1.f;
    }
    // s, and for a sigmoid's derivative 1 - s of a vector gate (with kHoldShut), s (1 - s) of a scalar one
    __device__ __forceinline__ void gates(const NormParams &p, float2 (&s)[kPairs], float2 (&by)[kPairs], float &slope) const
    {
        float2 e;
        slope = 1.f;
        if (p.gate_kind == TFE_GATE_VECTOR) {
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
                s[i] = gate.two(i);
                if (p.sigmoid) {
                    s[i] = make_float2(sigmoid<T>(s[i].x, e.x), sigmoid<T>(s[i].y, e.y));
                    if constexpr (kHoldShut<T>) by[i] = make_float2(shut(e.x, s[i].x), shut(e.y, s[i].y));
                }
            }
        } else {
            float x = scalar;
            if (p.gate_kind == TFE_GATE_SCALAR && p.sigmoid) {
                x = sigmoid<T>(scalar, e.x);
                slope = x * shut(e.x, x);
            }
#pragma unroll
            for (int i = 0; i < kPairs; ++i) s[i] = both(x);
        }
    }
    __device__ __forceinline__ float square_m() const
    {
        float2 s = both(0.f);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) s = fma(m.two(i), m.two(i), s);
        return join(s);
    }
};

// Whether a thread has registers to hold the next row's operands beside this row's: 16-bit rows in blocks of up to kBlock threads.
// 32,768 x 1,024 with a vector gate, forward and backward: bf16 57 and 107 us with it, 62 and 129 without; fp32 117 and 198 with it, 108 and
// 182 without.
template <typename T, int kThreads> constexpr bool kAhead = sizeof(T) == 2 && kThreads <= kBlock;

template <typename T, bool kVector, int kThreads>
__global__ void __launch_bounds__(kThreads, kThreads <= kBlock ? 2 : 1)
tfe_inject_norm_forward_kernel(const NormParams p)
{
    __shared__ float2 s_slots[kThreads / 32][2][32];
    tfe_wait_for_stream();
    // (the same number in all lanes of a warp, and taken from one of them: the rows' addresses are then computed once per warp)
    const int group = __shfl_sync(0xFFFFFFFFu, (int)threadIdx.x / p.row_threads, 0), t = threadIdx.x - group * p.row_threads;
    RowSum row_sum(&s_slots[group][0][0], group, p.row_threads, t, !kVector || kCols * t < p.d);
    float2 wp[kPairs], wn[kPairs];
    load_weight<kVector>(p.w_post, p.weights_f32, p.d, t, p.row_threads, wp);
    load_weight<kVector>(p.w_next, p.weights_f32, p.d, t, p.row_threads, wn);
    const float inv_d = 1.f / (float)p.d;
    const int64_t step = (int64_t)gridDim.x * p.groups;
    int64_t row = (int64_t)blockIdx.x * p.groups + group;
    Row<T, kVector> x, next;
    if (kAhead<T, kThreads> && row < p.Q) next.load(p, row, t);
    for (; row < p.Q; row += step) {
        if constexpr (kAhead<T, kThreads>) {
            x = next;
            if (row + step < p.Q) next.load(p, row + step, t);
        } else {
            x.load(p, row, t);
        }
        const float a = inverse_root(row_sum(x.square_m()), inv_d, p.eps);
        float2 u[kPairs], by[kPairs], square = both(0.f);
        float slope;
        x.gates(p, u, by, slope);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            u[i] = fma(mul(u[i], both(p.lam * a)), mul(x.m.two(i), wp[i]), x.h.two(i));
            square = fma(u[i], u[i], square);
        }
        const float b = inverse_root(row_sum(join(square)), inv_d, p.eps);
        store<T, kVector>(p.out, p.ld_out, row, p.d, t, p.row_threads, u);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) u[i] = mul(mul(u[i], both(b)), wn[i]);
        store<T, kVector>(p.normed, p.ld_normed, row, p.d, t, p.row_threads, u);
    }
}

template <typename T, bool kVector, int kThreads>
__global__ void __launch_bounds__(kThreads, 1)
tfe_inject_norm_backward_kernel(const NormParams p)
{
    __shared__ float2 s_slots[kThreads / 32][2][32];
    extern __shared__ float s_sum[];            // [2][d], for several groups
    tfe_wait_for_stream();
    // (the same number in all lanes of a warp, and taken from one of them: the rows' addresses are then computed once per warp)
    const int group = __shfl_sync(0xFFFFFFFFu, (int)threadIdx.x / p.row_threads, 0), t = threadIdx.x - group * p.row_threads;
    RowSum row_sum(&s_slots[group][0][0], group, p.row_threads, t, !kVector || kCols * t < p.d);
    float2 wp[kPairs], wn[kPairs], sum_p[kPairs], sum_n[kPairs];
    load_weight<kVector>(p.w_post, p.weights_f32, p.d, t, p.row_threads, wp);
    load_weight<kVector>(p.w_next, p.weights_f32, p.d, t, p.row_threads, wn);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) sum_p[i] = sum_n[i] = both(0.f);
    const float inv_d = 1.f / (float)p.d;
    const int64_t step = (int64_t)gridDim.x * p.groups;
    int64_t row = (int64_t)blockIdx.x * p.groups + group;
    struct All {
        Row<T, kVector> x;
        Eight<T, kVector> gu, gn;
        __device__ __forceinline__ void load(const NormParams &p, int64_t r, int t)
        {
            x.load(p, r, t);
            if (p.g_out) gu.load(p.g_out, p.ld_g_out, r, p.d, t, p.row_threads); else gu.zero();
            if (p.g_normed) gn.load(p.g_normed, p.ld_g_normed, r, p.d, t, p.row_threads); else gn.zero();
        }
    };
    All all, next;
    if (kAhead<T, kThreads> && row < p.Q) next.load(p, row, t);
    for (; row < p.Q; row += step) {
        if constexpr (kAhead<T, kThreads>) {
            all = next;
            if (row + step < p.Q) next.load(p, row + step, t);
        } else {
            all.load(p, row, t);
        }
        const Row<T, kVector> &x = all.x;
        const float a = inverse_root(row_sum(x.square_m()), inv_d, p.eps);
        const float la = p.lam * a;
        float2 s[kPairs], by[kPairs], q[kPairs], u[kPairs], uu = both(0.f), ut = both(0.f);
        float slope;
        x.gates(p, s, by, slope);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            q[i] = mul(x.m.two(i), wp[i]);      // y / a
            u[i] = fma(mul(s[i], both(la)), q[i], x.h.two(i));
            uu = fma(u[i], u[i], uu);
            ut = fma(u[i], mul(wn[i], all.gn.two(i)), ut);
        }
        const float2 two = row_sum(join(uu), join(ut));
        const float b = inverse_root(two.x, inv_d, p.eps), by_u = b * (b * (two.y * inv_d));      // (products in an order that stays within fp32 as long as b does)
        float2 sdh[kPairs], mx = both(0.f), uy = both(0.f);         // sdh: s dh; mx, uy and sum_p without their factors lam and a
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            const float2 bu = mul(u[i], both(b));
            sum_n[i] = fma(all.gn.two(i), bu, sum_n[i]);
            u[i] = fma(both(-by_u), bu, fma(mul(all.gn.two(i), both(b)), wn[i], all.gu.two(i)));      // dh
            sdh[i] = mul(s[i], u[i]);
            sum_p[i] = fma(sdh[i], mul(x.m.two(i), both(a)), sum_p[i]);
            mx = fma(q[i], sdh[i], mx);
        }
        if (p.g_h) store<T, kVector>(p.g_h, p.ld_g_h, row, p.d, t, p.row_threads, u);
        if (p.g_gate && p.gate_kind == TFE_GATE_SCALAR) {
#pragma unroll
            for (int i = 0; i < kPairs; ++i) uy = fma(u[i], q[i], uy);
            const float dot = row_sum(join(uy));
            if (t == 0) static_cast<float *>(p.g_gate)[row] = la * dot * slope;
        }
        if (p.g_m) {
            const float by_m = a * (a * (row_sum(join(mx)) * inv_d));
            float2 dm[kPairs];
#pragma unroll
            for (int i = 0; i < kPairs; ++i) dm[i] = mul(fma(both(-by_m), x.m.two(i), mul(wp[i], sdh[i])), both(la));
            store<T, kVector>(p.g_m, p.ld_g_m, row, p.d, t, p.row_threads, dm);
        }
        if (p.g_gate && p.gate_kind == TFE_GATE_VECTOR) {
#pragma unroll
            for (int i = 0; i < kPairs; ++i) q[i] = mul(q[i], both(la));
            if (p.sigmoid) {
#pragma unroll
                for (int i = 0; i < kPairs; ++i) {
                    if constexpr (!kHoldShut<T>) {
                        float2 e;
                        const float2 g = x.gate.two(i);
                        by[i] = make_float2(sigmoid<T>(-g.x, e.x), sigmoid<T>(-g.y, e.y));
                    }
                    q[i] = mul(q[i], mul(sdh[i], by[i]));
                }
            } else {
#pragma unroll
                for (int i = 0; i < kPairs; ++i) q[i] = mul(q[i], u[i]);
            }
            store<T, kVector>(p.g_gate, p.ld_g_gate, row, p.d, t, p.row_threads, q);
        }
    }
#pragma unroll
    for (int i = 0; i < kPairs; ++i) sum_p[i] = mul(sum_p[i], both(p.lam));
    if (!p.part) return;
    float *to = p.groups > 1 ? s_sum : p.part + (int64_t)blockIdx.x * 2 * p.d;
    for (int g = 0; g < p.groups; ++g) {
        if (group == g)
#pragma unroll
            for (int e = 0; e < kCols; ++e) {
                const int32_t c = column<kVector>(e, t, p.row_threads);
                const float sp = e & 1 ? sum_p[e / 2].y : sum_p[e / 2].x, sn = e & 1 ? sum_n[e / 2].y : sum_n[e / 2].x;
                if (c < p.d) {
                    to[c] = g == 0 ? sp : to[c] + sp;
                    to[p.d + c] = g == 0 ? sn : to[p.d + c] + sn;
                }
            }
        if (p.groups > 1) __syncthreads();
    }
    if (p.groups > 1)
        for (int32_t c = threadIdx.x; c < 2 * p.d; c += blockDim.x) p.part[(int64_t)blockIdx.x * 2 * p.d + c] = s_sum[c];
}

struct JoinParams {
    int32_t blocks, d, f32;
    const float *part;
    void *g_post, *g_next;
};
constexpr int kJoinCols = 32, kJoinParts = 32;

__global__ void __launch_bounds__(kJoinCols * kJoinParts)
tfe_inject_norm_join_kernel(const JoinParams p)
{
    __shared__ float s_sum[kJoinParts][kJoinCols + 1];
    tfe_wait_for_stream();
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
    const int32_t c = blockIdx.x * kJoinCols + lane;
    float sum = 0.f;
    if (c < 2 * p.d)
#pragma unroll 4
        for (int32_t b = part; b < p.blocks; b += kJoinParts) sum += p.part[(int64_t)b * 2 * p.d + c];
    s_sum[part][lane] = sum;
    __syncthreads();
    sum = s_sum[lane][part];                    // column `part` now, from 32 parts
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    const int32_t mine = blockIdx.x * kJoinCols + part;
    if (lane != 0 || mine >= 2 * p.d) return;
    void *to = mine < p.d ? p.g_post : p.g_next;
    if (!to) return;
    if (p.f32) static_cast<float *>(to)[mine % p.d] = sum;
    else static_cast<__nv_bfloat16 *>(to)[mine % p.d] = __float2bfloat16_rn(sum);
}

// ------------------------------------------------------------------ host side

struct Matrix { const void *at; int64_t ld; };

int64_t elem_size(int32_t dtype) { return dtype == TFE_DTYPE_BF16 ? 2 : 4; }
bool aligned(const void *p, uintptr_t to) { return p && reinterpret_cast<uintptr_t>(p) % to == 0; }
bool matrix_ok(const void *at, int64_t ld, int32_t d, int64_t es) { return aligned(at, es) && ld >= d && ld <= (1ll << 34); }

struct Span { const void *at; int64_t bytes; };
bool touch(const Span &a, const Span &b)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
    return a.at && b.at && x < y + (uintptr_t)b.bytes && y < x + (uintptr_t)a.bytes;
}

bool params_ok(const tfe_inject_norm_params *q)
{
    if (!q || (q->dtype != TFE_DTYPE_BF16 && q->dtype != TFE_DTYPE_F32) || (q->weight_dtype != TFE_DTYPE_BF16 && q->weight_dtype != TFE_DTYPE_F32)) return false;
    if (q->Q < 0 || q->Q > TFE_ROWS_MAX || q->d < 1 || q->d > TFE_INJECT_NORM_MAX_COLS) return false;
    if (q->gate_kind < TFE_GATE_NONE || q->gate_kind > TFE_GATE_VECTOR) return false;
    if (!(q->eps >= 0.f) || !(q->eps <= 1.f) || !(q->lam - q->lam == 0.f)) return false;
    const int64_t ws = elem_size(q->weight_dtype);
    if (!aligned(q->post_weight, ws) || !aligned(q->next_weight, ws)) return false;
    if (q->Q == 0) return true;
    const int64_t es = elem_size(q->dtype);
    if (!matrix_ok(q->h, q->ld_h, q->d, es) || !matrix_ok(q->m, q->ld_m, q->d, es)) return false;
    if (q->gate_kind == TFE_GATE_SCALAR && !aligned(q->gate, 4)) return false;
    if (q->gate_kind == TFE_GATE_VECTOR && !matrix_ok(q->gate, q->ld_gate, q->d, es)) return false;
    return true;
}

NormParams shared_params(const tfe_inject_norm_params *q)
{
    NormParams p{};
    p.Q = q->Q; p.d = q->d; p.h = q->h; p.m = q->m; p.gate = q->gate; p.ld_h = q->ld_h; p.ld_m = q->ld_m; p.ld_gate = q->ld_gate;
    p.gate_kind = q->gate_kind; p.sigmoid = q->sigmoid != 0; p.weights_f32 = q->weight_dtype == TFE_DTYPE_F32;
    p.w_post = q->post_weight; p.w_next = q->next_weight; p.lam = q->lam; p.eps = q->eps;
    p.row_threads = (q->d + 32 * kCols - 1) / (32 * kCols) * 32;
    return p;
}
int64_t span(int32_t Q, int64_t ld, int32_t d, int64_t es) { return ((int64_t)(Q - 1) * ld + d) * es; }

tfe_status device_sms(int *sms)
{
    int dev = 0;
    tfe_status st = tfe_note_cuda(cudaGetDevice(&dev), "cudaGetDevice");
    return st != TFE_OK ? st : tfe_note_cuda(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev), "cudaDeviceGetAttribute");
}

// Rows of a block at a time, and the blocks.  Few rows are spread over the SMs.
int plan_blocks(NormParams &p, int sms, int per_sm)
{
    p.groups = std::max(1, std::min({kBlock / p.row_threads, 15, (p.Q + sms - 1) / sms}));      // (named barriers 1..15)
    return (int)std::min<int64_t>({((int64_t)p.Q + p.groups - 1) / p.groups, (int64_t)sms * per_sm, (int64_t)kMaxBlocks});
}

template <typename F>
tfe_status pick(int32_t dtype, bool vec, bool wide, F go)
{
    if (dtype == TFE_DTYPE_BF16)
        return vec ? (wide ? go.template operator()<__nv_bfloat16, true, 1024>() : go.template operator()<__nv_bfloat16, true, kBlock>())
                   : (wide ? go.template operator()<__nv_bfloat16, false, 1024>() : go.template operator()<__nv_bfloat16, false, kBlock>());
    return vec ? (wide ? go.template operator()<float, true, 1024>() : go.template operator()<float, true, kBlock>())
               : (wide ? go.template operator()<float, false, 1024>() : go.template operator()<float, false, kBlock>());
}

struct GoForward {
    NormParams p; int grid; cudaStream_t stream;
    template <typename T, bool kVector, int kThreads> tfe_status operator()() const
    {
        return tfe_launch_serial(tfe_inject_norm_forward_kernel<T, kVector, kThreads>, (unsigned)grid, (unsigned)(p.row_threads * p.groups), 1, 0, stream,
                                 "injection launch", p);
    }
};
struct GoBackward {
    NormParams p; int grid; cudaStream_t stream;
    template <typename T, bool kVector, int kThreads> tfe_status operator()() const
    {
        const size_t smem = p.groups > 1 ? (size_t)2 * p.d * sizeof(float) : 0;
        return tfe_launch_serial(tfe_inject_norm_backward_kernel<T, kVector, kThreads>, (unsigned)grid, (unsigned)(p.row_threads * p.groups), 1, smem, stream,
                                 "injection gradient launch", p);
    }
};

// 16-byte vectors where every row of every matrix starts on such a boundary
bool vectors(int32_t dtype, int32_t d, std::initializer_list<Matrix> all)
{
    if (d % kCols != 0) return false;
    for (const Matrix &x : all)
        if (x.at && (reinterpret_cast<uintptr_t>(x.at) % 16 != 0 || x.ld * elem_size(dtype) % 16 != 0)) return false;
    return true;
}

}  // namespace

extern "C" {

tfe_status tfe_inject_norm_forward(const tfe_inject_norm_params *q, void *out, int64_t ld_out, void *normed, int64_t ld_normed, void *stream_)
{
    if (!params_ok(q)) return TFE_ERR_INVALID_ARG;
    if (q->Q == 0) return TFE_OK;
    const int64_t es = elem_size(q->dtype);
    if (!matrix_ok(out, ld_out, q->d, es) || !matrix_ok(normed, ld_normed, q->d, es)) return TFE_ERR_INVALID_ARG;
    const int64_t ws = elem_size(q->weight_dtype) * q->d;
    const Span o{out, span(q->Q, ld_out, q->d, es)}, n{normed, span(q->Q, ld_normed, q->d, es)}, h{q->h, span(q->Q, q->ld_h, q->d, es)};
    const Span gate{q->gate_kind == TFE_GATE_NONE ? nullptr : q->gate, q->gate_kind == TFE_GATE_SCALAR ? 4ll * q->Q : span(q->Q, q->ld_gate, q->d, es)};
    const Span others[] = {{q->m, span(q->Q, q->ld_m, q->d, es)}, gate, {q->post_weight, ws}, {q->next_weight, ws}};
    for (const Span &x : others)
        if (touch(o, x) || touch(n, x)) return TFE_ERR_INVALID_ARG;
    // out may be h itself: a row is read before it is written
    if (touch(o, n) || touch(n, h) || (touch(o, h) && !(out == q->h && ld_out == q->ld_h))) return TFE_ERR_INVALID_ARG;
    int sms = 0;
    if (tfe_status st = device_sms(&sms)) return st;
    NormParams p = shared_params(q);
    p.out = out; p.ld_out = ld_out; p.normed = normed; p.ld_normed = ld_normed;
    const int grid = plan_blocks(p, sms, 4);
    const bool vec = vectors(q->dtype, q->d, {{q->h, q->ld_h}, {q->m, q->ld_m}, {q->gate_kind == TFE_GATE_VECTOR ? q->gate : nullptr, q->ld_gate}, {out, ld_out}, {normed, ld_normed}});
    return pick(q->dtype, vec, p.row_threads > kBlock, GoForward{p, grid, static_cast<cudaStream_t>(stream_)});
}

int64_t tfe_inject_norm_workspace_bytes(int32_t Q, int32_t d)
{
    if (Q < 0 || Q > TFE_ROWS_MAX || d < 1 || d > TFE_INJECT_NORM_MAX_COLS) return -1;
    return std::min<int64_t>(Q, kMaxBlocks) * 2 * d * (int64_t)sizeof(float);
}

tfe_status tfe_inject_norm_backward(const tfe_inject_norm_params *q, const tfe_inject_norm_grads *g, void *workspace, int64_t workspace_bytes, void *stream_)
{
    if (!params_ok(q) || !g) return TFE_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const int64_t es = elem_size(q->dtype), wes = elem_size(q->weight_dtype), ws = wes * q->d;
    if ((g->grad_post && !aligned(g->grad_post, wes)) || (g->grad_next && !aligned(g->grad_next, wes))) return TFE_ERR_INVALID_ARG;
    if (q->Q == 0) {                            // sums over no rows
        if (g->grad_post)
            if (tfe_status st = tfe_note_cuda(cudaMemsetAsync(g->grad_post, 0, (size_t)ws, stream), "cudaMemsetAsync")) return st;
        return g->grad_next ? tfe_note_cuda(cudaMemsetAsync(g->grad_next, 0, (size_t)ws, stream), "cudaMemsetAsync") : TFE_OK;
    }
    const bool scalar = q->gate_kind == TFE_GATE_SCALAR, vector = q->gate_kind == TFE_GATE_VECTOR;
    if (!g->grad_out && !g->grad_normed) return TFE_ERR_INVALID_ARG;
    if ((g->grad_out && !matrix_ok(g->grad_out, g->ld_grad_out, q->d, es)) || (g->grad_normed && !matrix_ok(g->grad_normed, g->ld_grad_normed, q->d, es)))
        return TFE_ERR_INVALID_ARG;
    if ((g->grad_h && !matrix_ok(g->grad_h, g->ld_grad_h, q->d, es)) || (g->grad_m && !matrix_ok(g->grad_m, g->ld_grad_m, q->d, es))) return TFE_ERR_INVALID_ARG;
    if (g->grad_gate && !(scalar ? aligned(g->grad_gate, 4) : vector && matrix_ok(g->grad_gate, g->ld_grad_gate, q->d, es))) return TFE_ERR_INVALID_ARG;
    const bool sums = g->grad_post || g->grad_next;
    const int64_t need = tfe_inject_norm_workspace_bytes(q->Q, q->d);
    if (sums && !aligned(workspace, 16)) return TFE_ERR_INVALID_ARG;
    if (sums && workspace_bytes < need) return TFE_ERR_CAPACITY;
    const Span in[] = {{q->h, span(q->Q, q->ld_h, q->d, es)}, {q->m, span(q->Q, q->ld_m, q->d, es)},
                       {q->gate_kind == TFE_GATE_NONE ? nullptr : q->gate, scalar ? 4ll * q->Q : span(q->Q, q->ld_gate, q->d, es)},
                       {q->post_weight, ws}, {q->next_weight, ws}, {g->grad_out, span(q->Q, g->ld_grad_out, q->d, es)},
                       {g->grad_normed, span(q->Q, g->ld_grad_normed, q->d, es)}, {sums ? workspace : nullptr, need}};
    const Span made[] = {{g->grad_h, span(q->Q, g->ld_grad_h, q->d, es)}, {g->grad_m, span(q->Q, g->ld_grad_m, q->d, es)},
                         {g->grad_gate, scalar ? 4ll * q->Q : span(q->Q, g->ld_grad_gate, q->d, es)}, {g->grad_post, ws}, {g->grad_next, ws}};
    for (int i = 0; i < 5; ++i) {
        for (const Span &x : in)
            if (touch(made[i], x)) return TFE_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (touch(made[i], made[j])) return TFE_ERR_INVALID_ARG;
    }
    int sms = 0;
    if (tfe_status st = device_sms(&sms)) return st;
    NormParams p = shared_params(q);
    p.g_out = g->grad_out; p.ld_g_out = g->ld_grad_out; p.g_normed = g->grad_normed; p.ld_g_normed = g->ld_grad_normed;
    p.g_h = g->grad_h; p.ld_g_h = g->ld_grad_h; p.g_m = g->grad_m; p.ld_g_m = g->ld_grad_m; p.g_gate = g->grad_gate; p.ld_g_gate = g->ld_grad_gate;
    p.part = sums ? static_cast<float *>(workspace) : nullptr;
    const int grid = plan_blocks(p, sms, 1);
    const bool vec = vectors(q->dtype, q->d, {{q->h, q->ld_h}, {q->m, q->ld_m}, {vector ? q->gate : nullptr, q->ld_gate}, {g->grad_out, g->ld_grad_out},
                                              {g->grad_normed, g->ld_grad_normed}, {g->grad_h, g->ld_grad_h}, {g->grad_m, g->ld_grad_m},
                                              {vector ? g->grad_gate : nullptr, g->ld_grad_gate}});
    if (tfe_status st = pick(q->dtype, vec, p.row_threads > kBlock, GoBackward{p, grid, stream})) return st;
    if (!sums) return TFE_OK;
    JoinParams j{};
    j.blocks = grid; j.d = q->d; j.f32 = p.weights_f32; j.part = p.part; j.g_post = g->grad_post; j.g_next = g->grad_next;
    return tfe_launch_serial(tfe_inject_norm_join_kernel, (unsigned)((2 * q->d + kJoinCols - 1) / kJoinCols), kJoinCols * kJoinParts, 1, 0, stream, "injection join launch", j);
}

}  // extern "C"

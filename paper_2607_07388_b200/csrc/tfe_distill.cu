// Distillation of a teacher's top logits into a predictor over the whole vocabulary: the loss that trains an early-exit
// projection (paper Sec. 4.4: W_pref predicts the full model's next tokens) and its gradient.
//
// Per row, with student logits z[0..V), teacher entries (id_k, t_k), k < K, and temperature tau:
//     lse  = ln sum_v exp(z_v / tau)                          q = softmax over the valid k of t_k / tau
//     loss = tau^2 sum_k q_k (ln q_k - z[id_k] / tau + lse)   (tau^2 times the divergence from q to the student)
//     grad = g tau (exp(z_v / tau - lse) - sum of q_k with id_k = v)
//
//   tfe_distill_forward_kernel   one pass over the row: running maximum and sum of exponentials.  A row is taken by a
//                                warp, by a block, or by a cluster of blocks whose partial results meet in the shared
//                                memory of the first.  A warp of the row's first block does the K teacher entries in
//                                64 bits while the others stream.
//   tfe_distill_backward_kernel  one pass: read the logit, write the gradient.  A block owns its slice of the row, so
//                                the entries with a teacher weight are corrected by the block itself after its stream
//                                (equal ids are summed by the first of them, in order: no atomics), from logits it
//                                saved before; the gradient may therefore overwrite the logits.
//
// Both are bound by HBM.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "../../include/tfe.h"
#include "tfe_internal.h"
#include "tfe_rows.cuh"

namespace {

using namespace tfe_rows;
namespace cg = cooperative_groups;

constexpr int kBlock = 512;             // threads of a block that takes (a slice of) one row
constexpr int kSmallBlock = 256;        // ... and of one whose warps take a row each
constexpr int kMaxTop = TFE_DISTILL_MAX_TOP;
constexpr double kLog2e = 1.4426950408889634;

struct DistillParams {
    const void *logits; int64_t ld;
    int32_t N, V, K;
    float tau;
    const int32_t *ids; const float *t;
    float *loss, *lse;                  // forward
    const float *lse_in, *grad_loss;    // backward
    void *grad; int64_t ld_grad;
    int32_t slices;                     // blocks per row
};

__device__ __forceinline__ bool teacher_valid(int32_t id, int32_t V) { return id >= 0 && id < V; }

// A warp's view of a row's teacher entries: the largest valid t and sum of exp((t - largest) / tau).  NaN among the
// valid entries makes the sum NaN.  No valid entry, or all of them -inf: sum 0.
__device__ __forceinline__ void teacher_norm(const DistillParams &p, int64_t row, int lane, float &top, double &sum)
{
    top = -INFINITY;
    const int64_t at = row * p.K;
    for (int k = lane; k < p.K; k += 32)
        if (teacher_valid(p.ids[at + k], p.V)) top = fmaxf(top, p.t[at + k]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    sum = 0.0;
    for (int k = lane; k < p.K; k += 32)
        if (teacher_valid(p.ids[at + k], p.V)) {
            const float t = p.t[at + k];
            if (t != -INFINITY) sum += exp(((double)t - (double)top) / (double)p.tau);
        }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
}

// Running maximum and sum of exponentials of a thread's logits: m is the largest logit (the mask value before any), s the
// sum of exp2(z c - ref(m)).  The reference is the rounded product m c, which is known again wherever m is: what the rounding
// of c and of the product would do to the result is taken back exactly at the end (see finish_row), and a term costs one
// fused multiply-add and one exponential.
__device__ __forceinline__ float ref(float m, float c) { return __fmul_rn(m, c); }
__device__ __forceinline__ void fold(float &m, float &s, float m2, float s2, float c)
{
    const float top = fmaxf(m, m2);
    s = s * exp2_approx(ref(m, c) - ref(top, c)) + s2 * exp2_approx(ref(m2, c) - ref(top, c));
    m = top;
}

// The largest value of a vector; NaN does not count (its exponential makes the sum NaN).
template <typename T>
__device__ __forceinline__ float vector_max(const uint4 &raw)
{
    if constexpr (sizeof(T) == 2) {                     // in pairs
        const __nv_bfloat162 a = *reinterpret_cast<const __nv_bfloat162 *>(&raw.x), b = *reinterpret_cast<const __nv_bfloat162 *>(&raw.y);
        const __nv_bfloat162 d = *reinterpret_cast<const __nv_bfloat162 *>(&raw.z), e = *reinterpret_cast<const __nv_bfloat162 *>(&raw.w);
        const __nv_bfloat162 h = __hmax2(__hmax2(a, b), __hmax2(d, e));
        return fmaxf(__low2float(h), __high2float(h));
    } else {
        return fmaxf(fmaxf(__uint_as_float(raw.x), __uint_as_float(raw.y)), fmaxf(__uint_as_float(raw.z), __uint_as_float(raw.w)));
    }
}

// This thread's elements of a slice.  2,048 rows of 151,936 bf16 logits take 107 us with pairs of fused operations (16 exponentials
// per clock and SM alone would take 69 us), 137 us with single subtractions and products.
template <typename T, int U>
__device__ __forceinline__ void stream_row(const T *row, int64_t n, int slice, int slices, int tid, int threads, float c, float &m, float &s)
{
    constexpr int E = Elem<T>::kPerVec;
    const Cut cut = cut_row(row, n);
    const uint4 *body = reinterpret_cast<const uint4 *>(row + cut.head);
    const int64_t v0 = cut.n_vec * slice / slices, v1 = cut.n_vec * (slice + 1) / slices;
    m = kMasked;
    float2 sum = make_float2(0.f, 0.f);
    float minus = -ref(m, c);
    auto raise = [&](float top) {
        if (top > m) {
            const float scale = exp2_approx(-minus - ref(top, c));
            sum.x *= scale; sum.y *= scale;
            m = top;
            minus = -ref(m, c);
        }
    };
    auto add = [&](const uint4 &raw) {
        float f[E];
        Elem<T>::unpack(raw, f);
        const float2 cc = make_float2(c, c), mm = make_float2(minus, minus);
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            const float2 x = __ffma2_rn(make_float2(f[e], f[e + 1]), cc, mm);
            sum = __fadd2_rn(sum, make_float2(exp2_approx(x.x), exp2_approx(x.y)));
        }
    };
    auto take = [&](float z) {
        raise(z);
        sum.x += exp2_approx(fmaf(z, c, minus));
    };
    if (slice == 0) for (int64_t i = tid; i < cut.head; i += threads) take(Elem<T>::get(row + i));
    if (slice == slices - 1)
        for (int64_t i = cut.head + cut.n_vec * E + tid; i < n; i += threads) take(Elem<T>::get(row + i));
    int64_t v = v0 + tid;
    for (; v + (int64_t)(U - 1) * threads < v1; v += (int64_t)U * threads) {
        uint4 raw[U];
        float top[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = load_stream(body + v + (int64_t)u * threads);
#pragma unroll
        for (int u = 0; u < U; ++u) top[u] = vector_max<T>(raw[u]);
#pragma unroll
        for (int u = 1; u < U; ++u) top[0] = fmaxf(top[0], top[u]);
        raise(top[0]);
#pragma unroll
        for (int u = 0; u < U; ++u) add(raw[u]);
    }
    for (; v < v1; v += threads) {
        const uint4 raw = load_stream(body + v);
        raise(vector_max<T>(raw));
        add(raw);
    }
    s = sum.x + sum.y;
}

// The rounding of a reference beyond this is whole powers of two of every term, which leave fp32 from about 2^31 on (logits of -1e10
// where a mask has left nothing, say): such a row is summed once more, relative to its largest logit itself.
constexpr float kFarRef = 0x1p24f;
__device__ __forceinline__ bool far_row(float m, float c) { return m > kMasked && fabsf(ref(m, c)) >= kFarRef; }
template <typename T>
__device__ __noinline__ float far_sum(const T *row, int64_t n, int slice, int slices, int tid, int threads, float c, float m)
{
    const int64_t e0 = n * slice / slices, e1 = n * (slice + 1) / slices;
    float s = 0.f;
    for (int64_t i = e0 + tid; i < e1; i += threads) s += exp2_approx((Elem<T>::get(row + i) - m) * c);
    return s;
}

// sum_k q_k (ln q_k - z[id_k] / tau) in 64 bits, on every lane; +inf where a teacher weight meets a masked logit
template <typename T>
__device__ __forceinline__ double teacher_term(const DistillParams &p, const T *row, int64_t r, int lane, bool &any)
{
    float top;
    double sum;
    teacher_norm(p, r, lane, top, sum);
    any = !(sum == 0.0);
    if (!any) return 0.0;
    const double log_sum = log(sum);
    double term = 0.0;
    const int64_t at = r * p.K;
    for (int k = lane; k < p.K; k += 32) {
        const int32_t id = p.ids[at + k];
        if (!teacher_valid(id, p.V)) continue;
        const float t = p.t[at + k];
        if (t == -INFINITY) continue;
        const float z = Elem<T>::get(row + id);
        const double log_q = ((double)t - (double)top) / (double)p.tau - log_sum, q = exp(log_q);
        if (q > 0.0 || isnan(q)) term += z <= kMasked ? INFINITY : q * (log_q - (double)z / (double)p.tau);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) term += __shfl_xor_sync(0xFFFFFFFFu, term, o);
    return term;
}

__device__ __forceinline__ void finish_row(const DistillParams &p, int64_t r, float m, float s, float c, double term, bool any)
{
    // m still at the mask value: no logit above it (s counts masked ones then); NaN has made s NaN.  s is relative to the rounded
    // reference; relative to the largest logit it is s 2^(ref - m c), and every ratio exp2((z - m) c) in it has c's error on a
    // small difference only.  A far row's s is relative to the largest logit already.
    const bool empty = m <= kMasked && !isnan(s);
    const double shift = far_row(m, c) ? 0.0 : ((double)ref(m, c) - (double)m * (double)c) * 0.6931471805599453;
    const double lse = empty ? -INFINITY : (double)m / (double)p.tau + log((double)s) + shift;
    p.lse[r] = (float)lse;
    p.loss[r] = !any || empty ? 0.f : (float)((double)p.tau * (double)p.tau * (term + lse));
}

// Three blocks of 512 threads per SM (40 registers): 107 us for 2,048 x 151,936 bf16 against 124 us with two.
template <typename T, bool kWarpRows>
__global__ void __launch_bounds__(kWarpRows ? kSmallBlock : kBlock, kWarpRows ? 4 : 3)
tfe_distill_forward_kernel(const DistillParams p)
{
    tfe_wait_for_stream();
    const float c = (float)(kLog2e / (double)p.tau);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if constexpr (kWarpRows) {
        const int64_t r = (int64_t)blockIdx.x * (kSmallBlock / 32) + warp;
        if (r >= p.N) return;
        const T *row = static_cast<const T *>(p.logits) + r * p.ld;
        float m, s;
        stream_row<T, 2>(row, p.V, 0, 1, lane, 32, c, m, s);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) fold(m, s, __shfl_xor_sync(0xFFFFFFFFu, m, o), __shfl_xor_sync(0xFFFFFFFFu, s, o), c);
        if (far_row(m, c)) {
            s = far_sum(row, p.V, 0, 1, lane, 32, c, m);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
        }
        bool any;
        const double term = teacher_term<T>(p, row, r, lane, any);
        if (lane == 0) finish_row(p, r, m, s, c, term, any);
    } else {
        __shared__ float s_m[kBlock / 32], s_s[kBlock / 32];
        __shared__ float2 s_part;
        __shared__ float s_far;
        const int64_t r = blockIdx.x / p.slices;
        const int slice = (int)(blockIdx.x % p.slices);
        const T *row = static_cast<const T *>(p.logits) + r * p.ld;
        double term = 0.0;
        bool any = false;
        if (slice == 0 && warp == 0) term = teacher_term<T>(p, row, r, lane, any);
        float m, s;
        stream_row<T, 4>(row, p.V, slice, p.slices, threadIdx.x, kBlock, c, m, s);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) fold(m, s, __shfl_xor_sync(0xFFFFFFFFu, m, o), __shfl_xor_sync(0xFFFFFFFFu, s, o), c);
        if (lane == 0) { s_m[warp] = m; s_s[warp] = s; }
        __syncthreads();
        if (warp == 0) {
            m = lane < kBlock / 32 ? s_m[lane] : kMasked;
            s = lane < kBlock / 32 ? s_s[lane] : 0.f;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) fold(m, s, __shfl_xor_sync(0xFFFFFFFFu, m, o), __shfl_xor_sync(0xFFFFFFFFu, s, o), c);
            if (lane == 0) {
                s_part = make_float2(m, s);
                s_far = p.slices == 1 && far_row(m, c) ? m : kMasked;
            }
        }
        if (p.slices > 1) {
            cg::cluster_group cluster = cg::this_cluster();
            cluster.sync();
            if (slice == 0 && threadIdx.x == 0) {
                for (int b = 1; b < p.slices; ++b) {
                    const float2 other = *cluster.map_shared_rank(&s_part, b);
                    fold(m, s, other.x, other.y, c);
                }
                if (far_row(m, c))
                    for (int b = 0; b < p.slices; ++b) *cluster.map_shared_rank(&s_far, b) = m;
            }
            cluster.sync();                 // a block's shared memory lives until its partner has read it
        } else {
            __syncthreads();
        }
        const float row_m = s_far;
        if (row_m > kMasked) {              // the row's largest logit, if the row is a far one: the same in every thread
            float part = far_sum(row, p.V, slice, p.slices, threadIdx.x, kBlock, c, row_m);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) part += __shfl_xor_sync(0xFFFFFFFFu, part, o);
            if (lane == 0) s_s[warp] = part;
            __syncthreads();
            if (threadIdx.x == 0) {
                s = 0.f;
                for (int w = 0; w < kBlock / 32; ++w) s += s_s[w];
                s_part.y = s;
            }
            if (p.slices > 1) {
                cg::cluster_group cluster = cg::this_cluster();
                cluster.sync();
                if (slice == 0 && threadIdx.x == 0)
                    for (int b = 1; b < p.slices; ++b) s += cluster.map_shared_rank(&s_part, b)->y;
                cluster.sync();
            }
        }
        if (slice == 0 && threadIdx.x == 0) finish_row(p, r, m, s, c, term, any);
    }
}

// ------------------------------------------------------------------ gradient

// One row, or one slice of it, by `threads` threads that sync with `sync`.
template <typename T, int U, typename Sync>
__device__ __forceinline__ void backward_row(const DistillParams &p, int64_t r, int slice, int tid, int threads, bool first_warp,
                                             int32_t *s_id, float *s_q, float *s_z, float *s_norm, Sync sync)
{
    constexpr int E = Elem<T>::kPerVec;
    const T *row = static_cast<const T *>(p.logits) + r * p.ld;
    T *out = static_cast<T *>(p.grad) + r * p.ld_grad;
    const int lane = threadIdx.x & 31;
    const float g = p.grad_loss[r], lse = p.lse_in[r];
    const Cut cut = cut_row(row, p.V);
    const int64_t v0 = cut.n_vec * slice / p.slices, v1 = cut.n_vec * (slice + 1) / p.slices;
    // this slice's elements: [e0, e1), the head and the tail with the first and the last slice
    const int64_t e0 = slice == 0 ? 0 : cut.head + v0 * E, e1 = slice == p.slices - 1 ? (int64_t)p.V : cut.head + v1 * E;
    const bool same_cut = ((reinterpret_cast<uintptr_t>(row) ^ reinterpret_cast<uintptr_t>(out)) & 15u) == 0;

    if (first_warp) {
        float top;
        double sum;
        teacher_norm(p, r, lane, top, sum);
        if (lane == 0) { s_norm[0] = top; s_norm[1] = sum == 0.0 ? 0.f : (float)(1.0 / sum); }
    }
    sync();
    const float t_top = s_norm[0], t_inv = s_norm[1];
    const bool live = g != 0.f && t_inv != 0.f && lse != -INFINITY;
    if (live) {
        const int64_t at = r * p.K;
        for (int k = tid; k < p.K; k += threads) {
            const int32_t id = p.ids[at + k];
            const bool mine = id >= e0 && id < e1;
            s_id[k] = mine ? id : -1;
            if (mine) {
                const float t = p.t[at + k];
                s_q[k] = t == -INFINITY ? 0.f : (float)exp(((double)t - (double)t_top) / (double)p.tau) * t_inv;
                s_z[k] = Elem<T>::get(row + id);
            }
        }
    }
    sync();

    // z log2(e) / tau - lse log2(e), both constants in two parts: rounding them alone would cost up to 5e-7 of a probability
    const float coef = g * p.tau, c = (float)(kLog2e / (double)p.tau), shift = (float)((double)lse * kLog2e);
    const float c_lo = (float)(kLog2e / (double)p.tau - (double)c), shift_lo = (float)((double)lse * kLog2e - (double)shift);
    auto prob = [&](float z) { return z <= kMasked ? 0.f : exp2_approx(fmaf(z, c, -shift) + fmaf(z, c_lo, -shift_lo)); };
    if (!live) {
        if (same_cut) {
            for (int64_t i = e0 + tid; i < (slice == 0 ? cut.head : e0); i += threads) Elem<T>::put(out + i, 0.f);
            for (int64_t i = cut.head + v1 * E + tid; i < e1; i += threads) Elem<T>::put(out + i, 0.f);
            uint4 *ob = reinterpret_cast<uint4 *>(out + cut.head);
            for (int64_t v = v0 + tid; v < v1; v += threads) __stcs(ob + v, make_uint4(0, 0, 0, 0));
        } else {
            for (int64_t i = e0 + tid; i < e1; i += threads) Elem<T>::put(out + i, 0.f);
        }
        return;
    }
    if (same_cut) {
        if (slice == 0) for (int64_t i = tid; i < cut.head; i += threads) Elem<T>::put(out + i, coef * prob(Elem<T>::get(row + i)));
        for (int64_t i = cut.head + v1 * E + tid; i < e1; i += threads) Elem<T>::put(out + i, coef * prob(Elem<T>::get(row + i)));
        const uint4 *body = reinterpret_cast<const uint4 *>(row + cut.head);
        uint4 *ob = reinterpret_cast<uint4 *>(out + cut.head);
        for (int64_t v = v0 + tid; v < v1; v += (int64_t)U * threads) {
            uint4 raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (v + (int64_t)u * threads < v1) raw[u] = load_stream(body + v + (int64_t)u * threads);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (v + (int64_t)u * threads < v1) {
                    float f[E];
                    Elem<T>::unpack(raw[u], f);
#pragma unroll
                    for (int e = 0; e < E; ++e) f[e] = coef * prob(f[e]);
                    __stcs(ob + v + (int64_t)u * threads, Elem<T>::pack(f));
                }
        }
    } else {
        for (int64_t i = e0 + tid; i < e1; i += threads) Elem<T>::put(out + i, coef * prob(Elem<T>::get(row + i)));
    }
    sync();
    for (int k = tid; k < p.K; k += threads) {
        const int32_t id = s_id[k];
        if (id < 0) continue;
        float q = 0.f;
        bool first = true;
        for (int j = 0; j < p.K; ++j)
            if (s_id[j] == id) {
                if (j < k) first = false;
                q += s_q[j];
            }
        if (first) Elem<T>::put(out + id, coef * (prob(s_z[k]) - q));
    }
}

template <typename T, bool kWarpRows>
__global__ void __launch_bounds__(kWarpRows ? kSmallBlock : kBlock)
tfe_distill_backward_kernel(const DistillParams p)
{
    tfe_wait_for_stream();
    extern __shared__ float s_raw[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int per_row = 3 * p.K + 2;
    if constexpr (kWarpRows) {
        const int64_t r = (int64_t)blockIdx.x * (kSmallBlock / 32) + warp;
        if (r >= p.N) return;
        float *mine = s_raw + warp * per_row;
        backward_row<T, 2>(p, r, 0, lane, 32, true, reinterpret_cast<int32_t *>(mine), mine + p.K, mine + 2 * p.K, mine + 3 * p.K,
                           [] { __syncwarp(); });
    } else {
        backward_row<T, 4>(p, blockIdx.x / p.slices, (int)(blockIdx.x % p.slices), threadIdx.x, kBlock, warp == 0,
                           reinterpret_cast<int32_t *>(s_raw), s_raw + p.K, s_raw + 2 * p.K, s_raw + 3 * p.K, [] { __syncthreads(); });
    }
}

// ------------------------------------------------------------------ host side

size_t elem_size(int32_t dtype) { return dtype == TFE_DTYPE_BF16 ? 2 : 4; }

bool row_args_ok(const void *x, int32_t dtype, int32_t N, int32_t V, int64_t ld)
{
    if (dtype != TFE_DTYPE_BF16 && dtype != TFE_DTYPE_F32) return false;
    if (N < 0 || N > TFE_ROWS_MAX || V < 1 || ld < V || ld > (1ll << 34)) return false;
    return N == 0 || (x && reinterpret_cast<uintptr_t>(x) % elem_size(dtype) == 0);
}

// Warps take rows of up to this many bytes; beyond, a block per row and, with few rows, several.
constexpr int64_t kWarpRowBytes = 8192;

int32_t slices_for(int32_t N, int64_t row_bytes, int sms)
{
    int32_t s = 1;
    while (s < 8 && (int64_t)N * s < 2 * sms && row_bytes / (2 * s) >= 16384) s *= 2;
    return s;
}

template <typename F>
tfe_status launch_rows(F kernel, int grid, int block, int cluster, size_t smem, cudaStream_t stream, const DistillParams &p)
{
    return tfe_launch_serial(kernel, (unsigned)grid, (unsigned)block, (unsigned)cluster, smem, stream, "distillation launch", p);
}

tfe_status device_sms(int *sms)
{
    int dev = 0;
    tfe_status st = tfe_note_cuda(cudaGetDevice(&dev), "cudaGetDevice");
    return st != TFE_OK ? st : tfe_note_cuda(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev), "cudaDeviceGetAttribute");
}

bool teacher_args_ok(int32_t N, int32_t K, float tau, const int32_t *ids, const float *t)
{
    if (K < 1 || K > kMaxTop || !(tau > 0.f) || tau > 1e6f || tau < 1e-6f) return false;
    return N == 0 || (ids && t && reinterpret_cast<uintptr_t>(ids) % 4 == 0 && reinterpret_cast<uintptr_t>(t) % 4 == 0);
}

}  // namespace

extern "C" {

tfe_status tfe_distill_forward(const void *logits, int32_t dtype, int32_t N, int32_t V, int64_t ld, const int32_t *teacher_ids,
                               const float *teacher_logits, int32_t K, float tau, float *loss, float *lse, void *stream_)
{
    if (!row_args_ok(logits, dtype, N, V, ld) || !teacher_args_ok(N, K, tau, teacher_ids, teacher_logits)) return TFE_ERR_INVALID_ARG;
    if (N == 0) return TFE_OK;
    if (!loss || !lse) return TFE_ERR_INVALID_ARG;
    int sms = 0;
    if (tfe_status st = device_sms(&sms)) return st;
    DistillParams p{};
    p.logits = logits; p.ld = ld; p.N = N; p.V = V; p.K = K; p.tau = tau; p.ids = teacher_ids; p.t = teacher_logits;
    p.loss = loss; p.lse = lse;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const int64_t row_bytes = (int64_t)V * (int64_t)elem_size(dtype);
    if (row_bytes <= kWarpRowBytes) {
        p.slices = 1;
        const int grid = (N + kSmallBlock / 32 - 1) / (kSmallBlock / 32);
        return dtype == TFE_DTYPE_BF16 ? launch_rows(tfe_distill_forward_kernel<__nv_bfloat16, true>, grid, kSmallBlock, 1, 0, stream, p)
                                       : launch_rows(tfe_distill_forward_kernel<float, true>, grid, kSmallBlock, 1, 0, stream, p);
    }
    p.slices = slices_for(N, row_bytes, sms);
    return dtype == TFE_DTYPE_BF16 ? launch_rows(tfe_distill_forward_kernel<__nv_bfloat16, false>, N * p.slices, kBlock, p.slices, 0, stream, p)
                                   : launch_rows(tfe_distill_forward_kernel<float, false>, N * p.slices, kBlock, p.slices, 0, stream, p);
}

tfe_status tfe_distill_backward(const void *logits, int32_t dtype, int32_t N, int32_t V, int64_t ld, const int32_t *teacher_ids,
                                const float *teacher_logits, int32_t K, float tau, const float *lse, const float *grad_loss,
                                void *grad_logits, int64_t ld_grad, void *stream_)
{
    if (!row_args_ok(logits, dtype, N, V, ld) || !teacher_args_ok(N, K, tau, teacher_ids, teacher_logits)) return TFE_ERR_INVALID_ARG;
    if (!row_args_ok(grad_logits, dtype, N, V, ld_grad)) return TFE_ERR_INVALID_ARG;
    if (N == 0) return TFE_OK;
    if (!lse || !grad_loss) return TFE_ERR_INVALID_ARG;
    // the same rows in place, or buffers that do not touch
    const uintptr_t es = elem_size(dtype), out = reinterpret_cast<uintptr_t>(grad_logits);
    const uintptr_t out_bytes = ((uintptr_t)(N - 1) * (uintptr_t)ld_grad + (uintptr_t)V) * es;
    auto touches = [&](const void *operand, uintptr_t bytes) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(operand);
        return at < out + out_bytes && out < at + bytes;
    };
    if (grad_logits == logits ? ld_grad != ld : touches(logits, ((uintptr_t)(N - 1) * (uintptr_t)ld + (uintptr_t)V) * es)) return TFE_ERR_INVALID_ARG;
    const uintptr_t teacher_bytes = (uintptr_t)N * (uintptr_t)K * 4;
    if (touches(teacher_ids, teacher_bytes) || touches(teacher_logits, teacher_bytes) || touches(lse, (uintptr_t)N * 4) ||
        touches(grad_loss, (uintptr_t)N * 4))
        return TFE_ERR_INVALID_ARG;
    int sms = 0;
    if (tfe_status st = device_sms(&sms)) return st;
    DistillParams p{};
    p.logits = logits; p.ld = ld; p.N = N; p.V = V; p.K = K; p.tau = tau; p.ids = teacher_ids; p.t = teacher_logits;
    p.lse_in = lse; p.grad_loss = grad_loss; p.grad = grad_logits; p.ld_grad = ld_grad;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const int64_t row_bytes = (int64_t)V * (int64_t)elem_size(dtype);
    const size_t per_row = (size_t)(3 * K + 2) * sizeof(float);
    if (row_bytes <= kWarpRowBytes && K <= 256) {
        p.slices = 1;
        const int rows = kSmallBlock / 32, grid = (N + rows - 1) / rows;
        return dtype == TFE_DTYPE_BF16
                   ? launch_rows(tfe_distill_backward_kernel<__nv_bfloat16, true>, grid, kSmallBlock, 1, per_row * rows, stream, p)
                   : launch_rows(tfe_distill_backward_kernel<float, true>, grid, kSmallBlock, 1, per_row * rows, stream, p);
    }
    p.slices = slices_for(N, row_bytes, sms);
    return dtype == TFE_DTYPE_BF16
               ? launch_rows(tfe_distill_backward_kernel<__nv_bfloat16, false>, N * p.slices, kBlock, 1, per_row, stream, p)
               : launch_rows(tfe_distill_backward_kernel<float, false>, N * p.slices, kBlock, 1, per_row, stream, p);
}

}  // extern "C"

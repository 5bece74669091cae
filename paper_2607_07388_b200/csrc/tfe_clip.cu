// The norm of many gradients taken together, and clipping by it.
//
//   norm = sqrt(sum over all tensors of x^2)        x <- x min(1, max_norm / norm)
//
//   tfe_grad_norm_kernel   sums of squares of all tensors in one launch.  The tensors' list travels in the launch's parameters; the
//                          elements are cut into chunks, every block takes an equal run of chunks and leaves one fp64 sum.
//   tfe_grad_clip_kernel   every block adds up those sums in the same order, and scales its run of chunks, from its end to its
//                          beginning: what was read last is in L2 (with more than kLarge tensors, each launch's own).  Where nothing is to be
//                          scaled in place it reads no tensor.
//
// HBM bounds both: one read for the norm, one read and one write to scale (155.6 M bf16 elements: 51 + 98 us, 51 + 91 in place; writing 311 MB
// alone takes 80, so what L2 saves in reads shows little; 155.6 M fp32: 102 + 203 us).  A thread's eight or four squares are summed in fp32 and
// joined in fp64; where they leave fp32's range they are formed in fp64.  No atomics: the order depends on the sizes alone.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>
#include <new>

#include "../../include/tfe.h"
#include "tfe_internal.h"
#include "tfe_rows.cuh"

namespace {

using tfe_rows::Elem;

constexpr int kThreads = 256;
constexpr int64_t kChunkMin = 2048, kChunkMax = 16384;        // elements of a chunk: few tensors are spread over the SMs, many read in long runs
// What the norm leaves in L2 for the scaling (126 MB, and its writes pass through it), with elements of two bytes; of fp32 twice as much is
// marked, more than stays.
constexpr int64_t kKeepBytes = 80 << 20;
constexpr int kPerSm = 6;                       // blocks, all resident
constexpr int kBlocks = 148 * kPerSm;           // most blocks of a launch

struct Entry { uint64_t in, out; int64_t n; uint32_t first; int32_t dtype; };       // first: the tensor's first chunk
template <int kRoom> struct Table {
    int32_t tensors, parts, part0;              // parts: sums of all launches; part0: this launch's first
    uint32_t chunks;
    int64_t chunk;
    uint32_t keep;                              // chunks of a block's run that L2 has room for
    int32_t write_norm, in_place, only_norm;
    float max_norm;
    double *part;
    float *norm;
    Entry at[kRoom];
};
constexpr int kSmall = 64, kLarge = 900;        // 32 bytes each; a launch takes parameters of up to 32,764 bytes

// Sum of squares of a vector.  Below 2^-80 (and not zero) or not finite, fp32's range may have cut terms: once more in fp64.
template <typename T>
__device__ __forceinline__ double squares(const uint4 &raw)
{
    constexpr int E = Elem<T>::kPerVec;
    float f[E], s = 0.f;
    Elem<T>::unpack(raw, f);
#pragma unroll
    for (int e = 0; e < E; ++e) s = fmaf(f[e], f[e], s);
    if (!(s >= 0x1p-80f && s <= 3.4e38f)) {
        if ((raw.x | raw.y | raw.z | raw.w) == 0u) return 0.0;
        double d = 0.0;
#pragma unroll
        for (int e = 0; e < E; ++e) d = fma((double)f[e], (double)f[e], d);
        return d;
    }
    return (double)s;
}

template <int kRoom>
__device__ __forceinline__ int find_tensor(const Table<kRoom> &t, uint32_t chunk)      // the last whose first chunk is not beyond
{
    int lo = 0, hi = t.tensors - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (t.at[mid].first <= chunk) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// Policies of the L2 cache for what will be read again and for what will not.
__device__ __forceinline__ uint64_t policy(bool keep)
{
    uint64_t p;
    if (keep) asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(p));
    else asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
    return p;
}
__device__ __forceinline__ uint4 load_hint(const uint4 *at, uint64_t hint)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.L2::cache_hint.v4.u32 {%0, %1, %2, %3}, [%4], %5;" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(at), "l"(hint) : "memory");
    return v;
}

template <typename T>
__device__ __forceinline__ double chunk_squares(const T *x, int64_t n, uint64_t hint)
{
    const tfe_rows::Cut cut = tfe_rows::cut_row(x, n);
    const uint4 *body = reinterpret_cast<const uint4 *>(x + cut.head);
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < cut.head; i += kThreads) { const double v = (double)Elem<T>::get(x + i); sum += v * v; }
    for (int64_t i = cut.head + cut.n_vec * Elem<T>::kPerVec + threadIdx.x; i < n; i += kThreads) { const double v = (double)Elem<T>::get(x + i); sum += v * v; }
    constexpr int U = 4;
    int64_t v = threadIdx.x;
    for (; v + (U - 1) * kThreads < cut.n_vec; v += U * kThreads) {
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = load_hint(body + v + u * kThreads, hint);
#pragma unroll
        for (int u = 0; u < U; ++u) sum += squares<T>(raw[u]);
    }
    for (; v < cut.n_vec; v += kThreads) sum += squares<T>(load_hint(body + v, hint));
    return sum;
}

__device__ __forceinline__ double block_sum(double x, double *s_warp)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    if ((threadIdx.x & 31) == 0) s_warp[threadIdx.x >> 5] = x;
    __syncthreads();
    x = 0.0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) x += s_warp[w];
    return x;
}

template <int kRoom>
__global__ void __launch_bounds__(kThreads, kPerSm)
tfe_grad_norm_kernel(const __grid_constant__ Table<kRoom> t)
{
    __shared__ double s_warp[kThreads / 32];
    tfe_wait_for_stream();
    const uint32_t c0 = (uint32_t)((uint64_t)t.chunks * blockIdx.x / gridDim.x), c1 = (uint32_t)((uint64_t)t.chunks * (blockIdx.x + 1) / gridDim.x);
    double sum = 0.0;
    // the end of this block's run stays in L2 for the scaling, which begins there; the rest makes room for it
    const uint32_t kept = c1 - (uint32_t)min((uint64_t)(c1 - c0), (uint64_t)t.keep);
    const uint64_t last = policy(true), first = policy(false);
    if (c0 < c1) {
        int i = find_tensor(t, c0);
        for (uint32_t c = c0; c < c1; ++c) {
            while (i + 1 < t.tensors && t.at[i + 1].first <= c) ++i;
            const int64_t from = (int64_t)(c - t.at[i].first) * t.chunk, n = min(t.chunk, t.at[i].n - from);
            sum += t.at[i].dtype == TFE_DTYPE_BF16 ? chunk_squares(reinterpret_cast<const __nv_bfloat16 *>(t.at[i].in) + from, n, c >= kept ? last : first)
                                                   : chunk_squares(reinterpret_cast<const float *>(t.at[i].in) + from, n, c >= kept ? last : first);
        }
    }
    sum = block_sum(sum, s_warp);
    if (threadIdx.x == 0) t.part[t.part0 + blockIdx.x] = sum;
}

template <typename T>
__device__ __forceinline__ void chunk_scale(const T *x, T *y, int64_t n, float by, float pre, uint64_t hint)
{
    if (((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(y)) & 15u) != 0) {
        for (int64_t i = threadIdx.x; i < n; i += kThreads) Elem<T>::put(y + i, Elem<T>::get(x + i) * pre * by);
        return;
    }
    constexpr int E = Elem<T>::kPerVec;
    const tfe_rows::Cut cut = tfe_rows::cut_row(x, n);
    const uint4 *from = reinterpret_cast<const uint4 *>(x + cut.head);
    uint4 *to = reinterpret_cast<uint4 *>(y + cut.head);
    for (int64_t i = threadIdx.x; i < cut.head; i += kThreads) Elem<T>::put(y + i, Elem<T>::get(x + i) * pre * by);
    for (int64_t i = cut.head + cut.n_vec * E + threadIdx.x; i < n; i += kThreads) Elem<T>::put(y + i, Elem<T>::get(x + i) * pre * by);
    auto scale = [&](const uint4 &raw) {
        float f[E];
        Elem<T>::unpack(raw, f);
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = f[e] * pre * by;
        return Elem<T>::pack(f);
    };
    constexpr int U = 4;
    int64_t v = threadIdx.x;
    for (; v + (U - 1) * kThreads < cut.n_vec; v += U * kThreads) {
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = load_hint(from + v + u * kThreads, hint);
#pragma unroll
        for (int u = 0; u < U; ++u) __stcs(to + v + u * kThreads, scale(raw[u]));
    }
    for (; v < cut.n_vec; v += kThreads) __stcs(to + v, scale(load_hint(from + v, hint)));
}

template <int kRoom>
__global__ void __launch_bounds__(kThreads)
tfe_grad_clip_kernel(const __grid_constant__ Table<kRoom> t)
{
    __shared__ double s_warp[kThreads / 32];
    tfe_wait_for_stream();
    double sum = 0.0;
    for (int i = threadIdx.x; i < t.parts; i += kThreads) sum += __ldcg(t.part + i);
    const double norm = sqrt(block_sum(sum, s_warp));
    if (t.write_norm && blockIdx.x == 0 && threadIdx.x == 0) *t.norm = (float)norm;
    if (t.only_norm) return;
    // a norm that is not finite, as the caller sees it, scales nothing
    const double factor = norm > (double)t.max_norm && (float)norm <= 3.402823466e38f ? (double)t.max_norm / norm : 1.0;
    // a factor that fp32 holds with fewer digits, below 2^-126, is taken in two steps, of which the first is exact (elements that it is not
    // exact for end as 0 in any case)
    const float pre = factor < 0x1p-100 ? 0x1p-64f : 1.f, by = (float)(factor / (double)pre);
    if (by == 1.f && t.in_place) return;
    const uint32_t c0 = (uint32_t)((uint64_t)t.chunks * blockIdx.x / gridDim.x), c1 = (uint32_t)((uint64_t)t.chunks * (blockIdx.x + 1) / gridDim.x);
    if (c0 >= c1) return;
    const uint64_t hint = policy(false);
    int i = find_tensor(t, c1 - 1);
    for (uint32_t c = c1; c-- > c0;) {
        while (t.at[i].first > c) --i;
        const int64_t from = (int64_t)(c - t.at[i].first) * t.chunk, n = min(t.chunk, t.at[i].n - from);
        if (t.at[i].dtype == TFE_DTYPE_BF16)
            chunk_scale(reinterpret_cast<const __nv_bfloat16 *>(t.at[i].in) + from, reinterpret_cast<__nv_bfloat16 *>(t.at[i].out) + from, n, by, pre, hint);
        else
            chunk_scale(reinterpret_cast<const float *>(t.at[i].in) + from, reinterpret_cast<float *>(t.at[i].out) + from, n, by, pre, hint);
    }
}

// ------------------------------------------------------------------ host side

int64_t elem_size(int32_t dtype) { return dtype == TFE_DTYPE_BF16 ? 2 : 4; }

struct Job {
    const uint64_t *in, *out;                   // out null: in place
    const int64_t *n; const int32_t *dtype;
    int32_t tensors; bool only_norm;
    float max_norm, *norm; double *part; cudaStream_t stream; int sms;
    int64_t chunk;
};

int64_t launches(int32_t tensors) { return std::max<int64_t>(1, ((int64_t)tensors + kLarge - 1) / kLarge); }

// One launch for each kLarge tensors, the norm's first; `pass` 0: squares, 1: scaling.
template <int kRoom>
tfe_status run_pass(const Job &j, int pass, int32_t lo, int32_t hi, int32_t *part0, int32_t parts, bool first)
{
    Table<kRoom> t;                             // (only what is used of the table is written)
    t.tensors = 0; t.chunks = 0;
    uint64_t chunks = 0;
    for (int32_t i = lo; i < hi; ++i) {
        if (j.n[i] == 0) continue;
        t.at[t.tensors++] = {j.in[i], j.out ? j.out[i] : j.in[i], j.n[i], (uint32_t)chunks, j.dtype[i]};
        chunks += (uint64_t)((j.n[i] + j.chunk - 1) / j.chunk);
    }
    if (chunks > 0xFFFFFFFFull) return TFE_ERR_INVALID_ARG;
    t.chunks = (uint32_t)chunks; t.chunk = j.chunk;
    t.keep = (uint32_t)(j.only_norm ? 0 : kKeepBytes / (j.chunk * 2) / (kPerSm * j.sms));
    t.parts = parts; t.part0 = *part0; t.part = j.part; t.norm = j.norm; t.max_norm = j.max_norm;
    t.write_norm = first; t.in_place = j.out == nullptr; t.only_norm = j.only_norm;
    const unsigned grid = pass == 1 && j.only_norm ? 1u : (unsigned)std::max<uint64_t>(1, std::min<uint64_t>(chunks, (uint64_t)std::min(kBlocks, kPerSm * j.sms)));
    if (pass == 0) *part0 += (int32_t)grid;
    return tfe_launch_serial(pass == 0 ? tfe_grad_norm_kernel<kRoom> : tfe_grad_clip_kernel<kRoom>, grid, kThreads, 1, 0, j.stream, "gradient norm launch", t);
}

tfe_status run(const Job &j)
{
    int32_t parts = 0;
    for (int pass = 0; pass < 2; ++pass) {
        int32_t at = 0, lo = 0;
        do {
            const int32_t hi = (int32_t)std::min<int64_t>(j.tensors, (int64_t)lo + kLarge);
            const tfe_status st = hi - lo <= kSmall ? run_pass<kSmall>(j, pass, lo, hi, &at, parts, lo == 0) : run_pass<kLarge>(j, pass, lo, hi, &at, parts, lo == 0);
            if (st != TFE_OK) return st;
            lo = hi;
        } while (lo < j.tensors && !(pass == 1 && j.only_norm));
        parts = pass == 0 ? at : parts;
    }
    return TFE_OK;
}

tfe_status check_and_run(const uint64_t *in, const uint64_t *out, const int64_t *numel, const int32_t *dtype, int32_t n, bool only_norm, float max_norm,
                         float *norm, void *workspace, int64_t workspace_bytes, void *stream)
{
    if (n < 0 || n > TFE_CLIP_MAX_TENSORS || (n > 0 && (!in || !numel || !dtype)) || !norm || reinterpret_cast<uintptr_t>(norm) % 4 != 0) return TFE_ERR_INVALID_ARG;
    if (!only_norm && !(max_norm >= 0.f)) return TFE_ERR_INVALID_ARG;
    for (int32_t i = 0; i < n; ++i) {
        if (numel[i] < 0 || numel[i] > (1ll << 40) || (dtype[i] != TFE_DTYPE_BF16 && dtype[i] != TFE_DTYPE_F32)) return TFE_ERR_INVALID_ARG;
        const uint64_t es = (uint64_t)elem_size(dtype[i]);
        if (numel[i] > 0 && (!in[i] || in[i] % es != 0 || (out && (!out[i] || out[i] % es != 0)))) return TFE_ERR_INVALID_ARG;
    }
    if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 8 != 0) return TFE_ERR_INVALID_ARG;
    if (workspace_bytes < tfe_clip_workspace_bytes(n)) return TFE_ERR_CAPACITY;
    if (!only_norm) {
        // what is written must touch nothing else that is read or written, but a result may be its own tensor
        struct Range { uint64_t at, end; int32_t i; bool made; };
        Range *all = new (std::nothrow) Range[2 * (size_t)n + 2];
        if (!all) return TFE_ERR_INTERNAL;
        size_t k = 0;
        const uint64_t w = reinterpret_cast<uintptr_t>(workspace), s = reinterpret_cast<uintptr_t>(norm);
        all[k++] = {w, w + (uint64_t)tfe_clip_workspace_bytes(n), -1, true};
        all[k++] = {s, s + 4, -2, true};
        for (int32_t i = 0; i < n; ++i) {
            const uint64_t bytes = (uint64_t)(numel[i] * elem_size(dtype[i]));
            if (bytes == 0) continue;
            all[k++] = {in[i], in[i] + bytes, i, !out};
            if (out && out[i] != in[i]) all[k++] = {out[i], out[i] + bytes, i, true};
            else if (out) all[k - 1].made = true;
        }
        std::sort(all, all + k, [](const Range &a, const Range &b) { return a.at < b.at; });
        bool bad = false;
        uint64_t end_any = 0, end_made = 0;     // furthest end so far, of all and of those that are written
        for (size_t i = 0; i < k && !bad; ++i) {
            bad = all[i].at < (all[i].made ? end_any : end_made);
            end_any = std::max(end_any, all[i].end);
            if (all[i].made) end_made = std::max(end_made, all[i].end);
        }
        delete[] all;
        if (bad) return TFE_ERR_INVALID_ARG;
    }
    int dev = 0, sms = 0;
    if (tfe_status st = tfe_note_cuda(cudaGetDevice(&dev), "cudaGetDevice")) return st;
    if (tfe_status st = tfe_note_cuda(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev), "cudaDeviceGetAttribute")) return st;
    int64_t total = 0, chunk = kChunkMin;
    for (int32_t i = 0; i < n; ++i) total += numel[i];
    while (chunk < kChunkMax && total / (chunk * 2) >= 4 * kBlocks) chunk *= 2;
    return run({in, out, numel, dtype, n, only_norm, max_norm, norm, static_cast<double *>(workspace), static_cast<cudaStream_t>(stream), sms, chunk});
}

// DLTensor of the DLPack standard, version 1
struct DlTensor {
    void *data;
    struct { int32_t type, id; } device;        // type 2: CUDA
    int32_t ndim;
    struct { uint8_t code, bits; uint16_t lanes; } dtype;       // code 2: float, 4: bfloat
    int64_t *shape, *strides;                   // strides null: side by side in order
    uint64_t byte_offset;
};

}  // namespace

extern "C" {

tfe_status tfe_describe_tensors(void *objects, void *(*item)(void *, int64_t), int (*describe)(void *, void *), int32_t n, uint64_t *tensors, int64_t *numel,
                                int32_t *dtype, int32_t *device, int32_t *reason)
{
    if (!objects || !item || !describe || n < 1 || !tensors || !numel || !dtype || !device || !reason) return TFE_ERR_INVALID_ARG;
    *reason = 0;
    for (int32_t i = 0; i < n; ++i) {
        DlTensor t{};
        if (describe(item(objects, i), &t) != 0) { *reason = 4; return TFE_ERR_INVALID_ARG; }
        if (i == 0) *device = t.device.id;
        if (t.device.type != 2 || t.device.id != *device) *reason = 1;
        const bool bf16 = t.dtype.code == 4 && t.dtype.bits == 16 && t.dtype.lanes == 1, f32 = t.dtype.code == 2 && t.dtype.bits == 32 && t.dtype.lanes == 1;
        if (!*reason && !bf16 && !f32) *reason = 2;
        int64_t count = 1;
        bool in_order = true;
        for (int32_t k = t.ndim; k-- > 0;) {
            if (t.strides && t.shape[k] != 1 && t.strides[k] != count) in_order = false;
            count *= t.shape[k];
        }
        if (!*reason && !in_order && count != 0) *reason = 3;
        if (*reason) return TFE_ERR_INVALID_ARG;
        tensors[i] = count ? reinterpret_cast<uintptr_t>(t.data) + t.byte_offset : 0;
        numel[i] = count;
        dtype[i] = bf16 ? TFE_DTYPE_BF16 : TFE_DTYPE_F32;
    }
    return TFE_OK;
}

int64_t tfe_clip_workspace_bytes(int32_t n)
{
    return n < 0 || n > TFE_CLIP_MAX_TENSORS ? -1 : launches(n) * kBlocks * (int64_t)sizeof(double);
}

tfe_status tfe_grad_norm(const uint64_t *tensors, const int64_t *numel, const int32_t *dtype, int32_t n, float *norm, void *workspace,
                         int64_t workspace_bytes, void *stream)
{
    return check_and_run(tensors, nullptr, numel, dtype, n, true, 0.f, norm, workspace, workspace_bytes, stream);
}

tfe_status tfe_clip_grad_norm(const uint64_t *tensors, const uint64_t *results, const int64_t *numel, const int32_t *dtype, int32_t n, float max_norm,
                              float *norm, void *workspace, int64_t workspace_bytes, void *stream)
{
    return check_and_run(tensors, results, numel, dtype, n, false, max_norm, norm, workspace, workspace_bytes, stream);
}

}  // extern "C"

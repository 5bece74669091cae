// Drawing the next token of every sequence from its logits: temperature, min-p, top-k and top-p, then one draw by a given
// random number.  (The paper's lookups are keyed by the token ids that decoding produces; it names no sampling rule.)
//
// With x_i = (z_i - z_max) / T and w_i = exp(x_i), every restriction keeps a prefix of one order -- descending logit, equal
// logits by ascending index -- so the whole operator is three searches on that order's running mass:
//     min-p   drops entries with z < z_max + T ln(min_p)              (a comparison, before anything is counted)
//     top-k   the first k entries; their mass is S1
//     top-p   the shortest prefix of them with a mass of at least p S1; its mass is S2
//     draw    the first entry whose running mass exceeds u S2
// No sort of the row.
//
// bf16 rows have few different values: one pass counts the entries of each, in pairs.  Count times weight is a value's exact
// mass, so the ends of all searches follow from the counts, and one more pass finds the drawn value's entries.
//
// fp32 rows, and bf16 rows with logits too small to be counted: one pass counts the entries by bins of (z_max - z) / T, with the sum of their offsets in the bin; a
// bin's mass is then known to about 1e-5 of the total (its count times the weight at its mean), which names for every search
// the bin, seldom two, that holds its end.  One more pass sums the exact mass above those bins and collects their entries,
// which the first block sorts and searches.  Where the kept prefix is short all of it is collected and no sum is needed.
// Bins with more entries than the list (long runs of equal logits) send the row through an exact selection by key digits.
//
// A row is taken by a cluster of blocks, many rows by a block each; a slice that fits stays in shared memory.
//
// Numbers: a token's choice turns on sums of up to 10^5 nearly equal weights, next to borders 10^-5 apart, so weights are
// evaluated in 64 bits (relative error below 1e-14) and summed as 64-bit integers in units of 2^-shift -- exact, and the
// same in any order.
//
// What bounds it: 256 flat rows of 151,936 bf16 logits take 82 us (216 as fp32, by bins of distance, of about 110
// instructions a logit with 15 fp64 ones): 11 us the first read, 32 us the counting -- 10 instructions and an addition in
// shared memory a logit, and no faster with 2 or 4 loads ahead (86, 84 us) --, 14 us the second look, the rest steps of one
// block.  One fp32 row takes 29 us, the latency of the steps of a cluster of eight blocks; 64 with settings of their own take
// 74 us, where a row whose ends need sums weighs all its entries.  HBM would need 12, 0.1 and 6 us.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstddef>
#include <cstdint>

#include "../../include/tfe.h"
#include "tfe_internal.h"
#include "tfe_rows.cuh"

namespace {

using namespace tfe_rows;
namespace cg = cooperative_groups;
typedef unsigned long long u64;

constexpr int kThreads = 512;
constexpr int kBins = 4096;
constexpr int kList = 1024;             // entries that are collected and sorted at once
constexpr float kRange = 32.f;          // weights below exp(-32) share the last bin

struct SampleParams {
    const void *logits; int64_t ld;
    int32_t B, V;
    const float *temperature; const int32_t *top_k; const float *top_p, *min_p, *u;
    int32_t *tokens; float *prob;
    int32_t blocks;                     // per row
    int32_t slice_cap;                  // logits that fit the shared slice; smaller slices are kept there
    int32_t shift;                      // masses are integers in units of 2^-shift
};

// Composite key of an entry: greater keys come first in the order.  Never 0.
__device__ __forceinline__ u64 entry_key(float z, int32_t i)
{
    z += 0.f;                           // -0 and +0 are equal logits
    const uint32_t b = __float_as_uint(z);
    const uint32_t o = (b & 0x80000000u) ? ~b : (b | 0x80000000u);
    return ((u64)o << 32) | (uint32_t)~(uint32_t)i;
}
__device__ __forceinline__ float key_logit(u64 key)
{
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float((o & 0x80000000u) ? (o & 0x7FFFFFFFu) : ~o);
}
__device__ __forceinline__ int32_t key_index(u64 key) { return (int32_t)~(uint32_t)key; }

struct RowRule {
    double top, a;                      // a = 16 log2(e) / T
    float topf, cut;                    // entries with z < cut are out; cut is finite or +inf, so -inf and NaN always are
    float bins;                         // 256 bins per unit of top - z
    float floor;                        // at and below this logit nothing of a weight is left: 2^shift w rounds to 0
};

constexpr double kWhole = 4503599627370496.0;           // 2^52: what is added to it is rounded to a whole number

// w 2^shift + plus, with w = exp((z - top) / T) in 64 bits: y = 16 log2 w = n + f, n whole, |f| <= 1/2, so
// w = 2^(n / 16) 2^(f / 16); the first factor from a table of 2^(shift + j / 16) (16 entries, so that a warp's reads never
// meet in a bank) with n's multiples of 16 added to its exponent, the second by Taylor's series to the sixth power (|f| ln 2
// / 16 is at most 0.0217; the first term left out is below 5e-16).  The maximum weighs 2^shift exactly.  A z below the floor is
// weighed at the floor, which lies at most 4 (shift + 2) below 0 in log2 w: n fits the exponent for any z.
// plus = 2^52 rounds to a whole number, which stands in the result's low 52 bits.
__device__ __forceinline__ double weight_of(const RowRule &q, const double *table, float z, double plus)
{
    const double y = ((double)fminf(fmaxf(z, q.floor), 3.402823466e38f) - q.top) * q.a;
    constexpr double magic = 1.5 * kWhole;              // the low bits hold the whole number, negative ones too
    const double shifted = y + magic;
    const int n = __double2loint(shifted);
    const double f = y - (shifted - magic);
    constexpr double c = 0.6931471805599453 / 16;
    double p = c * c * c * c * c * c / 720;
    p = fma(p, f, c * c * c * c * c / 120);
    p = fma(p, f, c * c * c * c / 24);
    p = fma(p, f, c * c * c / 6);
    p = fma(p, f, c * c / 2);
    p = fma(p, f, c);
    p = fma(p, f, 1.0);
    const double t = table[n & 15];
    return fma(p, __hiloint2double(__double2hiint(t) + (int)((uint32_t)(n & ~15) << 16), __double2loint(t)), plus);
}
__device__ __forceinline__ u64 whole_of(double x) { return (u64)__double_as_longlong(x) & 0xFFFFFFFFFFFFFull; }    // after plus = kWhole
__device__ __forceinline__ u64 mass_of(const RowRule &q, const double *table, float z) { return whole_of(weight_of(q, table, z, kWhole)); }

// Place of a kept logit: 256 times its distance from the maximum in bins, rounded; the bin is place >> 8.  Not decreasing
// as z falls.  What lies beyond the last bin is in it.
__device__ __forceinline__ uint32_t place_of(const RowRule &q, float z)
{
    return __float_as_uint(fminf((q.topf - z) * q.bins, (float)(256 * kBins - 1)) + 8388608.f) & 0x7FFFFFu;
}

enum { kOpDone = 0, kOpCollect = 1, kOpDigits = 2 };
enum { kTopK = 0, kTopP = 1, kDraw = 2, kSearches = 3 };
struct Command {                        // what the first block asks of its cluster
    int op;
    int by_bins;                        // kOpCollect: by the bins below, or by (key & mask) == prefix
    int first;                          // by bins: the first collection of the row
    int sums;                           // by bins: 0 no masses, 1 those below the searches' bins, 2 of all entries too
    uint32_t lo[kSearches], hi[kSearches];      // by bins: places [lo, hi) of the searches (hi <= lo: none)
    int shift;                          // kOpDigits: histogram of (key >> shift) & 255
    u64 prefix, mask;                   // only entries with (key & mask) == prefix
    u64 each;                           // kOpDigits: the mass of every one of them, if they are equal logits; otherwise 0
};

struct alignas(16) Shared {
    u64 list[kList];
    u64 run[kList];                     // in the first block: running masses of the sorted list
    u64 digit_mass[256];
    double table[16];                   // 2^(shift + j / 16)
    u64 warp64[kSearches][kThreads / 32];
    u64 below[kSearches];               // masses below the top-p and the draw's bins, and of all entries
    u64 found_mass, found_key;
    Command cmd;
    alignas(16) uint32_t count[kBins];  // entries; afterwards, in the first block, running sums
    union { alignas(16) uint32_t offset[kBins]; alignas(16) float estimate[kBins]; };   // sums of place & 255; afterwards running masses by estimate
    uint32_t digit_count[256];
    uint32_t warp32[kThreads / 32];
    float warp_f[kThreads / 32];
    uint32_t fill;
    float warp_top[kThreads / 32];
    float top, low;                     // greatest logit of the slice, and the least unmasked one
    int32_t first;                      // index of the first greatest logit
    uint32_t found_count;
    int found_at;
    uint32_t from_i[kSearches], to_i[kSearches], before_n[kSearches];   // of each search: its entries in the sorted list, those before
    bool too_many;                      // for the list: the bins are not collected
    int small;                          // bf16: a kept logit is too small for the bins by value
};
static_assert(offsetof(Shared, offset) == offsetof(Shared, count) + sizeof(uint32_t) * kBins, "one array of 2 kBins for the bins by value");
static_assert(offsetof(Shared, count) % 16 == 0 && offsetof(Shared, offset) % 16 == 0 && sizeof(Shared) % 16 == 0, "16-byte accesses");

// Inclusive sums over the block in thread order.  All threads call it; the scratch is free again on return.
template <typename A>
__device__ __forceinline__ A block_scan(A *scratch, A x)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const A other = __shfl_up_sync(0xFFFFFFFFu, x, o);
        if (lane >= o) x += other;
    }
    if (lane == 31) scratch[warp] = x;
    __syncthreads();
    A w = lane < kThreads / 32 ? scratch[lane] : A(0);
#pragma unroll
    for (int o = 1; o < kThreads / 32; o <<= 1) {
        const A other = __shfl_up_sync(0xFFFFFFFFu, w, o);
        if (lane >= o) w += other;
    }
    const A before = __shfl_sync(0xFFFFFFFFu, w, warp > 0 ? warp - 1 : 0);
    __syncthreads();
    return warp > 0 ? x + before : x;
}

// A search's goal: the first entry of the order at which the running count (kind 0) or mass (1: at least, 2: more than)
// gets there.
struct Goal {
    int kind;
    uint32_t count;
    double mass;
    __device__ __forceinline__ bool met(uint32_t c, u64 m) const
    {
        return kind == 0 ? c >= count : kind == 1 ? (double)m >= mass : (double)m > mass;
    }
};

// The first i in [0, n) at which `met` holds, n if none; `met` stays true once it is.  Every thread takes the same way.
template <typename F>
__device__ __forceinline__ uint32_t first_of(uint32_t n, F met)
{
    uint32_t lo = 0, hi = n;
    while (lo < hi) {
        const uint32_t mid = (lo + hi) >> 1;
        if (met(mid)) hi = mid; else lo = mid + 1;
    }
    return lo;
}

// Descending bitonic sort of s.list[0..n).  The entries stay in registers, up to two per thread (512 apart): partners within a
// warp meet by shuffles, those in another warp through the list.  1,000 entries take 5 us, 13 us when every step goes through
// the list.
template <int E>
__device__ __forceinline__ void sort_registers(Shared &s, uint32_t n, uint32_t size)
{
    const uint32_t tid = threadIdx.x;
    u64 key[E];
#pragma unroll
    for (int e = 0; e < E; ++e) key[e] = tid + e * kThreads < n ? s.list[tid + e * kThreads] : 0;     // 0 is no key: it goes last
    for (uint32_t k = 2; k <= size; k <<= 1)
        for (uint32_t j = k >> 1; j > 0; j >>= 1) {
            if (E == 2 && j == (uint32_t)kThreads) {            // both are this thread's; the whole list is one descending run
                const u64 a = key[0], b = key[E - 1];
                key[0] = a > b ? a : b;
                key[E - 1] = a > b ? b : a;
                continue;
            }
            u64 other[E];
            if (j >= 32) {
                __syncthreads();
#pragma unroll
                for (int e = 0; e < E; ++e) s.list[tid + e * kThreads] = key[e];
                __syncthreads();
#pragma unroll
                for (int e = 0; e < E; ++e) other[e] = s.list[(tid ^ j) + e * kThreads];
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) other[e] = __shfl_xor_sync(0xFFFFFFFFu, key[e], j);
            }
            const bool first = (tid & j) == 0;                  // the one of the pair that comes first takes the greater, if descending
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const bool descending = ((tid + e * kThreads) & k) == 0;
                key[e] = (first == descending) == (key[e] > other[e]) ? key[e] : other[e];
            }
        }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < E; ++e) s.list[tid + e * kThreads] = key[e];
    __syncthreads();
}
__device__ __forceinline__ void sort_list(Shared &s, uint32_t n)
{
    static_assert(kList == 2 * kThreads, "two entries per thread");
    uint32_t size = 32;
    while (size < n) size <<= 1;
    if (n <= (uint32_t)kThreads) sort_registers<1>(s, n, size); else sort_registers<2>(s, n, size);
}

// The greatest and the least unmasked value of a vector; NaN counts for neither.
template <typename T>
__device__ __forceinline__ void see_vector(const uint4 &raw, float &top, float &low)
{
    if constexpr (sizeof(T) == 2) {                     // in pairs
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
        const __nv_bfloat162 masked = __float2bfloat162_rn(kMasked);
        __nv_bfloat162 hi, lo;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 x = *reinterpret_cast<const __nv_bfloat162 *>(&w[i]);
            const uint32_t open = __hgt2_mask(x, masked), y = (w[i] & open) | (0x7F807F80u & ~open);      // masked ones: +inf
            const __nv_bfloat162 z = *reinterpret_cast<const __nv_bfloat162 *>(&y);
            hi = i ? __hmax2(hi, x) : x;
            lo = i ? __hmin2(lo, z) : z;
        }
        top = fmaxf(top, fmaxf(__low2float(hi), __high2float(hi)));
        low = fminf(low, fminf(__low2float(lo), __high2float(lo)));
    } else {
        float f[4];
        Elem<float>::unpack(raw, f);
#pragma unroll
        for (int e = 0; e < 4; ++e) { top = fmaxf(top, f[e]); low = fminf(low, f[e] > kMasked ? f[e] : INFINITY); }
    }
}

constexpr int kPerThread = kList / kThreads;       // list entries of a thread, consecutive
constexpr int kBinsPerThread = kBins / kThreads;

template <typename T>
__global__ void __launch_bounds__(kThreads, 2)
tfe_sample_kernel(const SampleParams p)
{
    tfe_wait_for_stream();
    extern __shared__ __align__(16) uint8_t smem[];
    Shared &s = *reinterpret_cast<Shared *>(smem);
    T *slice = reinterpret_cast<T *>(smem + sizeof(Shared));
    constexpr int E = Elem<T>::kPerVec;
    cg::cluster_group cluster = cg::this_cluster();
    const int64_t r = blockIdx.x / p.blocks;
    const int part = (int)(blockIdx.x % p.blocks);
    const bool leader = part == 0;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const T *row = static_cast<const T *>(p.logits) + r * p.ld;

    // ---- this block's slice: whole vectors, and with the first and the last block the row's ends
    const Cut cut = cut_row(row, p.V);
    const int32_t v0 = (int32_t)(cut.n_vec * part / p.blocks), n_vec = (int32_t)(cut.n_vec * (part + 1) / p.blocks) - v0;
    const int32_t body0 = (int32_t)cut.head + v0 * E;
    const int32_t head_n = leader ? (int32_t)cut.head : 0, tail0 = (int32_t)(cut.head + cut.n_vec * E);
    const int32_t ends = head_n + (part == p.blocks - 1 ? p.V - tail0 : 0);
    const bool resident = n_vec * E <= p.slice_cap;
    const uint4 *from = reinterpret_cast<const uint4 *>(row + cut.head) + v0;
    uint4 *keep = reinterpret_cast<uint4 *>(slice);
    auto end_index = [&](int t) { return t < head_n ? t : tail0 + t - head_n; };
    // every entry of the slice, four at a time: take(f, i), f[e] being entry i + e; NaN where there is none
    auto sweep = [&](const uint4 *vectors, auto take) {
        auto take_vector = [&](const uint4 &raw, int32_t i) {
            if constexpr (E == 4) {
                float f[4];
                Elem<T>::unpack(raw, f);
                take(f, i);
            } else {
#pragma unroll 1
                for (int h = 0; h < 2; ++h) {
                    const uint32_t a = h ? raw.z : raw.x, b = h ? raw.w : raw.y;
                    const float f[4] = {__uint_as_float(a << 16), __uint_as_float(a & 0xFFFF0000u), __uint_as_float(b << 16), __uint_as_float(b & 0xFFFF0000u)};
                    take(f, i + 4 * h);
                }
            }
        };
        uint4 next = make_uint4(0, 0, 0, 0);            // one load ahead
        if (tid < n_vec) next = vectors[tid];
#pragma unroll 1
        for (int32_t v = tid; v < n_vec; v += kThreads) {
            const uint4 raw = next;
            if (v + kThreads < n_vec) next = vectors[v + kThreads];
            take_vector(raw, body0 + v * E);
        }
        if (ends && tid < 32) {                         // the row's ends, fewer than 2 E: a turn of their own
            const int32_t i = tid < ends ? end_index(tid) : 0;
            const float f[4] = {tid < ends ? Elem<T>::get(row + i) : __uint_as_float(0x7FFFFFFFu), __uint_as_float(0x7FFFFFFFu),
                                __uint_as_float(0x7FFFFFFFu), __uint_as_float(0x7FFFFFFFu)};
            take(f, i);
        }
    };

    // ---- its greatest and its least logit
    float top = -INFINITY, low = INFINITY;
    {
        auto see = [&](float z) {                       // fmaxf drops NaN
            top = fmaxf(top, z);
            low = fminf(low, z > kMasked ? z : INFINITY);
        };
        constexpr int U = 4;
        for (int32_t v = tid; v < n_vec; v += U * kThreads) {
            uint4 raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                raw[u] = make_uint4(0xFFFFFFFFu, 0xFFFFFFFFu, 0xFFFFFFFFu, 0xFFFFFFFFu);
                if (v + u * kThreads < n_vec) raw[u] = load_stream(from + v + u * kThreads);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (resident && v + u * kThreads < n_vec) keep[v + u * kThreads] = raw[u];
                see_vector<T>(raw[u], top, low);
            }
        }
        if (tid < ends) see(Elem<T>::get(row + end_index(tid)));
    }
    for (int i = tid; i < kBins; i += kThreads) { s.count[i] = 0; s.offset[i] = 0; }
    if (tid < 16) s.table[tid] = exp2((double)tid / 16 + p.shift);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        low = fminf(low, __shfl_xor_sync(0xFFFFFFFFu, low, o));
    }
    if (lane == 0) { s.warp_f[warp] = low; s.warp_top[warp] = top; }
    __syncthreads();
    if (warp == 0) {
        top = lane < kThreads / 32 ? s.warp_top[lane] : -INFINITY;
        low = lane < kThreads / 32 ? s.warp_f[lane] : INFINITY;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
            low = fminf(low, __shfl_xor_sync(0xFFFFFFFFu, low, o));
        }
        if (lane == 0) { s.top = top; s.low = low; s.first = 0x7FFFFFFF; s.small = 0; }
    }
    cluster.sync();
    top = -INFINITY;
    low = INFINITY;
    for (int b = 0; b < p.blocks; ++b) {
        top = fmaxf(top, *cluster.map_shared_rank(&s.top, b));
        low = fminf(low, *cluster.map_shared_rank(&s.low, b));
    }

    // ---- the row's rule
    const float T_ = p.temperature ? p.temperature[r] : 1.f;
    if (!(top > -INFINITY) || !(T_ > 0.f)) {            // nothing to draw from, or greedy: the same in every block
        if (top > -INFINITY) {
            int32_t first = 0x7FFFFFFF;
            sweep(resident ? keep : from, [&](const float (&f)[4], int32_t i) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (f[e] == top) first = min(first, i + e);
            });
            first = __reduce_min_sync(0xFFFFFFFFu, first);
            if (lane == 0 && first != 0x7FFFFFFF) atomicMin(&s.first, first);
        }
        cluster.sync();
        if (leader && tid == 0) {
            int32_t first = 0x7FFFFFFF;
            for (int b = 0; b < p.blocks; ++b) first = min(first, *cluster.map_shared_rank(&s.first, b));
            p.tokens[r] = top > -INFINITY ? first : -1;
            if (p.prob) p.prob[r] = top > -INFINITY ? 1.f : 0.f;
        }
        cluster.sync();                 // a block's shared memory lives until the first has read it
        return;
    }
    const float min_p = p.min_p ? p.min_p[r] : 0.f;
    RowRule q;
    q.topf = top;
    q.top = (double)fminf(q.topf, 3.402823466e38f);
    q.a = 16 * 1.4426950408889634 / (double)T_;
    {
        const double least = !(min_p > 0.f) ? -INFINITY
                             : min_p >= 1.f ? (double)q.topf : __dadd_rn((double)q.topf, __dmul_rn((double)T_, log((double)min_p)));
        q.cut = fmaxf(__double2float_ru(least), -3.402823466e38f);          // NaN (infinite maximum and temperature): the lowest
        if (q.topf == INFINITY) q.cut = INFINITY;                           // its equals share the draw, whatever the temperature
        // -ln w = ln 2 (shift + 2): a quarter of the unit.  What lies beyond that reach weighs nothing.
        const double reach = 0.6931471805599453 * (double)(p.shift + 2) * (double)T_;
        // So does the next logit below the maximum where it lies beyond the reach: weighed at that step, it would leave the range
        // of weight_of's exponent.  Otherwise a step is at most the reach, and rounding the floor down adds less than three of it.
        const double end = (double)q.topf - reach;
        q.floor = fmaxf(__double2float_rd(end), -3.402823466e38f);
        if (!((double)nextafterf(q.topf, -INFINITY) > end)) { q.cut = q.topf; q.floor = q.topf; }
    }
    const float inv_t = 1.f / T_;
    float range = fminf(kRange, (q.topf - low) * inv_t);                    // NaN: kRange
    if (!(range >= 0.f)) range = kRange;                                    // no unmasked logit
    const float width = range / (float)(kBins - 2);                         // of a bin, in units of -ln w
    // the last bin is for what lies beyond the range: masked logits, weights below exp(-kRange); it is estimated to weigh nothing
    q.bins = fminf(256.f * (float)(kBins - 2) / range * inv_t, 3.402823466e38f);  // T tiny, or all logits equal: one step is all bins
    if (!(inv_t > 0.f)) q.bins = 0.f;                                       // T infinite: all in the first bin
    const uint4 *src = resident ? keep : from;

    // ---- bf16: counts by value.  A bin holds one value -- 31 binades of either sign, 128 values each, and zero -- so that the
    // masses of the bins, and with them every search's end, are exact without weighing the entries one by one.  Rows with a kept
    // logit below those binades but zero (of 152,000 normal ones one row in a thousand) take the bins by distance.  Logits at
    // which nothing of a weight is left are not counted: they end no search but one by count, whose mass they do not change.
    bool by_value = sizeof(T) == 2 && q.topf < INFINITY;
    const float least = fmaxf(fmaxf(q.cut, q.floor), q.floor > kMasked ? low : -INFINITY);
    const int below_binades = max(1, (int)max(__float_as_uint(top) << 1 >> 24, __float_as_uint(least) << 1 >> 24) - 30) << 7;
    uint32_t *by_values = reinterpret_cast<uint32_t *>(smem + offsetof(Shared, count));      // 2 kBins, `count` and `offset`
    auto value_at = [&](uint32_t at) {                  // of a bin; bins in descending order
        const uint32_t h = at < (uint32_t)kBins ? kBins - 1 - at : at - kBins;
        return h == 0 ? 0.f : __uint_as_float((h - 128 + below_binades) << 16 | (at < (uint32_t)kBins ? 0u : 0x80000000u));
    };
    if (by_value) {
        const int up = kBins - 1 - 128 + below_binades;
        const __nv_bfloat162 least2 = __bfloat162bfloat162(__float2bfloat16_ru(least));
        const uint32_t up2 = (uint32_t)((up - 32767) & 0xFFFF) * 0x10001u, one2 = (uint32_t)((kBins - 1 - 32767) & 0xFFFF) * 0x10001u;
        constexpr uint32_t two2 = (uint32_t)(kBins - 2) * 0x10001u;
        // two logits at a time.  With mag the bits but the sign, h is 0 for zero, mag - below_binades + 128 for what the binades
        // hold, and 1 to 127 for what they do not: kBins - 1 - h = min(up - mag, max(kBins - 1 - mag, kBins - 2)).
        auto count_pair = [&](uint32_t w) {
            const uint32_t back = __viaddmin_s16x2(~w & 0x7FFF7FFFu, up2, __viaddmax_s16x2(~w & 0x7FFF7FFFu, one2, two2));
            const uint32_t at = (back ^ __vcmplts2(w, 0)) & (uint32_t)(2 * kBins - 1) * 0x10001u;         // negative: kBins + h
            const uint32_t kept = __hge2_mask(*reinterpret_cast<const __nv_bfloat162 *>(&w), least2);
            if (kept & 0xFFFFu) atomicAdd(&by_values[at & 0xFFFFu], 1u);
            if (kept >> 16) atomicAdd(&by_values[at >> 16], 1u);
        };
        uint4 next = make_uint4(0, 0, 0, 0);            // one load ahead
        if (tid < n_vec) next = src[tid];
#pragma unroll 1
        for (int32_t v = tid; v < n_vec; v += kThreads) {
            const uint4 raw = next;
            if (v + kThreads < n_vec) next = src[v + kThreads];
            count_pair(raw.x); count_pair(raw.y); count_pair(raw.z); count_pair(raw.w);
        }
        if (tid < ends) count_pair(0xFFFF0000u | __float_as_uint(Elem<T>::get(row + end_index(tid))) >> 16);      // and a NaN
        __syncthreads();
        if (tid < 127 && (by_values[kBins - 2 - tid] | by_values[kBins + 1 + tid])) s.small = 1;        // h of 1 to 127
        cluster.sync();
        for (int b = 0; b < p.blocks; ++b) by_value = by_value && *cluster.map_shared_rank(&s.small, b) == 0;
        if (!by_value)
            for (int i = tid; i < kBins; i += kThreads) { s.count[i] = 0; s.offset[i] = 0; }
        __syncthreads();
    }

    // ---- counts by bin; the last one, where masked logits and all weights of a cold row beyond the range meet, in registers
    if (!by_value) {
        uint32_t in_last = 0;
        sweep(src, [&](const float (&f)[4], int32_t) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t place = place_of(q, f[e]);
                if (f[e] >= q.cut) {
                    if (place < 256u * (kBins - 1)) {
                        atomicAdd(&s.count[place >> 8], 1u);
                        atomicAdd(&s.offset[place >> 8], place & 255u);
                    } else {
                        ++in_last;
                    }
                }
            }
        });
        in_last = __reduce_add_sync(0xFFFFFFFFu, in_last);
        if (lane == 0 && in_last) atomicAdd(&s.count[kBins - 1], in_last);
        cluster.sync();
    }
    if (p.blocks > 1) {                 // every block adds up its share of the bins
        const int share = kBins / p.blocks;
        for (int i = tid; i < share; i += kThreads) {
            const int b = part * share + i;
            uint32_t c = 0, o = 0;
            for (int other = 0; other < p.blocks; ++other) {
                c += cluster.map_shared_rank(s.count, other)[b];
                o += cluster.map_shared_rank(s.offset, other)[b];
            }
            s.count[b] = c; s.offset[b] = o;
        }
        cluster.sync();
        if (leader) {
#pragma unroll 4
            for (int b = share + tid; b < kBins; b += kThreads) {
                s.count[b] = cluster.map_shared_rank(s.count, b / share)[b];
                s.offset[b] = cluster.map_shared_rank(s.offset, b / share)[b];
            }
            __syncthreads();
        }
    }

    // ---- the first block decides, every block looks through its slice
    uint32_t base_n = 0, list_n = 0;
    u64 base_m = 0, limit = 0;                          // limit: mass of the prefix that is still in
    int stage = kDraw;

    auto share_of = [&](int st) {       // of the limit: what top-p wants reached, or the draw exceeded
        return st == kTopP ? fmaxf(p.top_p[r], 0.f) : fminf(fmaxf(p.u[r], 0.f), 1.f - 0x1p-24f);      // NaN: 0
    };
    auto goal_of = [&](int st) {
        Goal g;
        g.kind = st == kTopK ? 0 : st == kTopP ? 1 : 2;
        g.count = st == kTopK ? (uint32_t)p.top_k[r] : 0;
        g.mass = st == kTopK ? 0.0 : (double)share_of(st) * (double)limit;
        return g;
    };
    auto next_stage = [&](int st) { return st == kTopK && p.top_p && p.top_p[r] < 1.f ? (int)kTopP : (int)kDraw; };
    auto digits = [&](int shift, u64 prefix, u64 mask, u64 each) {
        if (tid == 0) { s.cmd.op = kOpDigits; s.cmd.shift = shift; s.cmd.prefix = prefix; s.cmd.mask = mask; s.cmd.each = each; }
    };
    // The entry at which the goal of `stage` is met, among list entries [i0, i1) with base_n entries of mass base_m before
    // them.  False if it is not among them.
    auto find_entry = [&](uint32_t i0, uint32_t i1, u64 &mass, u64 &key) {
        if (i1 <= i0) return false;
        const Goal g = goal_of(stage);
        const u64 off = base_m - (i0 ? s.run[i0 - 1] : 0);
        const uint32_t i = i0 + first_of(i1 - i0, [&](uint32_t j) { return g.met(base_n + j + 1, off + s.run[i0 + j]); });
        if (i >= i1 || (base_n > 0 && i == i0 && g.met(base_n, base_m))) return false;
        mass = off + s.run[i];
        key = s.list[i];
        return true;
    };

    // The bins [lo, hi) in which the searches from `stage` on end, as many of them as the list has room for, and what to do.
    auto plan = [&](bool first) {
        uint32_t from_i[kSearches] = {0, 0, 0}, to_i[kSearches] = {0, 0, 0}, before_n[kSearches] = {0, 0, 0};
        uint32_t lo[kSearches] = {0, 0, 0}, hi[kSearches] = {0, 0, 0};
        // mass that is still in, and by how much it may be more
        float kept_m = first ? s.estimate[kBins - 1] : (float)limit * exp2f((float)-p.shift), spare = 0.f;
        uint32_t behind = kBins;                                // no search ends behind the one before it
        bool whole = false;
        auto counted = [&](uint32_t b) { return b ? s.count[b - 1] : 0; };       // entries in the bins before b
        for (int st = stage;; st = next_stage(st)) {
            if (st == kTopK) {
                const uint32_t k = (uint32_t)p.top_k[r], b = first_of(kBins - 1, [&](uint32_t i) { return s.count[i] >= k; });
                const float m0 = b ? s.estimate[b - 1] : 0.f;
                kept_m = m0 + (s.estimate[b] - m0) * ((float)(k - counted(b)) / (float)(s.count[b] - counted(b)));
                lo[st] = b; hi[st] = behind = b + 1;    // exact: counts
            } else {
                const float share = share_of(st), slack = 1e-5f * s.estimate[kBins - 1];
                const float least = share * kept_m - slack, most = share * (kept_m + spare) + slack;
                lo[st] = first_of(kBins - 1, [&](uint32_t i) { return s.estimate[i] > least; });
                hi[st] = min(first_of(kBins - 1, [&](uint32_t i) { return s.estimate[i] > most; }) + 1, behind);
                lo[st] = min(lo[st], hi[st] - 1);
                behind = hi[st];
                kept_m = share * kept_m;
                spare = share * spare + __expf(-width * (float)lo[st]);      // the entry that reaches the goal is part
            }
            if (st == stage && st != kDraw && s.count[hi[st] - 1] <= (uint32_t)kList) {
                whole = true;                           // a short prefix is collected whole
                for (int t = 0; t < kSearches; ++t) { hi[t] = hi[st]; lo[t] = 0; }
                for (int t = 0; t < kSearches; ++t) { from_i[t] = 0; to_i[t] = s.count[hi[st] - 1]; before_n[t] = 0; }
                break;
            }
            if (st == kDraw) break;
        }
        bool too_many = false;
        for (int last = kDraw; !whole; --last) {        // where each search's entries stand in the sorted list of all
            uint32_t need = 0, end = 0;                 // bins before `end` are in the list, or above every search's
#pragma unroll
            for (int st = kDraw; st >= kTopK; --st) {
                if (st > last) hi[st] = lo[st] = from_i[st] = to_i[st] = 0;      // no room: a later pass
                if (hi[st] > lo[st]) {
                    before_n[st] = counted(lo[st]);
                    const uint32_t shared = lo[st] < end ? counted(min(end, hi[st])) - counted(lo[st]) : 0;
                    const uint32_t beyond = lo[st] < end && end > hi[st] ? counted(end) - counted(hi[st]) : 0;
                    from_i[st] = need - shared - beyond;
                    to_i[st] = from_i[st] + counted(hi[st]) - counted(lo[st]);
                    need = max(need, to_i[st]);
                    end = max(end, hi[st]);
                }
            }
            too_many = need > (uint32_t)kList;
            if (!too_many || last <= stage) break;
        }
        __syncthreads();                                // the last plan and command have been read
        if (tid == 0) {
            s.too_many = too_many;
            for (int st = 0; st < kSearches; ++st) { s.from_i[st] = from_i[st]; s.to_i[st] = to_i[st]; s.before_n[st] = before_n[st]; }
            s.cmd.op = kOpCollect;
            s.cmd.by_bins = 1;
            s.cmd.first = first;
            s.cmd.sums = !first || stage != kTopK ? 2 : whole ? 0 : 1;
            for (int st = 0; st < kSearches; ++st) { s.cmd.lo[st] = 256 * lo[st]; s.cmd.hi[st] = too_many ? 0 : 256 * hi[st]; }
        }
    };

    if (leader && by_value) {
        const uint32_t *counts = by_values + tid * 2 * kBinsPerThread;
        uint32_t c_sum = 0;
        u64 m_sum = 0;
        if (tid == 0) { by_values[kBins - 1] += by_values[kBins]; by_values[kBins] = 0; }      // -0 and +0 are equal logits
        __syncthreads();
#pragma unroll 4
        for (int j = 0; j < 2 * kBinsPerThread; ++j) {
            const uint32_t n = counts[j];
            c_sum += n;
            if (__any_sync(0xFFFFFFFFu, n)) m_sum += n * mass_of(q, s.table, value_at(tid * 2 * kBinsPerThread + j));
        }
        const uint32_t c_run = block_scan(s.warp32, c_sum);
        const u64 m_run = block_scan(s.warp64[0], m_sum);
        if (tid == kThreads - 1) { s.found_count = c_run; s.found_mass = m_run; }
        __syncthreads();
        const int32_t k = p.top_k ? p.top_k[r] : 0;
        stage = k > 0 && (uint32_t)k < s.found_count ? kTopK : next_stage(kTopK);
        limit = s.found_mass;
        int at;
        uint32_t n;
        for (;;) {                                      // at most three searches
            __syncthreads();
            if (tid == 0) s.found_at = -1;
            __syncthreads();
            const Goal g = goal_of(stage);
            uint32_t n0 = c_run - c_sum;
            u64 m0 = m_run - m_sum;
            const uint32_t in = __ballot_sync(0xFFFFFFFFu, c_sum && g.met(c_run, m_run) && (n0 == 0 || !g.met(n0, m0)));
            if (in) {                                   // this warp has the end: its bins, one per lane
                static_assert(2 * kBinsPerThread <= 32, "a thread's bins fit a warp");
                const int of = __ffs(in) - 1, bin = ((tid & ~31) + of) * 2 * kBinsPerThread + lane;
                n0 = __shfl_sync(0xFFFFFFFFu, n0, of);
                m0 = __shfl_sync(0xFFFFFFFFu, m0, of);
                const uint32_t here = lane < 2 * kBinsPerThread ? by_values[bin] : 0;
                const u64 each = here ? mass_of(q, s.table, value_at(bin)) : 0;
                uint32_t n1 = here;
                u64 m1 = here * each;
#pragma unroll
                for (int o = 1; o < 2 * kBinsPerThread; o <<= 1) {
                    const uint32_t n_up = __shfl_up_sync(0xFFFFFFFFu, n1, o);
                    const u64 m_up = __shfl_up_sync(0xFFFFFFFFu, m1, o);
                    if (lane >= o) { n1 += n_up; m1 += m_up; }
                }
                n1 += n0 - here;                        // before this bin
                m1 += m0 - here * each;
                if (here && g.met(n1 + here, m1 + here * each) && (n1 == 0 || !g.met(n1, m1))) {
                    const uint32_t i = first_of(here - 1, [&](uint32_t x) { return g.met(n1 + x + 1, m1 + (x + 1) * each); });
                    s.found_at = bin;
                    s.found_count = here;
                    s.found_mass = m1 + (i + 1) * each;
                    s.found_key = m1;
                    s.before_n[0] = n1;
                }
            }
            __syncthreads();
            at = s.found_at;
            n = s.found_count;
            if (at < 0 || stage == kDraw) break;
            limit = s.found_mass;
            stage = next_stage(stage);
        }
        if (at < 0) {
            digits(56, 0, 0, 0);
        } else {                                        // the drawn value is known: which of its entries, in index order
            base_n = s.before_n[0];
            base_m = s.found_key;
            const float z = value_at(at);
            int bits = 8;                               // of an index
            while (bits < 32 && (p.V - 1) >> bits) ++bits;
            const u64 prefix = entry_key(z, 0) & 0xFFFFFFFF00000000ull;
            if (n <= (uint32_t)kList) {
                if (tid == 0) { s.cmd.op = kOpCollect; s.cmd.by_bins = 0; s.cmd.prefix = prefix; s.cmd.mask = 0xFFFFFFFF00000000ull; }
            } else {                                    // the bits that all indexes have alike are ones in a key
                const u64 alike = 0xFFFFFFFFull >> bits << bits;
                digits(bits - 8, prefix | alike, 0xFFFFFFFF00000000ull | alike, mass_of(q, s.table, z));
            }
        }
    } else if (leader) {
        // running counts, and running masses estimated from the bins' means
        uint32_t c[kBinsPerThread], c_sum = 0;
        float m[kBinsPerThread], m_sum = 0.f;
        uint4 *counts = reinterpret_cast<uint4 *>(s.count + tid * kBinsPerThread), *offsets = reinterpret_cast<uint4 *>(s.offset + tid * kBinsPerThread);
#pragma unroll
        for (int h = 0; h < kBinsPerThread / 4; ++h) {
            const uint4 cv = counts[h], ov = offsets[h];
            const uint32_t cc[4] = {cv.x, cv.y, cv.z, cv.w}, oo[4] = {ov.x, ov.y, ov.z, ov.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float n = (float)cc[j], mean = (float)(tid * kBinsPerThread + h * 4 + j) + __fdividef((float)oo[j], 256.f * n);
                m_sum += cc[j] && tid * kBinsPerThread + h * 4 + j < kBins - 1 ? n * __expf(-width * mean) : 0.f;
                c_sum += cc[j];
                c[h * 4 + j] = c_sum;
                m[h * 4 + j] = m_sum;
            }
        }
        const uint32_t c_before = block_scan(s.warp32, c_sum) - c_sum;
        const float m_before = block_scan(s.warp_f, m_sum) - m_sum;
#pragma unroll
        for (int h = 0; h < kBinsPerThread / 4; ++h) {
            counts[h] = make_uint4(c[4 * h] + c_before, c[4 * h + 1] + c_before, c[4 * h + 2] + c_before, c[4 * h + 3] + c_before);
            float4 *e = reinterpret_cast<float4 *>(s.estimate + tid * kBinsPerThread);
            e[h] = make_float4(m[4 * h] + m_before, m[4 * h + 1] + m_before, m[4 * h + 2] + m_before, m[4 * h + 3] + m_before);
        }
        __syncthreads();
        const int32_t k = p.top_k ? p.top_k[r] : 0;
        // a k-th entry in the last bin restricts nothing: what is there weighs nothing (the range's end is below the unit of the
        // masses, and masked logits are, unless the temperature is beyond any use).  Infinite maxima are there too, and weigh.
        const bool last_is_nothing = q.topf < INFINITY && (range == kRange || mass_of(q, s.table, kMasked) == 0);
        const uint32_t countable = last_is_nothing ? s.count[kBins - 2] : s.count[kBins - 1];
        const bool k_on = k > 0 && (uint32_t)k < s.count[kBins - 1] && ((uint32_t)k <= countable || !last_is_nothing);
        stage = k_on ? kTopK : next_stage(kTopK);
        plan(true);
    }

    for (;;) {
        cluster.sync();
        const Command cmd = *cluster.map_shared_rank(&s.cmd, 0);
        if (cmd.op == kOpDone) break;
        if (tid == 0) s.fill = 0;
        if (cmd.op == kOpDigits && tid < 256) { s.digit_count[tid] = 0; s.digit_mass[tid] = 0; }
        __syncthreads();
        auto push = [&](u64 key) {
            const uint32_t at = atomicAdd(&s.fill, 1u);
            if (at < (uint32_t)kList) s.list[at] = key;
        };
        // where the prefix names a logit, four entries at a time are passed over if none has it
        const bool one_value = cmd.mask >> 32 == 0xFFFFFFFFu;
        const float value = key_logit(cmd.prefix);
        auto none = [&](const float (&f)[4]) { return one_value && f[0] != value && f[1] != value && f[2] != value && f[3] != value; };
        if (cmd.op == kOpDigits) {
            sweep(src, [&](const float (&f)[4], int32_t at) {
                if (none(f)) return;
#pragma unroll 1
                for (int e = 0; e < 4; ++e) {
                    if (!(f[e] >= q.cut)) continue;
                    const u64 key = entry_key(f[e], at + e);
                    if ((key & cmd.mask) != cmd.prefix) continue;
                    const int d = (int)((key >> cmd.shift) & 255u);
                    atomicAdd(&s.digit_count[d], 1u);
                    if (!cmd.each) atomicAdd(&s.digit_mass[d], mass_of(q, s.table, f[e]));
                }
            });
        } else if (sizeof(T) == 2 && !cmd.by_bins && one_value) {       // in pairs, several loads at once
            const __nv_bfloat162 value2 = __float2bfloat162_rn(value);
            auto take_pair = [&](uint32_t w, int32_t at) {
                const uint32_t is = __heq2_mask(*reinterpret_cast<const __nv_bfloat162 *>(&w), value2);
                if (is & 0xFFFFu) if (const u64 key = entry_key(value, at); (key & cmd.mask) == cmd.prefix) push(key);
                if (is >> 16) if (const u64 key = entry_key(value, at + 1); (key & cmd.mask) == cmd.prefix) push(key);
            };
            constexpr int U = 4;
#pragma unroll 1
            for (int32_t v = tid; v < n_vec; v += U * kThreads) {
                uint4 raw[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    raw[u] = make_uint4(0xFFFFFFFFu, 0xFFFFFFFFu, 0xFFFFFFFFu, 0xFFFFFFFFu);
                    if (v + u * kThreads < n_vec) raw[u] = src[v + u * kThreads];
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    auto is = [&](uint32_t w) { return __heq2_mask(*reinterpret_cast<const __nv_bfloat162 *>(&w), value2); };
                    if (is(raw[u].x) | is(raw[u].y) | is(raw[u].z) | is(raw[u].w)) {
                        const int32_t at = body0 + (v + u * kThreads) * E;
                        take_pair(raw[u].x, at); take_pair(raw[u].y, at + 2); take_pair(raw[u].z, at + 4); take_pair(raw[u].w, at + 6);
                    }
                }
            }
            if (tid < ends) take_pair(0xFFFF0000u | __float_as_uint(Elem<T>::get(row + end_index(tid))) >> 16, end_index(tid));
        } else if (!cmd.by_bins) {
            sweep(src, [&](const float (&f)[4], int32_t at) {
                if (none(f)) return;
#pragma unroll 1
                for (int e = 0; e < 4; ++e) {
                    const u64 key = entry_key(f[e], at + e);
                    if (f[e] >= q.cut && (key & cmd.mask) == cmd.prefix) push(key);
                }
            });
        } else {
            // all searches' places in one span; which of them an entry belongs to is asked of the few inside
            uint32_t span_lo = 0xFFFFFFFFu, span_hi = 0;
#pragma unroll
            for (int st = 0; st < kSearches; ++st)
                if (cmd.hi[st] > cmd.lo[st]) { span_lo = min(span_lo, cmd.lo[st]); span_hi = max(span_hi, cmd.hi[st]); }
            const uint32_t span = span_hi > span_lo ? span_hi - span_lo : 0;
            auto collect = [&](const float (&f)[4], int32_t at) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t place = place_of(q, f[e]);
                    bool in = false;
#pragma unroll
                    for (int st = 0; st < kSearches; ++st) in = in || (place >= cmd.lo[st] && place < cmd.hi[st]);
                    if (in && f[e] >= q.cut) push(entry_key(f[e], at + e));
                }
            };
            if (cmd.sums == 0) {
                sweep(src, [&](const float (&f)[4], int32_t at) {
                    bool any = false;
#pragma unroll
                    for (int e = 0; e < 4; ++e) any = any || place_of(q, f[e]) - span_lo < span;
                    if (any) collect(f, at);
                });
            } else {
                // masses below the draw's bins, below top-p's, and of all entries (or those below top-k's): whole numbers of at most
                // 2^46, four of them exact in a double, then added up as integers
                const uint32_t lo_all = cmd.sums == 2 ? 0xFFFFFFFFu : cmd.lo[kTopK], lo_p = cmd.lo[kTopP], lo_u = cmd.lo[kDraw];
                u64 sum_u = 0, sum_p = 0, sum_all = 0;
                sweep(src, [&](const float (&f)[4], int32_t at) {
                    double part_u = kWhole, part_p = kWhole, part_all = kWhole;
                    bool any = false;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t place = f[e] >= q.cut ? place_of(q, f[e]) : 0xFFFFFFFFu;
                        const double w = weight_of(q, s.table, f[e], kWhole) - kWhole;
                        part_all = fma(w, __hiloint2double(place < lo_all ? 0x3FF00000 : 0, 0), part_all);      // times 1 or 0
                        part_p = fma(w, __hiloint2double(place < lo_p ? 0x3FF00000 : 0, 0), part_p);
                        part_u = fma(w, __hiloint2double(place < lo_u ? 0x3FF00000 : 0, 0), part_u);
                        any = any || place - span_lo < span;
                    }
                    sum_all += whole_of(part_all);
                    sum_p += whole_of(part_p);
                    sum_u += whole_of(part_u);
                    if (any) collect(f, at);
                });
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    sum_all += __shfl_xor_sync(0xFFFFFFFFu, sum_all, o);
                    sum_p += __shfl_xor_sync(0xFFFFFFFFu, sum_p, o);
                    sum_u += __shfl_xor_sync(0xFFFFFFFFu, sum_u, o);
                }
                if (lane == 0) { s.warp64[0][warp] = sum_all; s.warp64[1][warp] = sum_p; s.warp64[2][warp] = sum_u; }
                __syncthreads();
                if (tid < kSearches) {
                    u64 total = 0;
                    for (int w = 0; w < kThreads / 32; ++w) total += s.warp64[tid][w];
                    s.below[tid] = total;
                }
            }
        }
        cluster.sync();
        if (!leader) continue;
        if (cmd.op == kOpCollect) {
            uint32_t n_of[8];
#pragma unroll
            for (int b = 0; b < 8; ++b) n_of[b] = b < p.blocks ? *cluster.map_shared_rank(&s.fill, b) : 0;
            list_n = n_of[0];
#pragma unroll
            for (int b = 1; b < 8; ++b)
                if (b < p.blocks) {
                    const u64 *theirs = cluster.map_shared_rank(s.list, b);
                    for (uint32_t i = tid; i < n_of[b] && list_n + i < (uint32_t)kList; i += kThreads) s.list[list_n + i] = theirs[i];
                    list_n += n_of[b];
                }
            list_n = min(list_n, (uint32_t)kList);
            __syncthreads();
            sort_list(s, list_n);
            u64 sum = 0, own[kPerThread];
#pragma unroll
            for (int j = 0; j < kPerThread; ++j) {
                const uint32_t i = (uint32_t)(tid * kPerThread + j);
                if (i < list_n) sum += mass_of(q, s.table, key_logit(s.list[i]));
                own[j] = sum;
            }
            const u64 before = block_scan(s.warp64[0], sum) - sum;
#pragma unroll
            for (int j = 0; j < kPerThread; ++j) s.run[tid * kPerThread + j] = own[j] + before;
            __syncthreads();
            u64 key = 0, mass = 1;
            bool done = true, later = false;
            if (cmd.by_bins) {
                u64 below[kSearches] = {0, 0, 0};
                if (cmd.sums)
                    for (int b = 0; b < p.blocks; ++b)
#pragma unroll
                        for (int i = 0; i < kSearches; ++i) below[i] += cluster.map_shared_rank(s.below, b)[i];
                if (cmd.first && stage != kTopK) limit = below[0];
                done = !s.too_many;
                const int planned = stage;
                while (done) {
                    if (s.to_i[stage] == 0) {           // this search was left for another pass, and starts from an exact limit;
                        later = stage != planned;       // or the estimate named empty bins: by digits (every pass ends a search)
                        done = later;
                        break;
                    }
                    base_n = s.before_n[stage];
                    base_m = stage == kTopK ? below[0] : stage == kTopP ? below[1] : below[2];
                    done = find_entry(s.from_i[stage], min(s.to_i[stage], list_n), mass, key);
                    if (!done || stage == kDraw) break;
                    limit = mass;
                    stage = next_stage(stage);
                }
            } else {
                // a selection by digits ends on the goal's entry
                if (!find_entry(0, list_n, mass, key)) { key = list_n ? s.list[0] : entry_key(q.topf, 0); mass = limit; }
                if (stage != kDraw) {                   // the next search, by digits again
                    limit = mass;
                    stage = next_stage(stage);
                    done = false;
                }
            }
            if (later) {
                plan(false);
            } else if (done) {
                if (tid == 0) {
                    p.tokens[r] = key_index(key);
                    const float z = key_logit(key);
                    if (p.prob) p.prob[r] = (float)(weight_of(q, s.table, z, 0.0) / (double)limit);
                    s.cmd.op = kOpDone;
                }
            } else {
                base_n = 0; base_m = 0;
                digits(56, 0, 0, 0);
            }
        } else {
            // digits in descending order: thread t holds digit 255 - t
            const int d = 255 - tid;
            uint32_t c = 0;
            u64 m = 0;
            if (tid < 256)
                for (int b = 0; b < p.blocks; ++b) { c += cluster.map_shared_rank(s.digit_count, b)[d]; m += cluster.map_shared_rank(s.digit_mass, b)[d]; }
            if (cmd.each) m = c * cmd.each;
            const uint32_t c_run = block_scan(s.warp32, c);
            const u64 m_run = block_scan(s.warp64[0], m);
            const Goal g = goal_of(stage);
            if (tid == 0) { s.found_at = 0; s.found_count = 0; s.found_key = 0; s.found_mass = 0; }
            __syncthreads();
            if (tid < 256 && c && g.met(base_n + c_run, base_m + m_run) &&
                (base_n + c_run - c == 0 || !g.met(base_n + c_run - c, base_m + m_run - m))) {
                s.found_at = d; s.found_count = c; s.found_key = (u64)(c_run - c); s.found_mass = m_run - m;
            }
            __syncthreads();
            const u64 prefix = cmd.prefix | ((u64)s.found_at << cmd.shift), mask = cmd.mask | (255ull << cmd.shift);
            const uint32_t inside = s.found_count;
            base_n += (uint32_t)s.found_key;
            base_m += s.found_mass;
            __syncthreads();
            if (inside <= (uint32_t)kList || cmd.shift == 0) {
                if (tid == 0) { s.cmd.op = kOpCollect; s.cmd.by_bins = 0; s.cmd.prefix = prefix; s.cmd.mask = mask; }
            } else {
                digits(cmd.shift - 8, prefix, mask, cmd.each);
            }
        }
    }
    cluster.sync();                     // the first block's command is read by now
}

}  // namespace

extern "C" tfe_status tfe_sample_tokens(const void *logits, int32_t dtype, int32_t B, int32_t V, int64_t ld,
                                        const tfe_sample_params *params, const float *u, int32_t *tokens, float *prob, void *stream_)
{
    if (!params || (dtype != TFE_DTYPE_BF16 && dtype != TFE_DTYPE_F32)) return TFE_ERR_INVALID_ARG;
    const int es = dtype == TFE_DTYPE_BF16 ? 2 : 4;
    if (B < 0 || B > TFE_ROWS_MAX || V < 1 || V > TFE_SAMPLE_MAX_VOCAB || ld < V || ld > (1ll << 34)) return TFE_ERR_INVALID_ARG;
    if (B == 0) return TFE_OK;
    if (!logits || reinterpret_cast<uintptr_t>(logits) % es != 0 || !u || !tokens) return TFE_ERR_INVALID_ARG;
    for (const void *a : {(const void *)u, (const void *)tokens, (const void *)prob, (const void *)params->temperature, (const void *)params->top_k,
                          (const void *)params->top_p, (const void *)params->min_p})
        if (reinterpret_cast<uintptr_t>(a) % 4 != 0) return TFE_ERR_INVALID_ARG;
    SampleParams p{};
    p.logits = logits; p.ld = ld; p.B = B; p.V = V;
    p.temperature = params->temperature; p.top_k = params->top_k; p.top_p = params->top_p; p.min_p = params->min_p; p.u = u;
    p.tokens = tokens; p.prob = prob;
    int dev = 0, sms = 0;
    if (tfe_status st = tfe_note_cuda(cudaGetDevice(&dev), "cudaGetDevice")) return st;
    if (tfe_status st = tfe_note_cuda(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev), "cudaDeviceGetAttribute")) return st;
    // up to 8 blocks a row while two blocks per SM have room for all rows, none with less than 2,048 logits
    p.blocks = 1;
    while (p.blocks < 8 && V / (2 * p.blocks) >= 2048 && (int64_t)B * 2 * p.blocks <= 2 * sms) p.blocks *= 2;
    // masses sum to less than 2^63
    int bits = 0;
    while ((1ll << bits) < V) ++bits;
    p.shift = std::min(45, 62 - bits);                  // exp(-kRange) rounds to nothing
    // a slice stays in shared memory where that leaves every SM the blocks it would otherwise have
    const int64_t want = ((int64_t)V * es / 16 / p.blocks + 1) * (16 / es);
    const int64_t room = ((int64_t)B * p.blocks <= sms ? 226 : 112) * 1024 - (int64_t)sizeof(Shared);
    p.slice_cap = want * es <= room ? (int32_t)want : 0;
    const size_t smem = sizeof(Shared) + (size_t)p.slice_cap * es;
    auto kernel = dtype == TFE_DTYPE_BF16 ? tfe_sample_kernel<__nv_bfloat16> : tfe_sample_kernel<float>;
    if (tfe_status st = tfe_note_cuda(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024), "sampling attribute")) return st;
    return tfe_launch_serial(kernel, (unsigned)B * (unsigned)p.blocks, kThreads, (unsigned)p.blocks, smem, static_cast<cudaStream_t>(stream_), "sampling launch", p);
}

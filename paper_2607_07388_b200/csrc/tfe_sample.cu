// Drawing the next token of every sequence from its logits: temperature, min-p, top-k and top-p, then one draw by a given
// random number.  (The paper's lookups are keyed by the token ids that decoding produces; it names no sampling rule.)
//
// With x_i = (z_i - z_max) / T and w_i = exp(x_i), every restriction keeps a prefix of one order -- descending logit, equal
// logits by ascending index -- so the whole operator is three searches on that order's running mass:
//     min-p   drops entries with z < z_max + T ln(min_p)              (a comparison, before anything is counted)
//     top-k   the first k entries; their mass is S1
//     top-p   the shortest prefix of them with a mass of at least p S1; its mass is S2
//     draw    the first entry whose running mass exceeds u S2
// No sort of the row: a histogram of counts and masses over (z_max - z) / T locates each search's bin, and only that
// bin's entries (or, where the kept prefix is short, all entries up to it) are collected and sorted.
//
// A row is taken by a cluster of blocks, each holding its slice of the logits in shared memory where it fits, so the row
// is read from HBM once; the histograms are added over distributed shared memory and the first block decides.
//
// Numbers: a token's choice turns on sums of up to 10^5 nearly equal weights, next to borders 10^-5 apart, so weights are
// evaluated in 64 bits (relative error about 1e-14) and summed as 64-bit integers in units of 2^-shift -- exact, and the
// same in any order.  What bounds the kernel is that arithmetic (about 20 fp64 operations a logit) and the latency of
// its steps, not the read of the logits.
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
typedef unsigned long long u64;

constexpr int kThreads = 512;
constexpr int kBins = 2048;
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

// exp(x) for x <= 0 in 64 bits: x = n ln 2 + r, |r| <= ln 2 / 2, Taylor's series of exp(r) to the 11th power (the first
// term left out is below 7e-15), scaled by 2^n.  exp(0) is 1 exactly; 0 below -700.
__device__ __forceinline__ double exp64(double x)
{
    if (!(x > -700.0)) return 0.0;
    const double n = rint(x * 1.4426950408889634);
    double r = fma(n, -0.693147180559945286, x);         // ln 2 in two parts
    r = fma(n, -2.31904681384629956e-17, r);
    double p = 1.0 / 39916800.0;
    p = fma(p, r, 1.0 / 3628800.0);
    p = fma(p, r, 1.0 / 362880.0);
    p = fma(p, r, 1.0 / 40320.0);
    p = fma(p, r, 1.0 / 5040.0);
    p = fma(p, r, 1.0 / 720.0);
    p = fma(p, r, 1.0 / 120.0);
    p = fma(p, r, 1.0 / 24.0);
    p = fma(p, r, 1.0 / 6.0);
    p = fma(p, r, 0.5);
    p = fma(p, r, 1.0);
    p = fma(p, r, 1.0);
    return __hiloint2double(__double2hiint(p) + ((int)n << 20), __double2loint(p));
}

struct RowRule {
    double inv_t, cut;                  // entries with z < cut are out
    double scale;                       // 2^shift
    float top, inv_t32, bins_per;       // bin = (top - z) * inv_t32 * bins_per
};

__device__ __forceinline__ u64 mass_of(const RowRule &q, float z)
{
    // an infinite maximum: its equals weigh 1, the rest nothing; an infinite temperature: all finite logits weigh 1
    const double x = z == q.top ? 0.0 : ((double)z - (double)q.top) * q.inv_t;
    return (u64)__double2ull_rn(exp64(x) * q.scale);
}
__device__ __forceinline__ bool kept(const RowRule &q, float z) { return z > -INFINITY && (double)z >= q.cut; }   // false for NaN
__device__ __forceinline__ int bin_of(const RowRule &q, float z)
{
    const float t = z == q.top ? 0.f : (q.top - z) * q.inv_t32 * q.bins_per;      // not increasing in z; may be +inf, or NaN (0 * inf: bin 0)
    return t < (float)kBins ? (int)t : (t >= (float)kBins ? kBins - 1 : 0);
}


enum { kOpDone = 0, kOpCollect = 1, kOpDigits = 2 };
struct Command {                        // what the first block asks of its cluster
    int op;
    int lo, hi;                         // bins concerned
    int shift;                          // kOpDigits: histogram of (key >> shift) & 255
    u64 prefix, mask;                   // only entries with (key & mask) == prefix
};

struct alignas(16) Shared {
    u64 mass[kBins];                    // histogram; afterwards, in the first block, its running sums
    u64 list[kList];
    u64 digit_mass[256];
    u64 warp64[kThreads / 32];
    u64 best;                           // greatest key of the slice
    u64 found_mass, found_key;
    Command cmd;
    uint32_t count[kBins];
    uint32_t digit_count[256];
    uint32_t warp32[kThreads / 32];
    uint32_t fill;
    float low;                          // least logit above -inf of the slice
    uint32_t found_count;
    int found_at;
};

// Inclusive sums over the block in thread order.  All threads call it; the shared scratch is free again on return.
__device__ __forceinline__ void block_scan(Shared &s, uint32_t &c, u64 &m)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t oc = __shfl_up_sync(0xFFFFFFFFu, c, o);
        const u64 om = __shfl_up_sync(0xFFFFFFFFu, m, o);
        if (lane >= o) { c += oc; m += om; }
    }
    if (lane == 31) { s.warp32[warp] = c; s.warp64[warp] = m; }
    __syncthreads();
    uint32_t wc = lane < kThreads / 32 ? s.warp32[lane] : 0;
    u64 wm = lane < kThreads / 32 ? s.warp64[lane] : 0;
#pragma unroll
    for (int o = 1; o < kThreads / 32; o <<= 1) {
        const uint32_t oc = __shfl_up_sync(0xFFFFFFFFu, wc, o);
        const u64 om = __shfl_up_sync(0xFFFFFFFFu, wm, o);
        if (lane >= o) { wc += oc; wm += om; }
    }
    if (warp > 0) {
        c += __shfl_sync(0xFFFFFFFFu, wc, warp - 1);
        m += __shfl_sync(0xFFFFFFFFu, wm, warp - 1);
    }
    __syncthreads();
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

// Descending bitonic sort of s.list[0..n); the rest up to a power of two is padded with 0 (no key).
__device__ __forceinline__ void sort_list(Shared &s, uint32_t n)
{
    uint32_t size = 2;
    while (size < n) size <<= 1;
    for (uint32_t i = n + threadIdx.x; i < size; i += kThreads) s.list[i] = 0;
    __syncthreads();
    for (uint32_t k = 2; k <= size; k <<= 1)
        for (uint32_t j = k >> 1; j > 0; j >>= 1) {
            for (uint32_t t = threadIdx.x; t < size / 2; t += kThreads) {
                const uint32_t i = 2 * t - (t & (j - 1)), l = i + j;
                const u64 a = s.list[i], b = s.list[l];
                const bool descending = (i & k) == 0;
                if ((a < b) == descending) { s.list[i] = b; s.list[l] = a; }
            }
            __syncthreads();
        }
}

constexpr int kPerThread = kList / kThreads;       // list entries of a thread, consecutive
constexpr int kBinsPerThread = kBins / kThreads;

template <typename T>
__global__ void __launch_bounds__(kThreads, 2)
tfe_sample_kernel(const SampleParams p)
{
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

    // ---- this block's slice, its greatest key and its least logit
    const Cut cut = cut_row(row, p.V);
    const int32_t v0 = (int32_t)(cut.n_vec * part / p.blocks), v1 = (int32_t)(cut.n_vec * (part + 1) / p.blocks);
    const int32_t body0 = (int32_t)cut.head + v0 * E, body1 = (int32_t)cut.head + v1 * E;
    const int32_t e0 = leader ? 0 : body0, e1 = part == p.blocks - 1 ? p.V : body1;
    const bool resident = body1 - body0 + 2 * E <= p.slice_cap;
    u64 best = 0;
    float low = INFINITY;
    auto see = [&](float z, int32_t i) {
        if (z > -INFINITY) {            // false for NaN
            const u64 key = entry_key(z, i);
            best = key > best ? key : best;
            low = fminf(low, z);
        }
    };
    {
        const uint4 *body = reinterpret_cast<const uint4 *>(row + cut.head);
        uint4 *keep = reinterpret_cast<uint4 *>(slice + E);
        for (int32_t v = v0 + tid; v < v1; v += kThreads) {
            const uint4 raw = load_stream(body + v);
            if (resident) keep[v - v0] = raw;
            float f[E];
            Elem<T>::unpack(raw, f);
#pragma unroll
            for (int e = 0; e < E; ++e) see(f[e], (int32_t)cut.head + v * E + e);
        }
        for (int32_t i = e0 + tid; i < body0; i += kThreads) {
            if (resident) slice[E + i - body0] = row[i];
            see(Elem<T>::get(row + i), i);
        }
        for (int32_t i = body1 + tid; i < e1; i += kThreads) {
            if (resident) slice[E + i - body0] = row[i];
            see(Elem<T>::get(row + i), i);
        }
    }
    for (int i = tid; i < kBins; i += kThreads) { s.mass[i] = 0; s.count[i] = 0; }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const u64 other = __shfl_xor_sync(0xFFFFFFFFu, best, o);
        best = other > best ? other : best;
        low = fminf(low, __shfl_xor_sync(0xFFFFFFFFu, low, o));
    }
    if (lane == 0) { s.warp64[warp] = best; s.warp32[warp] = __float_as_uint(low); }
    __syncthreads();
    if (warp == 0) {
        best = lane < kThreads / 32 ? s.warp64[lane] : 0;
        low = lane < kThreads / 32 ? __uint_as_float(s.warp32[lane]) : INFINITY;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const u64 other = __shfl_xor_sync(0xFFFFFFFFu, best, o);
            best = other > best ? other : best;
            low = fminf(low, __shfl_xor_sync(0xFFFFFFFFu, low, o));
        }
        if (lane == 0) { s.best = best; s.low = low; }
    }
    cluster.sync();
    best = 0;
    low = INFINITY;
    for (int b = 0; b < p.blocks; ++b) {
        const u64 other = *cluster.map_shared_rank(&s.best, b);
        best = other > best ? other : best;
        low = fminf(low, *cluster.map_shared_rank(&s.low, b));
    }

    // ---- the row's rule
    const float T_ = p.temperature ? p.temperature[r] : 1.f;
    const int32_t k = p.top_k ? p.top_k[r] : 0;
    const float top_p = p.top_p ? p.top_p[r] : 1.f, min_p = p.min_p ? p.min_p[r] : 0.f;
    const float u = fminf(fmaxf(p.u[r], 0.f), 1.f - 0x1p-24f);          // NaN: 0
    if (best == 0 || !(T_ > 0.f)) {                                     // nothing to draw from, or greedy: the same in every block
        if (leader && tid == 0) {
            p.tokens[r] = best == 0 ? -1 : key_index(best);
            if (p.prob) p.prob[r] = best == 0 ? 0.f : 1.f;
        }
        cluster.sync();
        return;
    }
    RowRule q;
    q.top = key_logit(best);
    q.inv_t = 1.0 / (double)T_;
    q.inv_t32 = 1.f / T_;
    q.cut = !(min_p > 0.f) ? -INFINITY : min_p >= 1.f ? (double)q.top : __dadd_rn((double)q.top, __dmul_rn((double)T_, log((double)min_p)));
    if (isnan(q.cut)) q.cut = (double)q.top;                            // infinite maximum and infinite temperature
    q.scale = ldexp(1.0, p.shift);
    q.bins_per = (float)kBins / fminf(kRange, (q.top - low) * q.inv_t32);     // 0 / 0 and the like: fminf drops NaN
    const T *src = resident ? slice + E - body0 : row;

    // ---- counts and masses by bin
    for (int32_t i = e0 + tid; i < e1; i += kThreads) {
        const float z = Elem<T>::get(src + i);
        if (kept(q, z)) {
            const int b = bin_of(q, z);
            atomicAdd(&s.count[b], 1u);
            const u64 m = mass_of(q, z);
            if (m) atomicAdd(&s.mass[b], m);
        }
    }
    cluster.sync();
    if (p.blocks > 1) {
        const int share = kBins / p.blocks;
        for (int i = tid; i < share; i += kThreads) {
            const int b = part * share + i;
            uint32_t c = 0;
            u64 m = 0;
            for (int o = 0; o < p.blocks; ++o) { c += cluster.map_shared_rank(s.count, o)[b]; m += cluster.map_shared_rank(s.mass, o)[b]; }
            s.count[b] = c; s.mass[b] = m;
        }
        cluster.sync();
        if (leader)
            for (int b = share + tid; b < kBins; b += kThreads) {
                s.count[b] = cluster.map_shared_rank(s.count, b / share)[b];
                s.mass[b] = cluster.map_shared_rank(s.mass, b / share)[b];
            }
        __syncthreads();
    }

    // ---- the searches: the first block decides, every block looks through its slice
    enum { kTopK = 0, kTopP = 1, kDraw = 2, kAll = 3 };
    uint32_t total_n = 0, base_n = 0, list_n = 0;
    u64 total_m = 0, base_m = 0, limit = 0;             // limit: mass of the prefix that is still in
    int stage = kDraw, list_lo = 0, list_hi = -1;       // bins that the sorted list holds whole
    bool k_on = false, p_on = false;
    u64 run_m[kPerThread];                              // running mass of this thread's list entries

    auto goal_of = [&](int st) {
        Goal g;
        g.kind = st == kTopK ? 0 : st == kTopP ? 1 : 2;
        g.count = (uint32_t)k;
        g.mass = st == kTopP ? (double)fmaxf(top_p, 0.f) * (double)limit : (double)u * (double)limit;
        return g;
    };
    // the first bin whose running sums meet the goal (there is one); sets base_n / base_m to the sums before it
    auto find_bin = [&](const Goal &g) {
#pragma unroll
        for (int j = 0; j < kBinsPerThread; ++j) {
            const int b = tid * kBinsPerThread + j;
            const uint32_t c0 = b ? s.count[b - 1] : 0;
            const u64 m0 = b ? s.mass[b - 1] : 0;
            if (g.met(s.count[b], s.mass[b]) && (b == 0 || !g.met(c0, m0))) { s.found_at = b; s.found_count = c0; s.found_mass = m0; }
        }
        __syncthreads();
        const int b = min(max(s.found_at, 0), kBins - 1);
        base_n = s.found_count; base_m = s.found_mass;
        __syncthreads();
        return b;
    };
    auto command = [&](int op, int lo, int hi, int shift, u64 prefix, u64 mask) {
        if (tid == 0) { s.cmd.op = op; s.cmd.lo = lo; s.cmd.hi = hi; s.cmd.shift = shift; s.cmd.prefix = prefix; s.cmd.mask = mask; }
    };
    // the entry of the sorted list at which the goal is met: running mass and key
    auto find_entry = [&](const Goal &g, u64 &mass, u64 &key) {
#pragma unroll
        for (int j = 0; j < kPerThread; ++j) {
            const uint32_t i = (uint32_t)(tid * kPerThread + j);
            if (i < list_n) {
                const u64 own = mass_of(q, key_logit(s.list[i]));
                if (g.met(base_n + i + 1, base_m + run_m[j]) && (i == 0 || !g.met(base_n + i, base_m + run_m[j] - own))) {
                    s.found_mass = base_m + run_m[j];
                    s.found_key = s.list[i];
                }
            }
        }
        __syncthreads();
        mass = s.found_mass; key = s.found_key;
        __syncthreads();
    };
    // starts the search of `stage`, and goes on through the searches that the list at hand answers
    auto advance = [&](bool first) {
        for (;;) {
            if (!first) {
                u64 mass, key;
                find_entry(goal_of(stage), mass, key);
                if (stage == kDraw) {
                    if (tid == 0) {
                        p.tokens[r] = key_index(key);
                        const float z = key_logit(key);
                        const double x = z == q.top ? 0.0 : ((double)z - (double)q.top) * q.inv_t;
                        if (p.prob) p.prob[r] = (float)(exp64(x) * q.scale / (double)limit);
                    }
                    command(kOpDone, 0, -1, 0, 0, 0);
                    return;
                }
                limit = mass;
                stage = stage == kTopK && p_on ? kTopP : kDraw;
            }
            const int b = find_bin(goal_of(stage));
            if (list_lo <= b && b <= list_hi) {
                base_n = list_lo ? s.count[list_lo - 1] : 0;
                base_m = list_lo ? s.mass[list_lo - 1] : 0;
                first = false;
                continue;
            }
            const uint32_t inside = s.count[b] - base_n;
            if (inside <= (uint32_t)kList) {
                list_lo = list_hi = b;
                command(kOpCollect, b, b, 0, 0, 0);
            } else {
                list_lo = 0; list_hi = -1;
                command(kOpDigits, b, b, 56, 0, 0);
            }
            return;
        }
    };

    if (leader) {
        // running sums over the bins
        uint32_t c[kBinsPerThread], c_sum = 0;
        u64 m[kBinsPerThread], m_sum = 0;
#pragma unroll
        for (int j = 0; j < kBinsPerThread; ++j) {
            c_sum += s.count[tid * kBinsPerThread + j]; c[j] = c_sum;
            m_sum += s.mass[tid * kBinsPerThread + j]; m[j] = m_sum;
        }
        uint32_t c_run = c_sum;
        u64 m_run = m_sum;
        block_scan(s, c_run, m_run);
#pragma unroll
        for (int j = 0; j < kBinsPerThread; ++j) {
            s.count[tid * kBinsPerThread + j] = c_run - c_sum + c[j];
            s.mass[tid * kBinsPerThread + j] = m_run - m_sum + m[j];
        }
        __syncthreads();
        total_n = s.count[kBins - 1];
        total_m = s.mass[kBins - 1];
        limit = total_m;
        k_on = k > 0 && (uint32_t)k < total_n;
        p_on = top_p < 1.f;
        stage = k_on ? kTopK : p_on ? kTopP : kDraw;
        // a short prefix is collected whole: one list answers every search
        bool whole = false;
        if (stage != kDraw) {
            const int b = find_bin(goal_of(stage));
            if (s.count[b] <= (uint32_t)kList) {
                whole = true;
                base_n = 0; base_m = 0;
                list_lo = 0; list_hi = b;
                command(kOpCollect, 0, b, 0, 0, 0);
            }
        }
        if (!whole) advance(true);
    }

    for (;;) {
        cluster.sync();
        const Command cmd = *cluster.map_shared_rank(&s.cmd, 0);
        if (cmd.op == kOpDone) break;
        if (tid == 0) s.fill = 0;
        if (cmd.op == kOpDigits && tid < 256) { s.digit_count[tid] = 0; s.digit_mass[tid] = 0; }
        __syncthreads();
        for (int32_t i = e0 + tid; i < e1; i += kThreads) {
            const float z = Elem<T>::get(src + i);
            if (!kept(q, z)) continue;
            const int b = bin_of(q, z);
            if (b < cmd.lo || b > cmd.hi) continue;
            const u64 key = entry_key(z, i);
            if ((key & cmd.mask) != cmd.prefix) continue;
            if (cmd.op == kOpCollect) {
                const uint32_t at = atomicAdd(&s.fill, 1u);
                if (at < (uint32_t)kList) s.list[at] = key;
            } else {
                const int d = (int)((key >> cmd.shift) & 255u);
                atomicAdd(&s.digit_count[d], 1u);
                atomicAdd(&s.digit_mass[d], mass_of(q, z));
            }
        }
        cluster.sync();
        if (!leader) continue;
        if (cmd.op == kOpCollect) {
            list_n = min(s.fill, (uint32_t)kList);
            for (int b = 1; b < p.blocks; ++b) {
                const uint32_t n = *cluster.map_shared_rank(&s.fill, b);
                const u64 *theirs = cluster.map_shared_rank(s.list, b);
                for (uint32_t i = tid; i < n; i += kThreads)
                    if (list_n + i < (uint32_t)kList) s.list[list_n + i] = theirs[i];
                list_n = min(list_n + n, (uint32_t)kList);
            }
            __syncthreads();
            sort_list(s, list_n);
            uint32_t none = 0;
            u64 sum = 0;
#pragma unroll
            for (int j = 0; j < kPerThread; ++j) {
                const uint32_t i = (uint32_t)(tid * kPerThread + j);
                if (i < list_n) sum += mass_of(q, key_logit(s.list[i]));
                run_m[j] = sum;
            }
            u64 run = sum;
            block_scan(s, none, run);
#pragma unroll
            for (int j = 0; j < kPerThread; ++j) run_m[j] += run - sum;
            advance(false);
        } else {
            // digits in descending order: thread t holds digit 255 - t
            const int d = 255 - tid;
            uint32_t c = 0;
            u64 m = 0;
            if (tid < 256)
                for (int b = 0; b < p.blocks; ++b) { c += cluster.map_shared_rank(s.digit_count, b)[d]; m += cluster.map_shared_rank(s.digit_mass, b)[d]; }
            uint32_t c_run = c;
            u64 m_run = m;
            block_scan(s, c_run, m_run);
            const Goal g = goal_of(stage);
            if (tid < 256 && c && g.met(base_n + c_run, base_m + m_run) && !(c_run > c && g.met(base_n + c_run - c, base_m + m_run - m))) {
                s.found_at = d; s.found_count = c; s.found_key = (u64)(c_run - c); s.found_mass = m_run - m;
            }
            __syncthreads();
            const u64 prefix = cmd.prefix | ((u64)s.found_at << cmd.shift), mask = cmd.mask | (255ull << cmd.shift);
            const uint32_t inside = s.found_count;
            base_n += (uint32_t)s.found_key;
            base_m += s.found_mass;
            __syncthreads();
            if (inside <= (uint32_t)kList || cmd.shift == 0) command(kOpCollect, cmd.lo, cmd.hi, 0, prefix, mask);
            else command(kOpDigits, cmd.lo, cmd.hi, cmd.shift - 8, prefix, mask);
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
    // up to 8 blocks a row, none with less than 2,048 logits
    p.blocks = 1;
    while (p.blocks < 8 && V / (2 * p.blocks) >= 2048) p.blocks *= 2;
    // masses sum to less than 2^63
    int bits = 0;
    while ((1ll << bits) < V) ++bits;
    p.shift = std::min(46, 62 - bits);
    // the slice and the parts of a vector at both its ends; two blocks per SM where that is possible
    const int per_vec = 16 / es;
    const int64_t want = ((int64_t)V / per_vec / p.blocks + 1) * per_vec + 2 * per_vec;
    const int64_t room = (226 * 1024 - (int64_t)sizeof(Shared)) / es;
    p.slice_cap = want <= room ? (int32_t)want : 0;
    const size_t smem = sizeof(Shared) + (size_t)p.slice_cap * es;
    auto kernel = dtype == TFE_DTYPE_BF16 ? tfe_sample_kernel<__nv_bfloat16> : tfe_sample_kernel<float>;
    if (tfe_status st = tfe_note_cuda(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024), "sampling attribute")) return st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)p.blocks;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)B * (unsigned)p.blocks); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = smem;
    cfg.stream = static_cast<cudaStream_t>(stream_);
    cfg.attrs = attr; cfg.numAttrs = 1;
    return tfe_note_cuda(cudaLaunchKernelEx(&cfg, kernel, p), "sampling launch");
}

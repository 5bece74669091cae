// Softmax cross entropy of hidden states against a vocabulary projection, loss and gradients, without keeping the logits: the
// loss that trains an early-exit projection (paper Sec. 4.4) on the tokens themselves.
//
// Per row n with target t:   z_v = W_v . h_n      lse = ln sum_v exp z_v      loss = lse - z_t
//     G_nv = g_n (exp(z_v - lse) - [v = t])       grad H = G W                grad W = G^T H
//
//   tfe_xent_compact_kernel   lists the rows that have a target (and a gradient) and copies their hidden states together: the
//                             products below run over those rows only, and a row that has none takes part in no sum.  For the
//                             gradients the rows are put in the order of their targets.
//   tfe_xent_gemm_kernel      one persistent, warp-specialised tcgen05 kernel with three epilogues:
//       kLse    z tile by tile, each kept only as its row maxima and row sums of exponentials, the rows' targets left out;
//       kProb   z of a piece of the vocabulary once more, turned into that piece of G (bf16, in the workspace);
//       kGrads  both products of the piece with G: grad W is complete with its piece, grad H adds up over the pieces in fp32.
//   tfe_xent_few_kernel       the loss of up to 64 rows.
//   tfe_xent_loss_kernel      joins a row's partial maxima and sums with its target's logit.
//   tfe_xent_rest_kernel      G at the targets, and what its rounding took from it.
//   tfe_xent_rows_kernel      joins grad H's sums, rounds them and puts them back to their rows; completes grad W's rows of the targets.
//
// All products are 2 N V d operations; the loss makes one, the gradients three (z again and the two with G).  For 2,048 x 151,936 x 1,024 the
// tensor cores bound all of it: 490 us the loss (1.30 PFLOP/s), 518 us z again, 994 us both products with G with the card idle before; back
// to back the power limit does, at 559 to 582 us for the loss (the library's product of this size beside it: 565 to 584).  Up to 256 rows
// memory does: the weights are read three times and their gradient is written once.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>

#include "../../include/tfe.h"
#include "tfe_internal.h"
#include "tfe_rows.cuh"
#include "tfe_tc.cuh"

namespace {

using bf16 = __nv_bfloat16;

constexpr int kCtas = 2;                        // CTAs that share a tile: a cluster
constexpr int kRowsA = 128;                     // rows of A per CTA (MMA M per CTA)
constexpr int kM = kRowsA * kCtas;              // rows of a tile
constexpr int kN = 256;                         // columns of a tile at most (MMA N)
constexpr int kStepK = 64;                      // k of a stage: 128 bytes, one swizzle row
constexpr uint32_t kBytesA = kRowsA * kStepK * 2, kBytesB = kN / kCtas * kStepK * 2, kStageBytes = kBytesA + kBytesB;
constexpr int kStages = 6;
constexpr int kBuffers = 2;                     // accumulators of kN columns: all of tensor memory
constexpr int kEpilogueWarps = 8;               // two per lane quarter of tensor memory, half of the tile's columns each
constexpr int kThreads = 32 * (4 + kEpilogueWarps);
constexpr uint32_t kRoom = 32 * 128;            // bytes of an epilogue warp's outgoing piece: 32 rows of 64 bf16
constexpr size_t kSmem = 1024 + (size_t)kStages * kStageBytes + kEpilogueWarps * kRoom;
constexpr float kLog2e = 1.4426950408889634f;
// The tensor cores cut what they add to a sum in fp32, always towards zero, so a long sum comes out too small: a loss over 1,024 k was off by
// 6e-7 that way.  A sum of the loss therefore takes at most this many steps, and the epilogue adds those up: 3e-7, whatever d.  (With 4
// steps 1.4e-7 and 624 us instead of 561 for 2,048 x 151,936 x 1,024; the few-row kernel has time for a sum per stage.)
constexpr int kSumSteps = 8;
// Registers per thread in the loss's kernel: the first four warps give most of theirs to the epilogue's, which hold 128 sums each.  The
// sum, 128 x 40 + 256 x 216, must not exceed what the block is launched with; the host checks that before the launch.
constexpr int kFewRegs = 40, kManyRegs = 216;

constexpr uint32_t kTimeoutLoader = 1u, kTimeoutMma = 2u, kTimeoutEpilogue = 4u;
__device__ uint32_t g_xent_status;
// For tests: all waits run out at once, or those of who issues the MMAs at the end of its first sum, with copies and MMAs under way.
constexpr uint32_t kAtOnce = 1, kUnderWay = 2;
std::atomic<uint32_t> g_xent_give_up{0};

__global__ void tfe_xent_status_kernel(uint32_t told) { atomicAnd(&g_xent_status, ~told); }

enum Op { kLse, kProb, kGrads };
struct GemmParams {
    int32_t N, V, d, n_pad;
    int32_t tn;                                 // columns of a tile
    int32_t per_unit, n_tiles;                  // kLse: tiles of a unit, all column tiles
    int32_t v0, width;                          // kProb, kGrads: the piece, [v0, v0 + width)
    int32_t splits, first;                      // kGrads: parts of the sums over a piece for grad H; the first piece
    int32_t m_room;                             // row tiles that there is room for
    int32_t want_h, want_w;
    uint32_t give_up;
    const int32_t *n_live;                      // rows taken part in (null: N)
    const int32_t *target;
    const float *lse, *coef;
    float *rest;                                // kProb: G at each row's target as the products have it
    float *part_p; int64_t ld_p;                // kProb: [2 * column tiles of a piece][ld_p] sums of probabilities, the targets' left out, over all pieces so far
    uint32_t *first_row;                        // [V]: the first row whose target is this id, kNone where there is none
    float *sum_w; int32_t by_id;                // kGrads: rows of grad W before they are rounded, d apart: of the ids that are targets, by their first row, or of all ids
    float2 *part; int64_t ld_part;              // kLse: [2 * units per row][ld_part] maxima and sums
    float *sum_h;                               // kGrads: [splits][m_room][column tiles][tn / 4][kM][4]
    uint32_t *failed;                           // set if a wait ran out
    uint32_t *ticket;                           // kGrads: units handed out so far
};

// ------------------------------------------------------------------ rows that take part

struct CompactParams {
    int32_t N, V, d, rows_per_block;
    const bf16 *h; int64_t ld;
    const int32_t *target;
    const float *lse, *grad;                    // null: the loss
    bf16 *h_out;
    int32_t *pos, *target_out, *n_live;
    float *lse_out, *coef_out;
    uint32_t *failed;                           // cleared here, with the units' counters behind it
    int32_t counters;
    uint32_t *first_row;                        // set to kNone here
    int32_t *group_at;                          // where each kGroup rows begin among those that take part, and their end
};
constexpr uint32_t kNone = 0xFFFFFFFFu;
// Rows are ordered by their targets within this many: every row is compared with all others of its group, so the work is linear in
// the rows.  131,072 rows x 256: 300 us (of 10.8 ms for both gradients against 32,003 ids); in groups of 32,768 830 us, and 50 us less
// where an id's runs are put together.
constexpr int32_t kGroup = 8192;

// Every block counts the rows before its own by itself, so one launch does: 11 us for 4,096 rows of 1,024 of which 30 % are left out, 16 us in the
// order of their targets, 5 us for 256.
constexpr int kCompactThreads = 256, kTile = 4 * kCompactThreads;

template <bool kOrdered>
__global__ void __launch_bounds__(kCompactThreads)
tfe_xent_compact_kernel(const CompactParams p)
{
    __shared__ int32_t s_before[kCompactThreads / 32], s_all[kCompactThreads / 32];
    __shared__ int32_t s_from[kCompactThreads], s_to[kCompactThreads];
    __shared__ __align__(16) int32_t s_key[kOrdered ? kTile : 4];
    tfe_wait_for_stream();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int64_t r0 = (int64_t)blockIdx.x * p.rows_per_block, r1 = min((int64_t)p.N, r0 + p.rows_per_block);
    const int64_t from = kOrdered ? r0 / kGroup * kGroup : r0;      // what lies before it comes before all of this block's
    constexpr int32_t kNever = 1 << 30;
    auto key = [&](int64_t r) {                 // a row's target, or more than any (no branches: loads in a loop stay together)
        const int64_t at = min(r, (int64_t)p.N - 1);
        const int32_t t = p.target[at];
        const float g = kOrdered ? p.grad[at] : 1.f;
        const bool ok = (r < p.N) & ((uint32_t)t < (uint32_t)p.V) & !(g == 0.f);
        return ok ? t : kNever;
    };
    // how many before this block's rows, and in all (every block counts for itself: the targets are a few KB in L2)
    int32_t before = 0, all = 0;
#pragma unroll 8
    for (int64_t r = tid; r < p.N; r += kCompactThreads) {
        const int32_t one = key(r) != kNever;
        all += one;
        before += r < from ? one : 0;
    }
    before = __reduce_add_sync(0xFFFFFFFFu, before);
    all = __reduce_add_sync(0xFFFFFFFFu, all);
    if (lane == 0) { s_before[warp] = before; s_all[warp] = all; }
    __syncthreads();
    before = all = 0;
    for (int w = 0; w < kCompactThreads / 32; ++w) { before += s_before[w]; all += s_all[w]; }
    if (blockIdx.x == 0 && tid == 0) *p.n_live = all;
    if (blockIdx.x == 0)
        for (int32_t i = tid; i <= p.counters; i += kCompactThreads) p.failed[i] = 0;
    if (kOrdered && r0 == from && r0 < p.N && tid == 0) p.group_at[r0 / kGroup] = before;
    if (kOrdered && blockIdx.x == 0 && tid == 0) p.group_at[(p.N + kGroup - 1) / kGroup] = all;
    const int vecs = p.d / 8;
    const int32_t batch = kOrdered ? min(p.rows_per_block, kCompactThreads) : kCompactThreads;      // rows at a time
    for (int64_t base = r0; base < r1; base += batch) {
        int32_t total = 0;
        __syncthreads();
        if constexpr (kOrdered) {
            // a row's place is the number of those of its group that come before it: by their targets, and as they were where those are the same
            const int32_t parts = kCompactThreads / batch, mine = tid & (batch - 1), part = tid / batch;
            const int32_t t = key(base + mine);
            if (tid < batch) s_to[tid] = before;
            int32_t count = 0;
            const int64_t end = min((int64_t)p.N, from + kGroup);
            int32_t next[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) next[i] = key(from + tid + i * kCompactThreads);
            for (int64_t at = from; at < end; at += kTile) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < 4; ++i) s_key[tid + i * kCompactThreads] = next[i];
                __syncthreads();
#pragma unroll
                for (int i = 0; i < 4; ++i) next[i] = key(at + kTile + tid + i * kCompactThreads);
                if (at + kTile <= base || at >= base + batch) {
                    const int32_t below = t + (at < base ? 1 : 0);          // (if t is kNever, its place is not used)
#pragma unroll 8
                    for (int32_t i = part; i < kTile / 4; i += parts) {
                        const int4 x = reinterpret_cast<const int4 *>(s_key)[i];
                        count += (x.x < below) + (x.y < below) + (x.z < below) + (x.w < below);
                    }
                } else {
                    const int32_t own = (int32_t)(base + mine - at);
#pragma unroll 8
                    for (int32_t i = part; i < kTile / 4; i += parts) {
                        const int4 x = reinterpret_cast<const int4 *>(s_key)[i];
                        count += (x.x < t + (4 * i < own)) + (x.y < t + (4 * i + 1 < own)) + (x.z < t + (4 * i + 2 < own)) + (x.w < t + (4 * i + 3 < own));
                    }
                }
            }
            atomicAdd(&s_to[mine], count);
            __syncthreads();
            if (tid < batch) {
                const int64_t r = base + tid;
                const int32_t at = t != kNever ? s_to[tid] : -1;
                s_to[tid] = at;
                if (r < r1) p.pos[r] = at;
                if (at >= 0) { p.target_out[at] = t; p.lse_out[at] = p.lse[r]; p.coef_out[at] = p.grad[r]; }
            }
            total = batch;
        } else {
            const int64_t r = base + tid;
            const bool one = r < r1 && key(r) != kNever;
            const uint32_t vote = __ballot_sync(0xFFFFFFFFu, one);
            if (lane == 0) s_before[warp] = __popc(vote);
            __syncthreads();
            int32_t at = before;
            for (int w = 0; w < kCompactThreads / 32; ++w) { at += w < warp ? s_before[w] : 0; total += s_before[w]; }
            at += __popc(vote & ((1u << lane) - 1u));
            if (r < r1) p.pos[r] = one ? at : -1;
            if (one) {
                s_from[at - before] = tid;
                p.target_out[at] = p.target[r];
            }
        }
        __syncthreads();
#pragma unroll 4
        for (int32_t i = tid; i < total * vecs; i += kCompactThreads) {        // whose row it is does not matter: all loads at once
            const int32_t k = i / vecs, v = i - k * vecs, row = kOrdered ? k : s_from[k], at = kOrdered ? s_to[k] : before + k;
            if (at >= 0) reinterpret_cast<uint4 *>(p.h_out + (int64_t)at * p.d)[v] = __ldg(reinterpret_cast<const uint4 *>(p.h + (base + row) * p.ld) + v);
        }
        if (!kOrdered) before += total;
    }
    // zeros up to the end of the last tile: the sums over rows run to there
    const int64_t end = max((int64_t)(all + kM - 1) / kM, (int64_t)1) * kM;
    const int64_t n_zero = (end - all) * vecs;
    uint4 *dst = reinterpret_cast<uint4 *>(p.h_out + (int64_t)all * p.d);
    for (int64_t i = (int64_t)blockIdx.x * kCompactThreads + tid; i < n_zero; i += (int64_t)gridDim.x * kCompactThreads) dst[i] = make_uint4(0, 0, 0, 0);
    if (blockIdx.x == 0)
        for (int64_t i = all + tid; i < end; i += kCompactThreads) p.target_out[i] = -1;
    if constexpr (kOrdered)                     // (there is room up to the next multiple of 4)
        for (int64_t i = (int64_t)blockIdx.x * kCompactThreads + tid; i < (p.V + 3) / 4; i += (int64_t)gridDim.x * kCompactThreads)
            reinterpret_cast<uint4 *>(p.first_row)[i] = make_uint4(kNone, kNone, kNone, kNone);
}

// ------------------------------------------------------------------ the products

// Shared-memory operand whose rows are 64 consecutive bf16 along M or N for one k (written by TMA with the 128-byte swizzle): rows
// 128 bytes apart, groups of 8 k 1,024 bytes apart (stride offset), the next 64 along M or N 64 rows further (leading offset).
__device__ __forceinline__ uint64_t umma_desc_mn_sw128(uint32_t smem_addr)
{
    uint64_t d = (uint64_t)((smem_addr & 0x3FFFFu) >> 4);
    d |= (uint64_t)(kStepK * 128 >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
// kind::f16: D fp32 ([4,6) = 1), A and B bf16 ([7,10) = [10,13) = 1), bit 15 / 16: A / B run along M / N in memory
__host__ __device__ constexpr uint32_t umma_idesc(uint32_t M, uint32_t N, bool a_mn, bool b_mn)
{
    return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((N >> 3) << 17) | ((M >> 4) << 24);
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap *map, uint32_t from, int32_t x, int32_t y)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(reinterpret_cast<uint64_t>(map)), "r"(from),
                 "r"(x), "r"(y)
                 : "memory");
}

// What a unit of work multiplies.  A's tile is kM rows (or columns of G) from a_at, B's tn from b_at, the sum runs over steps of 64 from k_at.
struct Unit {
    int32_t a_at, b_at, k_at, steps, tiles;
    bool grad_h;                                // kGrads: G W, else G^T H
    int32_t index;                              // kLse: column unit; kGrads: place of grad H's sum
};

template <int kOp>
struct Units {
    int32_t m_tiles, n_live, cols;              // row tiles, rows, column tiles of d (kGrads)
    int64_t n_h, n_w, n;                        // units of grad H, of grad W, all
    int32_t steps_h, steps_w;

    __device__ __forceinline__ explicit Units(const GemmParams &p)
    {
        n_live = p.n_live ? *p.n_live : p.N;
        m_tiles = max(1, (n_live + kM - 1) / kM);
        cols = (p.d + p.tn - 1) / p.tn;
        n_h = n_w = 0; steps_h = steps_w = 0;
        if constexpr (kOp == kLse) {
            n = n_live ? (int64_t)m_tiles * ((p.n_tiles + p.per_unit - 1) / p.per_unit) : 0;
        } else if constexpr (kOp == kProb) {
            n = (int64_t)m_tiles * ((p.width + p.tn - 1) / p.tn);
        } else {
            const int32_t all = (p.width + kStepK - 1) / kStepK;
            steps_h = (all + p.splits - 1) / p.splits;
            steps_w = max(1, (n_live + kStepK - 1) / kStepK);
            n_h = p.want_h ? (int64_t)m_tiles * cols * p.splits : 0;
            n_w = p.want_w ? (int64_t)((p.width + kM - 1) / kM) * cols : 0;
            n = n_h + n_w;
        }
    }
    __device__ __forceinline__ Unit at(const GemmParams &p, int64_t u) const
    {
        Unit w{};
        w.tiles = 1;
        if constexpr (kOp != kGrads) {          // neighbours, which run at about the same time, share the column tile
            const int32_t mt = (int32_t)(u % m_tiles), nt = (int32_t)(u / m_tiles);
            w.a_at = mt * kM;
            w.steps = (p.d + kStepK - 1) / kStepK;
            if constexpr (kOp == kLse) {
                w.b_at = nt * p.per_unit * p.tn;
                w.tiles = min(p.per_unit, p.n_tiles - nt * p.per_unit);
                w.index = nt;
            } else {
                w.b_at = nt * p.tn;             // within the piece
            }
        } else {
            const bool h_first = steps_h >= steps_w;        // the longer units first: the shares come out more even
            w.grad_h = h_first ? u < n_h : u >= n_w;
            if (w.grad_h) {                     // neighbours share the rows of W, and of G
                const int32_t i = (int32_t)(h_first ? u : u - n_w), ct = i % cols, mt = i / cols % m_tiles, s = i / cols / m_tiles;
                const int32_t all = (p.width + kStepK - 1) / kStepK;
                w.a_at = mt * kM;
                w.b_at = ct * p.tn;
                w.k_at = s * steps_h * kStepK;
                w.steps = max(0, min(steps_h, all - s * steps_h));
                w.index = (s * p.m_room + mt) * cols + ct;
            } else {
                const int32_t i = (int32_t)(h_first ? u - n_h : u);         // neighbours share the columns of G
                w.a_at = i / cols * kM;         // within the piece
                w.b_at = i % cols * p.tn;
                w.steps = steps_w;
            }
        }
        return w;
    }
};

// Instructions of a pair of CTAs: the first issues the MMAs, each holds its rows of A and of the sums, and half of B.
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t in_first(uint32_t smem_addr)        // the same place in the first CTA's shared memory
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(smem_addr));
    return r;
}
__device__ __forceinline__ uint32_t in_second(uint32_t smem_addr)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 1;" : "=r"(r) : "r"(smem_addr));
    return r;
}
__device__ __forceinline__ void store_cluster(uint32_t cluster_addr, uint32_t x)
{
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_addr), "r"(x) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait_cluster(uint32_t bar, uint32_t parity)      // what the other CTA wrote before it arrived is seen
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool mbar_wait_cluster(uint32_t bar, uint32_t parity, volatile uint32_t *abort_flag)         // bounded, as mbar_wait
{
    for (uint32_t i = 0; i < TC_WAIT_LIMIT; ++i) {
        if (mbar_try_wait_cluster(bar, parity)) return true;
        if ((i & 1023u) == 1023u && *abort_flag) return false;
    }
    return false;
}
__device__ __forceinline__ void arrive_cluster(uint32_t bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void pair_load_2d(uint32_t dst, const CUtensorMap *map, uint32_t bar, int32_t x, int32_t y, uint64_t hint)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
        " [%0], [%1, {%3, %4}], [%2], %5;"
        :
        : "r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y), "l"(hint)
        : "memory");
}
__device__ __forceinline__ void pair_mma(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        :
        : "r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// One arrival at this place in both CTAs when every MMA issued so far by this thread has completed.
__device__ __forceinline__ void pair_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void pair_tmem_alloc(uint32_t dst_smem, uint32_t cols)
{
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void pair_tmem_dealloc(uint32_t taddr, uint32_t cols)
{
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(cols) : "memory");
}

// What rounding G to bf16 takes away weighs most at a row's target, where G is largest and its error is one factor for a whole row of
// grad W; and with one coefficient for all rows, a mean, it is nearly the same factor in every row of an id.  That difference is kept in
// fp32 (rest), and the sums over it are added to the products before those are rounded: grad H's where its parts are joined, grad W's in the
// same kernel, for which the rows of the ids that are targets are kept in fp32 (sum_w).
// G at the target, g (p - 1), is minus the sum of the row's other probabilities: from p it would be off by the error of z_t and of lse, which for
// a logit of 28 over 1,024 k is 4e-5, and so wrong in every digit where 1 - p is less.  That sum is known after the last piece; the products have
// what z_t gives in its place, or nothing where p is near 1, and the difference is part of the rest.
constexpr float kSure = 0x1p-8f;                // 1 - p below which the products have nothing

// The gradients' units, of two lengths, go to the pairs as they come free, in an order in which those under way together read the same
// operands: 2,048 x 50,688 x 1,024 take 321 us, with equal shares that each pair works off by itself 450 us.  The order of every sum is
// fixed by the unit, not by who computes it.  The other units are all alike, and short ones of the gradients' cost less than the asking:
// there every pair takes each pairs-th (the loss of 2,048 x 151,936 x 1,024: 561 us against 590; gradients of 256 rows, 4 steps a unit
// of grad W: 201 against 221).
constexpr int32_t kShort = 16;                  // steps of a unit of grad W
constexpr int kTickets = 4;                     // units that are known ahead (16: 371 us for the piece above, since neighbours then go to one pair)
constexpr int kListeners = kCtas * (2 + kEpilogueWarps) + 1;        // loaders, epilogue warps, and the one that issues the MMAs

struct Maps { CUtensorMap a, b, a_w, b_w, out; };           // kLse, kProb: H, W, -, -, G;  kGrads: G by rows, W, G by columns, H, grad W

template <int kOp>
__global__ void __launch_bounds__(kThreads, 1)
tfe_xent_gemm_kernel(const __grid_constant__ Maps maps, const GemmParams p)
{
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t s_full[kStages], s_empty[kStages], s_acc_full[kBuffers], s_acc_empty[kBuffers], s_drain;
    __shared__ __align__(8) uint64_t s_told[kTickets], s_heard[kTickets];
    __shared__ volatile uint32_t s_ticket[kTickets];
    __shared__ uint32_t s_tmem_base;
    __shared__ volatile uint32_t s_abort, s_issued[kCtas][2];       // alike in both CTAs at the end: whether a wait ran out, steps that each loader has issued

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    if (threadIdx.x == 0) {
        for (int t = 0; t < kTickets; ++t) { mbar_init(smem_u32(&s_told[t]), 1); mbar_init(smem_u32(&s_heard[t]), kListeners); }
        for (int s = 0; s < kStages; ++s) { mbar_init(smem_u32(&s_full[s]), 2); mbar_init(smem_u32(&s_empty[s]), 1); }
        for (int a = 0; a < kBuffers; ++a) { mbar_init(smem_u32(&s_acc_full[a]), 1); mbar_init(smem_u32(&s_acc_empty[a]), kCtas * kEpilogueWarps); }
        mbar_init(smem_u32(&s_drain), 1);
        s_abort = 0;
        for (int c = 0; c < kCtas; ++c) s_issued[c][0] = s_issued[c][1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    const uint32_t rank = cluster_rank();
    const int64_t pair = blockIdx.x / kCtas, pairs = gridDim.x / kCtas;
    if (warp == 1) pair_tmem_alloc(smem_u32(&s_tmem_base), kBuffers * kN);
    tc_fence_before();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem_base = s_tmem_base;
    tfe_wait_for_stream();
    const Units<kOp> units(p);
    auto in_both = [&](volatile uint32_t *at, uint32_t x) {
        const uint32_t here = smem_u32(const_cast<uint32_t *>(at));
        store_cluster(in_first(here), x);
        store_cluster(in_second(here), x);
    };
    auto give_up = [&](uint32_t who) {          // a wait ran out
        atomicOr(&g_xent_status, who);
        in_both(&s_abort, 1u);
    };
    // A step's copies of one operand, counted in the first CTA; both CTAs' are awaited where the MMAs are issued.
    auto expect = [&](uint32_t stage, bool is_a) {
        if (rank == 0) mbar_expect_tx(smem_u32(&s_full[stage]), kCtas * (is_a ? kBytesA : (uint32_t)(p.tn / kCtas) * kStepK * 2));
    };
    // The next unit of this pair, or one beyond the last.  Every role hears of each by itself.
    const bool handed_out = kOp == kGrads && units.steps_w >= kShort;
    uint32_t t_slot = 0, t_phase = 0;
    int64_t u = pair - pairs;
    auto next_unit = [&](bool one_thread) {
        if (!handed_out) {
            u += pairs;
            return true;
        }
        bool ok = mbar_wait_cluster(smem_u32(&s_told[t_slot]), t_phase, &s_abort);
        if (!one_thread) ok = __all_sync(0xFFFFFFFFu, ok);
        u = s_ticket[t_slot];
        if (!one_thread) __syncwarp();
        if (ok && (one_thread || lane == 0)) arrive_cluster(in_first(smem_u32(&s_heard[t_slot])));
        if (++t_slot == kTickets) { t_slot = 0; t_phase ^= 1u; }
        return ok;
    };

    if (warp < 4) {
        if constexpr (kOp == kLse) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFewRegs));
        if ((warp == 0 || warp == 3) && lane == 0) {
            // ============================ TMA producers ===========================
            // one thread for A, one for B: a copy takes its thread some 150 clocks to issue, a step of MMAs 512
            const bool is_a = warp == 0;
            const uint64_t hint = 0x1000000000000000ull;            // no preference
            const int32_t b_part = p.tn / kCtas;
            const uint32_t place = smem_base + (is_a ? 0u : kBytesA);
            uint32_t stage = 0, phase = 0, issued = 0;
            bool ok = p.give_up != kAtOnce;
            while (ok) {
                ok = next_unit(true);
                if (!ok) give_up(kTimeoutLoader);
                if (!ok || u >= units.n) break;
                const Unit w = units.at(p, u);
                for (int32_t t = 0; ok && t < w.tiles; ++t) {
                    const int32_t a_at = w.a_at + (int32_t)rank * kRowsA, b_at = w.b_at + t * p.tn + (int32_t)rank * b_part;
                    for (int32_t ks = 0; ks < w.steps; ++ks) {
                        if (!mbar_wait(smem_u32(&s_empty[stage]), phase ^ 1u, &s_abort)) {
                            give_up(kTimeoutLoader);
                            ok = false;
                            break;
                        }
                        const uint32_t bar = in_first(smem_u32(&s_full[stage])), dst = place + stage * kStageBytes;
                        const int32_t k = w.k_at + ks * kStepK;
                        expect(stage, is_a);
                        if (is_a) {
                            if (kOp != kGrads) pair_load_2d(dst, &maps.a, bar, k, a_at, hint);
                            else if (w.grad_h) pair_load_2d(dst, &maps.a, bar, 0, k / 64 * p.n_pad + a_at, hint);
                            else
                                for (int32_t j = 0; j < kRowsA; j += 64) pair_load_2d(dst + j * kStepK * 2, &maps.a_w, bar, 0, (a_at + j) / 64 * p.n_pad + k, hint);
                        } else {
                            if (kOp != kGrads) pair_load_2d(dst, &maps.b, bar, k, (kOp == kProb ? p.v0 : 0) + b_at, hint);
                            else
                                for (int32_t j = 0; j < b_part; j += 64) pair_load_2d(dst + j * kStepK * 2, w.grad_h ? &maps.b : &maps.b_w, bar, b_at + j, (w.grad_h ? p.v0 : 0) + k, hint);
                        }
                        ++issued;
                        if (++stage == kStages) { stage = 0; phase ^= 1u; }
                    }
                }
            }
            in_both(&s_issued[rank][is_a], issued);
        } else if (handed_out && warp == 2 && lane == 0 && rank == 0) {
            // ============================ units to both CTAs ======================
            uint32_t slot = 0, phase = 0;
            bool ok = p.give_up != kAtOnce;
            while (ok) {
                ok = mbar_wait_cluster(smem_u32(&s_heard[slot]), phase ^ 1u, &s_abort);
                if (!ok) { give_up(kTimeoutLoader); break; }
                const uint32_t ticket = atomicAdd(p.ticket, 1u);
                s_ticket[slot] = ticket;
                store_cluster(in_second(smem_u32(const_cast<uint32_t *>(&s_ticket[slot]))), ticket);
                arrive_cluster(in_first(smem_u32(&s_told[slot])));
                arrive_cluster(in_second(smem_u32(&s_told[slot])));
                if (ticket >= units.n) break;
                if (++slot == kTickets) { slot = 0; phase ^= 1u; }
            }
        } else if (warp == 1 && lane == 0 && rank == 0) {
            // ============================ MMA issuer ==============================
            uint32_t stage = 0, phase = 0, buf = 0, buf_phase = 0;
            bool ok = p.give_up != kAtOnce;
            while (ok) {
                ok = next_unit(true);
                if (!ok) give_up(kTimeoutMma);
                if (!ok || u >= units.n) break;
                const Unit w = units.at(p, u);
                const bool a_mn = kOp == kGrads && !w.grad_h, b_mn = kOp == kGrads;
                const uint32_t idesc = umma_idesc(kM, (uint32_t)p.tn, a_mn, b_mn);
                // 16 k further: 32 bytes along the swizzled row, or 16 rows of 128 bytes
                const uint64_t a_step = a_mn ? 128u : 2u, b_step = b_mn ? 128u : 2u;
                const int32_t span = kOp == kLse ? kSumSteps : w.steps;         // steps of a sum
                for (int32_t t = 0; ok && t < w.tiles; ++t)
                    for (int32_t k0 = 0; ok && k0 < w.steps; k0 += span) {
                        ok = mbar_wait_cluster(smem_u32(&s_acc_empty[buf]), buf_phase ^ 1u, &s_abort);
                        for (int32_t ks = k0; ok && ks < min(k0 + span, w.steps); ++ks) {
                            ok = mbar_wait(smem_u32(&s_full[stage]), phase, &s_abort);
                            if (!ok) break;
                            tc_fence_after();
                            const uint32_t a = smem_base + stage * kStageBytes, b = a + kBytesA;
                            const uint64_t a_desc = a_mn ? umma_desc_mn_sw128(a) : umma_desc_sw128(a), b_desc = b_mn ? umma_desc_mn_sw128(b) : umma_desc_sw128(b);
#pragma unroll
                            for (int k = 0; k < kStepK / 16; ++k)
                                pair_mma(tmem_base + buf * kN, a_desc + k * a_step, b_desc + k * b_step, idesc, ks > k0 || k > 0 ? 1u : 0u);
                            pair_commit(smem_u32(&s_empty[stage]));
                            if (++stage == kStages) { stage = 0; phase ^= 1u; }
                        }
                        if (p.give_up == kUnderWay) ok = false;     // (once a sum: asked at every step it costs 4 % of the products)
                        if (!ok) {
                            give_up(kTimeoutMma);
                            break;
                        }
                        pair_commit(smem_u32(&s_acc_full[buf]));
                        if (++buf == kBuffers) { buf = 0; buf_phase ^= 1u; }
                    }
            }
        }
        tc_fence_before();
        __syncwarp();
        cluster_sync();                         // neither leaves while the other may still reach its shared or tensor memory
        if (s_abort) {                          // (alike in both)
            // Copies and MMAs in flight end before their memory goes, whoever gave up and whoever came to an end.  A step's barrier in the first CTA
            // counts the copies of both operands and CTAs, so each loader makes up for the steps that another has issued before it (one round of the
            // stages at most, since no stage is filled again before all have filled it); what it loads is not used.
            if ((warp == 0 || warp == 3) && lane == 0) {
                const bool is_a = warp == 0;
                uint32_t most = 0;
                for (int c = 0; c < kCtas; ++c) most = max(most, max(s_issued[c][0], s_issued[c][1]));
                for (uint32_t k = s_issued[rank][is_a]; k < most; ++k) {
                    const uint32_t stage = k % kStages, bar = in_first(smem_u32(&s_full[stage])), dst = smem_base + stage * kStageBytes + (is_a ? 0u : kBytesA);
                    expect(stage, is_a);
                    if (is_a) pair_load_2d(dst, &maps.a, bar, 0, 0, 0x1000000000000000ull);
                    else
                        for (int32_t j = 0; j < p.tn / kCtas; j += kOp == kGrads ? 64 : p.tn / kCtas) pair_load_2d(dst + j * kStepK * 2, &maps.b, bar, 0, 0, 0x1000000000000000ull);
                }
                if (is_a && rank == 0)
                    for (uint32_t st = 0; st < kStages; ++st) {
                        const uint32_t fills = (most + kStages - 1u - st) / kStages;
                        for (uint32_t t = 0; fills && t < TC_WAIT_LIMIT && !mbar_try_wait(smem_u32(&s_full[st]), (fills - 1u) & 1u); ++t) { }
                    }
            }
            if (warp == 1 && lane == 0) {
                if (rank == 0) pair_commit(smem_u32(&s_drain));
                for (uint32_t t = 0; t < TC_WAIT_LIMIT && !mbar_try_wait(smem_u32(&s_drain), 0); ++t) { }
            }
            __syncwarp();
            cluster_sync();
        }
    } else {
        // ============================ epilogue ================================
        if constexpr (kOp == kLse) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kManyRegs));
        const int e = warp - 4;
        const uint32_t quarter = (uint32_t)warp & 3u;               // tensor-memory lanes 32 * quarter .. + 31
        const int32_t half = e >> 2, cols = p.tn / 2, c0 = half * cols;     // this warp's columns: a multiple of 16
        const int32_t first_row = (int32_t)(rank * kRowsA + quarter * 32u), row_in_tile = first_row + lane;
        const uint32_t room = smem_base + kStages * kStageBytes + (uint32_t)e * kRoom;
        uint32_t buf = 0, buf_phase = 0;
        bool ok = p.give_up != kAtOnce;
        // 64 finished columns of this warp's rows leave by an asynchronous copy
        auto send = [&](const uint32_t (&out)[32], int32_t x, int32_t y, bool there) {
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");     // what was there has left
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 8; ++i)
                asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(room + (uint32_t)(lane * 128 + ((i ^ (lane & 7)) * 16))), "r"(out[4 * i]),
                             "r"(out[4 * i + 1]), "r"(out[4 * i + 2]), "r"(out[4 * i + 3])
                             : "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                if (there) tma_store_2d(&maps.out, room, x, y);
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            }
        };
        while (ok) {
            ok = next_unit(false);
            if (!ok || u >= units.n) break;
            const Unit w = units.at(p, u);
            const int32_t row = w.a_at + row_in_tile;
            const bool live = row < units.n_live;                   // (grad W's rows are the vocabulary's: it has no use for this)
            int32_t target = -1;
            float lse = 0.f, coef = 0.f, top = -3.4e38f;
            float2 sum = make_float2(0.f, 0.f);                     // kLse: relative to the top; kProb: of probabilities
            float was = 0.f;
            float *part_p = nullptr;
            if (kOp != kGrads && live) target = p.target[row];
            if (kOp == kProb && live) {
                lse = p.lse[row];
                coef = p.coef[row];
                part_p = p.part_p + (int64_t)(2 * (w.b_at / p.tn) + half) * p.ld_p + row;
                if (!p.first) was = *part_p;
            }
            float *kept_row = nullptr;                              // grad W: where this thread's vocabulary row is kept in fp32, if it is a target
            if (kOp == kGrads && !w.grad_h && p.v0 + row < p.V) {
                const uint32_t at = p.first_row[p.v0 + row];
                if (at != kNone) kept_row = p.sum_w + (p.by_id ? (int64_t)(p.v0 + row) : (int64_t)at) * p.d + w.b_at + c0;
            }
            for (int32_t t = 0; t < w.tiles; ++t) {
                float4 *at = nullptr;                               // grad H's sums of this row, four columns each
                if constexpr (kOp == kGrads) {
                    at = reinterpret_cast<float4 *>(p.sum_h) + ((int64_t)w.index * (p.tn / 4) + c0 / 4) * kM + row_in_tile;
                    if (w.steps == 0) {         // (a part of a short last piece that has nothing to add)
                        if (p.first && live)
                            for (int32_t c = 0; c < cols; c += 4) at[(int64_t)(c / 4) * kM] = make_float4(0.f, 0.f, 0.f, 0.f);
                        continue;
                    }
                }
                if constexpr (kOp == kLse) {
                    float2 z[kN / 4];
#pragma unroll
                    for (int j = 0; j < kN / 4; ++j) z[j] = make_float2(0.f, 0.f);
                    for (int32_t k0 = 0; k0 < w.steps; k0 += kSumSteps) {
                        ok = mbar_wait(smem_u32(&s_acc_full[buf]), buf_phase, &s_abort);
                        if (!__all_sync(0xFFFFFFFFu, ok)) { ok = false; break; }
                        tc_fence_after();
                        const uint32_t taddr = tmem_base + ((quarter * 32u) << 16) + buf * kN + (uint32_t)c0;
#pragma unroll
                        for (int c = 0; c < kN / 2; c += 32) {
                            uint32_t r[32];
                            tmem_ld32(taddr + (uint32_t)c, r);
                            tmem_ld_wait();
#pragma unroll
                            for (int j = 0; j < 16; ++j) z[c / 2 + j] = __fadd2_rn(z[c / 2 + j], make_float2(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1])));
                        }
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) arrive_cluster(in_first(smem_u32(&s_acc_empty[buf])));
                        if (++buf == kBuffers) { buf = 0; buf_phase ^= 1u; }
                    }
                    if (!ok) break;
                    const int32_t v0 = w.b_at + t * p.tn + c0, left = p.V - v0, mine = target - v0;
                    if (left < kN / 2)
#pragma unroll
                        for (int j = 0; j < kN / 4; ++j) {
                            z[j].x = 2 * j < left ? z[j].x : -INFINITY;
                            z[j].y = 2 * j + 1 < left ? z[j].y : -INFINITY;
                        }
                    if ((uint32_t)mine < (uint32_t)(kN / 2))        // the target takes part where the sums are joined
#pragma unroll
                        for (int j = 0; j < kN / 4; ++j) {
                            z[j].x = mine == 2 * j ? -INFINITY : z[j].x;
                            z[j].y = mine == 2 * j + 1 ? -INFINITY : z[j].y;
                        }
                    float best[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) best[i] = top;
#pragma unroll
                    for (int j = 0; j < kN / 4; ++j) best[j & 7] = fmaxf(best[j & 7], fmaxf(z[j].x, z[j].y));
#pragma unroll
                    for (int i = 4; i > 0; i >>= 1)
#pragma unroll
                        for (int j = 0; j < i; ++j) best[j] = fmaxf(best[j], best[j + i]);
                    const float by = tfe_rows::exp2_approx((top - best[0]) * kLog2e);
                    top = best[0];
                    sum.x *= by; sum.y *= by;
                    float2 more = make_float2(0.f, 0.f);
                    const float2 minus = make_float2(-top, -top), times = make_float2(kLog2e, kLog2e);
#pragma unroll
                    for (int j = 0; j < kN / 4; ++j) {
                        const float2 y = __fmul2_rn(__fadd2_rn(z[j], minus), times), x = make_float2(tfe_rows::exp2_approx(y.x), tfe_rows::exp2_approx(y.y));
                        if (j & 1) more = __fadd2_rn(more, x); else sum = __fadd2_rn(sum, x);
                    }
                    sum = __fadd2_rn(sum, more);
                    continue;
                }
                ok = mbar_wait(smem_u32(&s_acc_full[buf]), buf_phase, &s_abort);
                if (!__all_sync(0xFFFFFFFFu, ok)) { ok = false; break; }
                tc_fence_after();
                const uint32_t taddr = tmem_base + ((quarter * 32u) << 16) + buf * kN + (uint32_t)c0;
                auto release = [&] {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) arrive_cluster(in_first(smem_u32(&s_acc_empty[buf])));
                };
                // 16 columns at a time, the next ones on their way meanwhile
                uint32_t r[2][16];
                tmem_ld16(taddr, r[0]);
                if (kOp == kProb || !w.grad_h) {
                    const int32_t v0 = p.v0 + w.b_at + c0, left = p.V - v0, mine = target - v0;
                    const float2 minus = make_float2(-lse, -lse), by = make_float2(kLog2e, kLog2e), times = make_float2(coef, coef);
                    // 16 columns in bf16: of G, or of grad W
                    auto take = [&](const uint32_t (&x)[16], int32_t c, uint32_t (&out)[8]) {
                        float2 y[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) y[j] = make_float2(__uint_as_float(x[2 * j]), __uint_as_float(x[2 * j + 1]));
                        if constexpr (kOp == kProb) {
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                y[j] = __fmul2_rn(__fadd2_rn(y[j], minus), by);
                                y[j] = make_float2(tfe_rows::exp2_approx(y[j].x), tfe_rows::exp2_approx(y[j].y));
                            }
                            if (c + 16 > left)
#pragma unroll
                                for (int j = 0; j < 8; ++j) {
                                    y[j].x = c + 2 * j < left ? y[j].x : 0.f;
                                    y[j].y = c + 2 * j + 1 < left ? y[j].y : 0.f;
                                }
                            const bool here = (uint32_t)(mine - c) < 16u;
                            float z = 0.f;
                            if (here)
#pragma unroll
                                for (int j = 0; j < 16; ++j) {
                                    z = mine - c == j ? __uint_as_float(x[j]) : z;
                                    (j & 1 ? y[j / 2].y : y[j / 2].x) = mine - c == j ? 0.f : (j & 1 ? y[j / 2].y : y[j / 2].x);
                                }
                            float2 more = __fadd2_rn(y[0], y[1]);
#pragma unroll
                            for (int j = 2; j < 8; ++j) more = __fadd2_rn(more, y[j]);
                            sum = __fadd2_rn(sum, more);
#pragma unroll
                            for (int j = 0; j < 8; ++j) y[j] = __fmul2_rn(y[j], times);
                            if (here) {
                                const float g = expm1f(z - lse), kept = g > -kSure ? 0.f : __bfloat162float(__float2bfloat16_rn(coef * g));
                                p.rest[row] = kept;
                                atomicMin(p.first_row + target, (uint32_t)row);
#pragma unroll
                                for (int j = 0; j < 8; ++j) {
                                    y[j].x = mine - c == 2 * j ? kept : y[j].x;
                                    y[j].y = mine - c == 2 * j + 1 ? kept : y[j].y;
                                }
                            }
                            if (!live)          // (not 0 times what may be NaN where a weight is infinite)
#pragma unroll
                                for (int j = 0; j < 8; ++j) y[j] = make_float2(0.f, 0.f);
                        } else {
                            if (kept_row)
#pragma unroll
                                for (int i = 0; i < 4; ++i)
                                    if (w.b_at + c0 + c + 4 * i < p.d)
                                        *reinterpret_cast<float4 *>(kept_row + c + 4 * i) = make_float4(y[2 * i].x, y[2 * i].y, y[2 * i + 1].x, y[2 * i + 1].y);
                        }
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const __nv_bfloat162 b2 = __floats2bfloat162_rn(y[j].x, y[j].y);
                            out[j] = *reinterpret_cast<const uint32_t *>(&b2);
                        }
                    };
                    for (int32_t c = 0; c < cols; c += 64) {        // (cols: 64 or 128)
                        uint32_t out[4][8];
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            tmem_ld_wait();
                            if (q < 3 || c + 64 < cols) tmem_ld16(taddr + (uint32_t)(c + 16 * (q + 1)), r[(q + 1) & 1]);
                            take(r[q & 1], c + 16 * q, out[q]);
                        }
                        if (c + 64 >= cols) release();
                        if constexpr (kOp == kProb) {
                            send(reinterpret_cast<const uint32_t (&)[32]>(out), 0, (w.b_at + c0 + c) / 64 * p.n_pad + w.a_at + first_row, true);
                        } else {                // (what lies beyond the matrix is not written)
                            const int32_t x0 = w.b_at + c0 + c, y0 = p.v0 + w.a_at + first_row;
                            send(reinterpret_cast<const uint32_t (&)[32]>(out), x0, y0, x0 < p.d && y0 < p.V);
                        }
                    }
                } else {
                    float4 old[2][4];
                    auto fetch = [&](int32_t c, float4 (&x)[4]) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[i] = p.first || !live ? make_float4(0.f, 0.f, 0.f, 0.f) : at[(int64_t)(c / 4 + i) * kM];
                    };
                    auto take = [&](const uint32_t (&x)[16], int32_t c, const float4 (&was)[4]) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (live) at[(int64_t)(c / 4 + i) * kM] = make_float4(__uint_as_float(x[4 * i]) + was[i].x, __uint_as_float(x[4 * i + 1]) + was[i].y,
                                                                        __uint_as_float(x[4 * i + 2]) + was[i].z, __uint_as_float(x[4 * i + 3]) + was[i].w);
                    };
                    fetch(0, old[0]);
                    for (int32_t c = 0; c < cols; c += 32) {        // (cols: 64 or 128)
                        fetch(c + 16, old[1]);
                        tmem_ld_wait();
                        tmem_ld16(taddr + (uint32_t)(c + 16), r[1]);
                        take(r[0], c, old[0]);
                        if (c + 32 < cols) fetch(c + 32, old[0]);
                        tmem_ld_wait();
                        if (c + 32 < cols) tmem_ld16(taddr + (uint32_t)(c + 32), r[0]);
                        take(r[1], c + 16, old[1]);
                    }
                    release();
                }
                if (++buf == kBuffers) { buf = 0; buf_phase ^= 1u; }
            }
            if (!ok) break;
            if constexpr (kOp == kLse)
                if (live) p.part[(int64_t)(2 * w.index + half) * p.ld_part + row] = make_float2(top, sum.x + sum.y);
            if constexpr (kOp == kProb)
                if (live) *part_p = was + (sum.x + sum.y);
        }
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        if (!ok && lane == 0) {                 // a wait ran out: no results that look like some (the last kernel sees to that)
            give_up(kTimeoutEpilogue);
            *p.failed = 1;
        }
        tc_fence_before();
        __syncwarp();
        cluster_sync();                         // as the others: once, and once more for what is in flight
        if (s_abort) cluster_sync();
    }
    if (warp == 1) {
        tc_fence_after();
        pair_tmem_dealloc(tmem_base, kBuffers * kN);
    }
}

// ------------------------------------------------------------------ few rows

// The loss of up to this many rows: the read of the weights bounds it.  The weights' rows are the MMA's M (128), the hidden states' its
// N (16..64), so no tensor time goes to rows that are not there: 1 x 151,936 x 1,024 takes 54 us (5.8 TB/s), 65 us in tiles of 256 rows.  The
// vocabulary is cut into equal row ranges, one per SM.  A thread holds one vocabulary row at a time and keeps the running maxima and
// sums of its columns, the hidden states, in registers until the end.
constexpr int kFewRows = 64;
constexpr int kFewCtas = 160;                   // at most: bounds the partial results
constexpr int kFewM = 128, kFewSteps = 2;       // rows of a tile, steps of a stage
constexpr int kFewMaxStages = 6, kFewBuffers = 4;
constexpr int kFewEpilogueWarps = 8, kFewThreads = 32 * (2 + kFewEpilogueWarps);
__host__ __device__ constexpr int few_stage(int tn) { return kFewSteps * (kFewM + tn) * kStepK * 2; }       // bytes
__host__ __device__ constexpr int few_stages(int tn) { return 223 * 1024 / few_stage(tn) < kFewMaxStages ? 223 * 1024 / few_stage(tn) : kFewMaxStages; }

struct FewParams {
    int32_t N, V, steps, rows_per_cta, tail_rows;
    uint32_t give_up;
    const int32_t *target;
    float2 *part; int64_t ld_part;              // [4 * CTAs][ld_part]
};

template <int TN>
__global__ void __launch_bounds__(kFewThreads, 1)
tfe_xent_few_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_w_tail, const __grid_constant__ CUtensorMap map_h,
                    const FewParams p)
{
    constexpr int kStagesHere = few_stages(TN), kCols = TN / 2;
    constexpr uint32_t kTmemCols = kFewBuffers * TN, kW = kFewM * kStepK * 2, kH = TN * kStepK * 2, kBytes = kFewSteps * (kW + kH);
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t s_full[kFewMaxStages], s_empty[kFewMaxStages], s_acc_full[kFewBuffers], s_acc_empty[kFewBuffers], s_drain;
    __shared__ uint32_t s_tmem_base;
    __shared__ volatile uint32_t s_abort, s_issued;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStagesHere; ++s) { mbar_init(smem_u32(&s_full[s]), 1); mbar_init(smem_u32(&s_empty[s]), 1); }
        for (int a = 0; a < kFewBuffers; ++a) { mbar_init(smem_u32(&s_acc_full[a]), 1); mbar_init(smem_u32(&s_acc_empty[a]), kFewEpilogueWarps); }
        mbar_init(smem_u32(&s_drain), 1);
        s_abort = s_issued = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(smem_u32(&s_tmem_base), kTmemCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = s_tmem_base;
    tfe_wait_for_stream();
    const int64_t r0 = (int64_t)blockIdx.x * p.rows_per_cta;
    const int32_t n_rows = (int32_t)min((int64_t)p.rows_per_cta, p.V - r0), n_tiles = (n_rows + kFewM - 1) / kFewM;

    if (warp == 0) {
        // ============================ TMA producer ============================
        if (lane == 0) {
            const uint64_t hint_w = 0x12F0000000000000ull, hint_h = 0x14F0000000000000ull;      // evict first, evict last
            uint32_t stage = 0, phase = 0, issued = 0;
            bool ok = p.give_up != kAtOnce;
            for (int32_t t = 0; ok && t < n_tiles; ++t) {
                const int32_t valid = min(kFewM, n_rows - t * kFewM);
                // a short last tile is fetched with the short box: only its rows are read
                const bool tail = valid < kFewM && valid == p.tail_rows;
                const uint32_t w_bytes = tail ? (uint32_t)p.tail_rows * kStepK * 2 : kW;
                for (int32_t ks = 0; ks < p.steps; ks += kFewSteps) {
                    if (!mbar_wait(smem_u32(&s_empty[stage]), phase ^ 1u, &s_abort)) {
                        atomicOr(&g_xent_status, kTimeoutLoader);
                        s_abort = 1;
                        ok = false;
                        break;
                    }
                    const uint32_t bar = smem_u32(&s_full[stage]), dst = smem_base + stage * kBytes;
                    const int32_t n = min(kFewSteps, p.steps - ks);
                    mbar_expect_tx(bar, (uint32_t)n * (w_bytes + kH));
                    for (int32_t i = 0; i < n; ++i) {
                        tma_load_2d(dst + i * (kW + kH), tail ? &map_w_tail : &map_w, bar, (ks + i) * kStepK, (int32_t)(r0 + (int64_t)t * kFewM), hint_w);
                        tma_load_2d(dst + i * (kW + kH) + kW, &map_h, bar, (ks + i) * kStepK, 0, hint_h);
                    }
                    ++issued;
                    if (++stage == kStagesHere) { stage = 0; phase ^= 1u; }
                }
            }
            s_issued = issued;
        }
    } else if (warp == 1) {
        // ============================ MMA issuer ==============================
        if (lane == 0) {
            constexpr uint32_t idesc = umma_idesc(kFewM, TN, false, false);
            uint32_t stage = 0, phase = 0, buf = 0, buf_phase = 0;
            bool ok = p.give_up != kAtOnce;
            for (int32_t t = 0; ok && t < n_tiles; ++t)
                for (int32_t ks = 0; ok && ks < p.steps; ks += kFewSteps) {
                    ok = mbar_wait(smem_u32(&s_acc_empty[buf]), buf_phase ^ 1u, &s_abort) && mbar_wait(smem_u32(&s_full[stage]), phase, &s_abort);
                    if (ok) {
                        tc_fence_after();
                        for (int32_t i = 0; i < min(kFewSteps, p.steps - ks); ++i) {
                            const uint32_t at = smem_base + stage * kBytes + i * (kW + kH);
                            const uint64_t w_desc = umma_desc_sw128(at), h_desc = umma_desc_sw128(at + kW);
#pragma unroll
                            for (int k = 0; k < kStepK / 16; ++k)
                                umma_bf16(tmem_base + buf * TN, w_desc + 2 * k, h_desc + 2 * k, idesc, i > 0 || k > 0 ? 1u : 0u);
                        }
                        umma_commit(smem_u32(&s_empty[stage]));
                        if (++stage == kStagesHere) { stage = 0; phase ^= 1u; }
                    }
                    if (p.give_up == kUnderWay) ok = false;
                    if (!ok) {
                        atomicOr(&g_xent_status, kTimeoutMma);
                        s_abort = 1;
                        break;
                    }
                    umma_commit(smem_u32(&s_acc_full[buf]));
                    if (++buf == kFewBuffers) { buf = 0; buf_phase ^= 1u; }
                }
        }
    } else {
        // ============================ epilogue ================================
        const uint32_t quarter = (uint32_t)warp & 3u;               // tensor-memory lanes 32 * quarter .. + 31
        const int32_t c0 = ((warp - 2) >> 2) * kCols, row_in_tile = (int32_t)(quarter * 32u) + lane;
        float top[kCols], sum[kCols];
        int32_t target[kCols];
#pragma unroll
        for (int j = 0; j < kCols; ++j) {
            top[j] = -3.4e38f;
            sum[j] = 0.f;
            target[j] = c0 + j < p.N ? p.target[c0 + j] : -1;
        }
        uint32_t buf = 0, buf_phase = 0;
        bool ok = p.give_up != kAtOnce;
        for (int32_t t = 0; ok && t < n_tiles; ++t) {
            float z[kCols];
            for (int32_t k0 = 0; k0 < p.steps; k0 += kFewSteps) {
                ok = mbar_wait(smem_u32(&s_acc_full[buf]), buf_phase, &s_abort);
                if (!__all_sync(0xFFFFFFFFu, ok)) { ok = false; break; }
                tc_fence_after();
                const uint32_t taddr = tmem_base + ((quarter * 32u) << 16) + buf * TN + (uint32_t)c0;
                uint32_t r[kCols];
                if constexpr (kCols == 32) tmem_ld32(taddr, r);
                else if constexpr (kCols == 16) tmem_ld16(taddr, r);
                else tmem_ld8(taddr, r);
                tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < kCols; ++j) z[j] = k0 == 0 ? __uint_as_float(r[j]) : z[j] + __uint_as_float(r[j]);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&s_acc_empty[buf]));
                if (++buf == kFewBuffers) { buf = 0; buf_phase ^= 1u; }
            }
            if (!ok) break;
            const int32_t row = t * kFewM + row_in_tile, v = (int32_t)r0 + row;
            if (row >= n_rows) continue;
#pragma unroll
            for (int j = 0; j < kCols; ++j) {
                const float x = target[j] == v ? -INFINITY : z[j];  // (the target takes part where the sums are joined)
                const float best = fmaxf(top[j], x);
                sum[j] = sum[j] * tfe_rows::exp2_approx((top[j] - best) * kLog2e) + tfe_rows::exp2_approx((x - best) * kLog2e);
                top[j] = best;
            }
        }
        if (!ok) {                              // a wait ran out: no results that look like some
            if (lane == 0) atomicOr(&g_xent_status, kTimeoutEpilogue);
            s_abort = 1;
#pragma unroll
            for (int j = 0; j < kCols; ++j) sum[j] = __int_as_float(0x7FFFFFFF);
        }
#pragma unroll
        for (int j = 0; j < kCols; ++j) {
            for (int o = 16; o > 0; o >>= 1) {
                const float top2 = __shfl_xor_sync(0xFFFFFFFFu, top[j], o), sum2 = __shfl_xor_sync(0xFFFFFFFFu, sum[j], o), best = fmaxf(top[j], top2);
                sum[j] = sum[j] * tfe_rows::exp2_approx((top[j] - best) * kLog2e) + sum2 * tfe_rows::exp2_approx((top2 - best) * kLog2e);
                top[j] = best;
            }
            if (lane == 0 && c0 + j < p.N) p.part[(int64_t)(4 * blockIdx.x + quarter) * p.ld_part + c0 + j] = make_float2(top[j], sum[j]);
        }
    }

    tc_fence_before();
    __syncthreads();
    if (s_abort) {                              // copies and MMAs in flight end before their memory goes
        if (warp == 0 && lane == 0)
            for (uint32_t s = 0; s < kStagesHere; ++s) {
                const uint32_t fills = (s_issued + kStagesHere - 1u - s) / kStagesHere;
                for (uint32_t t = 0; fills && t < TC_WAIT_LIMIT && !mbar_try_wait(smem_u32(&s_full[s]), (fills - 1u) & 1u); ++t) { }
            }
        if (warp == 1 && lane == 0) {
            umma_commit(smem_u32(&s_drain));
            for (uint32_t t = 0; t < TC_WAIT_LIMIT && !mbar_try_wait(smem_u32(&s_drain), 0); ++t) { }
        }
        __syncthreads();
    }
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tmem_base, kTmemCols);
    }
}

// ------------------------------------------------------------------ joining

struct LossParams {
    int32_t N, V, d, chunks, rows;              // rows: of a block, a power of two
    const float2 *part; int64_t ld_part;
    const int32_t *target, *pos;                // pos null: rows are where they were
    const uint32_t *failed;                     // null: a failure is in the partial results
    const bf16 *h, *w; int64_t ld_h, ld_w;
    float *loss, *lse;
};
constexpr int kLossThreads = 512, kLossRows = 32;

// Joins maxima and sums, relative to the greater of the maxima (which is never -inf: tiles begin at -3.4e38).
__device__ __forceinline__ void fold(float &top, float &sum, float top2, float sum2)
{
    const float best = fmaxf(top, top2);
    sum = sum * tfe_rows::exp2_approx((top - best) * kLog2e) + sum2 * tfe_rows::exp2_approx((top2 - best) * kLog2e);
    top = best;
}

// A row's partial results joined by kLossThreads / rows threads: 5 us for one row (a chain of loads), 16 us for 4,096.  With o the log of
// the other ids' sum, loss = ln(1 + exp(o - z_t)): however near zero, it is as exact as a fraction as the logits are.  (As lse - z_t with the
// target in the sums it was off by 1e-7, a tenth of a loss of 1e-6.)  z_t is summed here: the tensor cores cut what they add.
__global__ void __launch_bounds__(kLossThreads)
tfe_xent_loss_kernel(const LossParams p)
{
    constexpr int kWarps = kLossThreads / 32;
    __shared__ float s_top[kLossRows][kWarps], s_sum[kLossRows][kWarps];
    __shared__ double s_z[kLossRows];
    tfe_wait_for_stream();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t r0 = (int64_t)blockIdx.x * p.rows;
    auto place = [&](int64_t r) -> int64_t {    // of a row among those that took part, -1 if it did not
        const int32_t t = r < p.N ? p.target[r] : -1;
        return t < 0 || t >= p.V ? -1 : p.pos ? p.pos[r] : r;
    };
    {
        const int i = threadIdx.x & (p.rows - 1), step = kLossThreads / p.rows;
        const int64_t r = r0 + i, at = r < p.N ? p.pos ? p.pos[r] : r : -1;         // (rows without a target have results too, or none)
        float top = -3.4e38f, sum = 0.f;
        if (at >= 0) {
#pragma unroll 4
            for (int32_t c = threadIdx.x / p.rows; c < p.chunks; c += step) {
                const float2 x = p.part[(int64_t)c * p.ld_part + at];
                fold(top, sum, x.x, x.y);
            }
        }
        for (int o = 16; o >= p.rows; o >>= 1) fold(top, sum, __shfl_xor_sync(0xFFFFFFFFu, top, o), __shfl_xor_sync(0xFFFFFFFFu, sum, o));
        if (lane < p.rows) { s_top[i][warp] = top; s_sum[i][warp] = sum; }
    }
    for (int i = warp; i < p.rows; i += kWarps) {
        const int64_t r = r0 + i;
        const int32_t t = r < p.N ? p.target[r] : -1;
        if (t < 0 || t >= p.V) continue;
        const uint4 *h = reinterpret_cast<const uint4 *>(p.h + r * p.ld_h), *w = reinterpret_cast<const uint4 *>(p.w + (int64_t)t * p.ld_w);
        double z = 0.0;
#pragma unroll 4
        for (int32_t v = lane; v < p.d / 8; v += 32) {
            float a[8], b[8], x = 0.f;
            tfe_rows::Elem<bf16>::unpack(h[v], a);
            tfe_rows::Elem<bf16>::unpack(w[v], b);
#pragma unroll
            for (int j = 0; j < 8; ++j) x = fmaf(a[j], b[j], x);
            z += (double)x;
        }
        for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xFFFFFFFFu, z, o);
        if (lane == 0) s_z[i] = z;
    }
    __syncthreads();
    for (int i = warp; i < p.rows; i += kWarps) {
        const int64_t r = r0 + i, at = place(r);
        float top = s_top[i][lane & (kWarps - 1)], sum = s_sum[i][lane & (kWarps - 1)];
        for (int o = kWarps / 2; o > 0; o >>= 1) fold(top, sum, __shfl_xor_sync(0xFFFFFFFFu, top, o), __shfl_xor_sync(0xFFFFFFFFu, sum, o));
        if (lane != 0 || r >= p.N) continue;
        if (at < 0) { p.loss[r] = p.lse[r] = 0.f; continue; }
        const double z = s_z[i], others = (double)top + log((double)sum), x = others - z, more = log1p(exp(-fabs(x)));
        // z_t = -inf: a loss of +inf, the log-sum-exp of the others.  +inf: NaN, as lse - z_t is
        const bool bad = !(z < INFINITY) || (p.failed && *p.failed);
        p.lse[r] = bad ? __int_as_float(0x7FFFFFFF) : (float)(fmax(others, z) + more);
        p.loss[r] = bad ? __int_as_float(0x7FFFFFFF) : (float)(fmax(x, 0.0) + more);
    }
}

struct RestParams {
    int32_t chunks;
    const int32_t *n_live;
    const float *part_p; int64_t ld_p;
    const float *coef;
    float *rest;                                // in: what the products have; out: G less that
};
constexpr int kRestWarps = 32;

// A block for 32 rows, whose sums lie side by side: a chain of loads, 4 us of the 91 that both gradients of 33 x 32,003 x 1,000 take.
__global__ void __launch_bounds__(32 * kRestWarps)
tfe_xent_rest_kernel(const RestParams p)
{
    __shared__ float s_sum[kRestWarps][33];
    tfe_wait_for_stream();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t row = blockIdx.x * 32 + lane, n_live = *p.n_live;
    float sum = 0.f;
    if (row < n_live)
#pragma unroll 16
        for (int32_t c = warp; c < p.chunks; c += kRestWarps) sum += p.part_p[(int64_t)c * p.ld_p + row];
    s_sum[warp][lane] = sum;
    __syncthreads();
    sum = s_sum[lane][warp];                    // row `warp` now, from 32 parts
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    const int32_t mine = blockIdx.x * 32 + warp;
    if (lane != 0 || mine >= n_live) return;
    const float kept = p.rest[mine];            // (where it is not finite the products have made the results what they are)
    p.rest[mine] = fabsf(kept) <= 3.402823466e38f ? fmaf(-p.coef[mine], sum, -kept) : 0.f;
}

struct RowsParams {
    int32_t N, V, d, splits, m_room, cols, tn, groups;          // groups: of 32 columns
    const float *sum_h, *rest;
    const int32_t *pos, *target, *n_live;
    const bf16 *h, *w; int64_t ld_weight;       // h: the rows together, d apart
    const uint32_t *failed, *first_row;
    float *sum_w; int32_t by_id;
    const int32_t *group_at;
    int32_t slices, id_blocks;                  // slices of columns; blocks for the targets' rows of grad W, which are the first
    bf16 *grad_h; int64_t ld_h;
    bf16 *grad_w; int64_t ld_w;
};
constexpr int kRowsThreads = 256;

// Completes the rows of grad W of the targets: the row that was kept, and the sum over the id's rows of rest h, rounded.  The rows lie in
// the order of their targets, so those of an id are one run in each group.  A block looks at kSpan rows and takes the ids whose first row
// is among them, 256 columns: a warp for each id, or the whole block where the first run is longer than kLong, its warps in turn.
constexpr int kSpan = 32, kLong = 16, kSlice = 256;

struct Run { int32_t at, end; };
// The run of an id that begins at `at`, or is sought from there to `end` (a warp's work).
__device__ __forceinline__ int32_t run_end(const int32_t *target, int32_t at, int32_t end, int32_t id, int lane)
{
    for (; at < end; at += 32) {
        const uint32_t other = __ballot_sync(0xFFFFFFFFu, at + lane >= end || target[at + lane] != id);
        if (other) return at + __ffs(other) - 1;
    }
    return end;
}
__device__ __forceinline__ int32_t find_run(const int32_t *target, int32_t lo, int32_t hi, int32_t id, int lane)      // the first that is not below id
{
    while (lo < hi) {
        const int32_t step = (hi - lo + 31) / 32, at = lo + lane * step;
        const uint32_t below = __ballot_sync(0xFFFFFFFFu, at < hi && target[at] < id);        // a run of ones from lane 0
        const int32_t n = __popc(below);
        if (n == 0) return lo;
        hi = min(hi, lo + n * step);
        lo += (n - 1) * step + 1;
    }
    return lo;
}
// rest h over the rows from `at`, every step-th, eight columns
__device__ __forceinline__ void add_rows(const RowsParams &p, int32_t at, int32_t end, int32_t step, int32_t c, float (&acc)[8])
{
#pragma unroll 4
    for (int32_t k = at; k < end; k += step) {
        float f[8];
        tfe_rows::Elem<bf16>::unpack(__ldg(reinterpret_cast<const uint4 *>(p.h + (int64_t)k * p.d + c)), f);
        const float by = p.rest[k];
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = fmaf(by, f[j], acc[j]);
    }
}
__device__ __forceinline__ void finish_row(const RowsParams &p, int32_t id, int32_t first, int32_t c, const float (&acc)[8])
{
    const float4 *kept = reinterpret_cast<const float4 *>(p.sum_w + (p.by_id ? (int64_t)id : (int64_t)first) * p.d + c);
    const float4 a = kept[0], b = kept[1];
    const float f[8] = {a.x + acc[0], a.y + acc[1], a.z + acc[2], a.w + acc[3], b.x + acc[4], b.y + acc[5], b.z + acc[6], b.w + acc[7]};
    *reinterpret_cast<uint4 *>(p.grad_w + (int64_t)id * p.ld_w + c) = tfe_rows::Elem<bf16>::pack(f);
}

__device__ __forceinline__ void finish_targets(const RowsParams &p, int32_t first, int32_t column)
{
    __shared__ float4 s_part[kRowsThreads / 32][2][32];
    __shared__ uint32_t s_long;
    constexpr int kWarps = kRowsThreads / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t n_live = *p.n_live, all_groups = (p.N + kGroup - 1) / kGroup, c = column + lane * 8;
    if (first >= n_live) return;
    const int32_t mine = first + lane < n_live ? p.target[first + lane] : -1;
    const uint32_t heads = __ballot_sync(0xFFFFFFFFu, mine >= 0 && p.first_row[mine] == (uint32_t)(first + lane));
    if (threadIdx.x == 0) s_long = 0;
    __syncthreads();
    int32_t group = 0;                          // that these rows are in
    while (group + 1 < all_groups && p.group_at[group + 1] <= first) ++group;
    auto next_run = [&](Run &r, int32_t &g, int32_t id) {           // in the groups behind
        for (++g; g < all_groups; ++g) {
            const int32_t end = p.group_at[g + 1];
            r.at = find_run(p.target, p.group_at[g], end, id, lane);
            r.end = run_end(p.target, r.at, end, id, lane);
            if (r.at < r.end) return true;
        }
        return false;
    };
    int32_t turn = 0;
    for (uint32_t left = heads; left; left &= left - 1, ++turn) {
        if (turn % kWarps != warp) continue;
        const int32_t l = __ffs(left) - 1, id = __shfl_sync(0xFFFFFFFFu, mine, l);
        int32_t g = group;
        while (g + 1 < all_groups && p.group_at[g + 1] <= first + l) ++g;      // (the block's rows may run over a group's end)
        Run r{first + l, 0};
        r.end = run_end(p.target, r.at, p.group_at[g + 1], id, lane);
        if (r.end - r.at > kLong) {
            if (lane == 0) atomicOr(&s_long, 1u << l);
            continue;
        }
        float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        do {
            if (c < p.d) add_rows(p, r.at, r.end, 1, c, acc);
        } while (next_run(r, g, id));
        if (c < p.d) finish_row(p, id, first + l, c, acc);
    }
    __syncthreads();
    for (uint32_t left = s_long; left; left &= left - 1) {
        const int32_t l = __ffs(left) - 1, id = __shfl_sync(0xFFFFFFFFu, mine, l);
        int32_t g = group;
        while (g + 1 < all_groups && p.group_at[g + 1] <= first + l) ++g;
        Run r{first + l, 0};
        r.end = run_end(p.target, r.at, p.group_at[g + 1], id, lane);
        float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        do {
            if (c < p.d) add_rows(p, r.at + warp, r.end, kWarps, c, acc);
        } while (next_run(r, g, id));
        __syncthreads();
        s_part[warp][0][lane] = make_float4(acc[0], acc[1], acc[2], acc[3]);
        s_part[warp][1][lane] = make_float4(acc[4], acc[5], acc[6], acc[7]);
        __syncthreads();
        if (warp == 0) {
            for (int w = 1; w < kWarps; ++w) {
                const float4 x = s_part[w][0][lane], y = s_part[w][1][lane];
                acc[0] += x.x; acc[1] += x.y; acc[2] += x.z; acc[3] += x.w;
                acc[4] += y.x; acc[5] += y.y; acc[6] += y.z; acc[7] += y.w;
            }
            if (c < p.d) finish_row(p, id, first + l, c, acc);
        }
    }
}

// grad H's sums over the parts, rounded, to their rows, a block for 32 rows and 32 columns; NaN everywhere if a product before it failed.
// Bound by the read of the parts: 24 us for 4,096 x 1,024; 44 us with the targets' rows of grad W, 180 us where all rows have one target.
__global__ void __launch_bounds__(kRowsThreads)
tfe_xent_rows_kernel(const RowsParams p)
{
    __shared__ float4 s_sum[32][kRowsThreads / 32 + 1];
    tfe_wait_for_stream();
    const bool failed = *p.failed != 0;
    const bf16 nan = __float2bfloat16_rn(__int_as_float(0x7FFFFFFF));
    if (blockIdx.x < p.id_blocks) {
        if (!failed) finish_targets(p, (int32_t)(blockIdx.x / p.slices) * kSpan, (int32_t)(blockIdx.x % p.slices) * kSlice);
    } else {
        const uint32_t block = blockIdx.x - p.id_blocks;
        const int64_t r0 = block / p.groups * 32ll;
        const int32_t c0 = (int32_t)(block % p.groups) * 32;
        {
            const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
            const int32_t at = r0 + lane < p.N ? p.pos[r0 + lane] : -1, c = c0 + 4 * warp;
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
            if (at >= 0 && c < p.d) {
                const float4 *from = reinterpret_cast<const float4 *>(p.sum_h) + (((int64_t)(at / kM) * p.cols + c / p.tn) * (p.tn / 4) + c % p.tn / 4) * kM + at % kM;
                const int64_t step = (int64_t)p.m_room * p.cols * (p.tn / 4) * kM;
#pragma unroll 8
                for (int32_t s = 0; s < p.splits; ++s) {
                    const float4 x = from[s * step];
                    sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
                }
            }
            s_sum[lane][warp] = sum;
        }
        __syncthreads();
        const int i = threadIdx.x >> 3, q = threadIdx.x & 7;
        const int64_t r = r0 + i;
        const int32_t c = c0 + 4 * q;
        if (r < p.N && c < p.d) {
            float4 sum = s_sum[i][q];
            const int32_t at = p.pos[r];
            if (at >= 0) {
                const float rest = p.rest[at];
                const uint2 x = *reinterpret_cast<const uint2 *>(p.w + (int64_t)p.target[at] * p.ld_weight + c);
                auto add = [&](float &to, uint32_t weight) {         // (an infinite weight has made the sum what it is)
                    to = (weight & 0x7FFFFFFFu) == 0x7F800000u ? to : fmaf(rest, __uint_as_float(weight), to);
                };
                add(sum.x, x.x << 16);
                add(sum.y, x.x & 0xFFFF0000u);
                add(sum.z, x.y << 16);
                add(sum.w, x.y & 0xFFFF0000u);
            }
            if (failed) sum.x = sum.y = sum.z = sum.w = __int_as_float(0x7FFFFFFF);
            const __nv_bfloat162 lo = __floats2bfloat162_rn(sum.x, sum.y), hi = __floats2bfloat162_rn(sum.z, sum.w);
            *reinterpret_cast<uint2 *>(p.grad_h + r * p.ld_h + c) = make_uint2(*reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&hi));
        }
    }
    if (failed && p.grad_w)
        for (int64_t v = blockIdx.x; v < p.V; v += gridDim.x)
            for (int32_t c = threadIdx.x; c < p.d; c += kRowsThreads) p.grad_w[v * p.ld_w + c] = nan;
}

// ------------------------------------------------------------------ host side

// bf16 matrix [rows][cols], rows `ld` elements apart; box = 64 columns x box_rows rows, 128-byte swizzle, zeros outside
bool make_map(CUtensorMap *map, const void *base, int64_t rows, int64_t cols, int64_t ld, uint32_t box_rows)
{
    encode_tiled_fn enc = get_encode_tiled();
    if (!enc) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)ld * 2};
    const cuuint32_t box[2] = {64, box_rows};
    const cuuint32_t estr[2] = {1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The sizes that workspace and launches go by.
struct Plan {
    int64_t n_pad;                              // room for rows: whole tiles
    int32_t m_room;
    int32_t tn, n_tiles, per_unit, chunks;      // loss
    int64_t piece; int32_t pieces, splits;      // gradients
    int32_t cols, tn_d;
    bool few, gather;
};
constexpr int64_t kUnits = 8192;                // units of the loss beyond which tiles are joined: bounds the partial results
constexpr int64_t kPieceElements = 128 << 20;   // of G: 256 MB; a boundary between pieces costs some 30 us (4,096 rows: 3,430 us with 128 MB, 3,195 with 512)
constexpr int64_t kSumElements = 64 << 20;      // of all parts of grad H's sums together: 256 MB
constexpr int64_t kMaxSplits = 64, kPairs = 74; // kPairs: of the device that the sizes are meant for
constexpr int64_t kPieceMin = 4096;             // columns of a piece at least

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

Plan make_plan(int32_t N, int32_t V, int32_t d)
{
    Plan q{};
    q.n_pad = std::max<int64_t>(kM, round_up(N, kM));
    q.m_room = (int32_t)(q.n_pad / kM);
    q.gather = N > kM;                          // fewer are one row of tiles, with or without the rows that have no target
    q.tn = kN;
    q.n_tiles = (V + q.tn - 1) / q.tn;
    q.per_unit = (int32_t)std::max<int64_t>(1, (int64_t)q.n_tiles * q.m_room / kUnits);
    q.few = N <= kFewRows;
    q.chunks = q.few ? 4 * kFewCtas : 2 * ((q.n_tiles + q.per_unit - 1) / q.per_unit);
    const int64_t most = std::max(kPieceMin, kPieceElements / q.n_pad / kN * kN);
    q.pieces = (int32_t)((V + most - 1) / most);
    q.piece = round_up((V + q.pieces - 1) / q.pieces, kN);
    q.pieces = (int32_t)((V + q.piece - 1) / q.piece);
    q.tn_d = d >= kN ? kN : 128;
    q.cols = (d + q.tn_d - 1) / q.tn_d;
    // parts of grad H's sums: units of about a sixth of a pair's share of the work, so that the shares come out even (a unit of grad W takes
    // as long as six steps at least, which is what its tile takes to leave)
    const int64_t steps = q.piece / kStepK, work = q.cols * (q.m_room * steps + q.piece / kM * std::max<int64_t>(6, q.n_pad / kStepK));
    const int64_t most_splits = std::min<int64_t>(kMaxSplits, std::max<int64_t>(1, kSumElements / ((int64_t)q.m_room * q.cols * kM * q.tn_d)));
    q.splits = (int32_t)std::min<int64_t>(most_splits, (steps + std::max<int64_t>(16, work / kPairs / 6) - 1) / std::max<int64_t>(16, work / kPairs / 6));
    return q;
}

struct Room {                                   // hands out pieces of the workspace
    uint8_t *base;
    int64_t used;
    template <typename T> T *take(int64_t n)
    {
        T *at = reinterpret_cast<T *>(base + used);
        used += round_up(n * (int64_t)sizeof(T), 256);
        return at;
    }
};
struct ForwardRoom {
    float2 *part; bf16 *h; int32_t *pos, *target, *n_live; uint32_t *failed;
    int64_t bytes;
    ForwardRoom(const Plan &q, int32_t N, int32_t d, void *ws)
    {
        Room r{static_cast<uint8_t *>(ws), 0};
        part = r.take<float2>((int64_t)q.chunks * q.n_pad);
        if (q.gather) { h = r.take<bf16>(q.n_pad * d); pos = r.take<int32_t>(N); target = r.take<int32_t>(q.n_pad); n_live = r.take<int32_t>(1); failed = r.take<uint32_t>(1); }
        else { h = nullptr; pos = target = n_live = nullptr; failed = r.take<uint32_t>(1); }
        bytes = r.used;
    }
};
struct BackwardRoom {
    bf16 *g, *h; float *sum_h, *sum_w, *lse, *coef, *rest, *part_p; int32_t *pos, *target, *n_live, *group_at; uint32_t *failed, *first_row;
    int64_t bytes;
    BackwardRoom(const Plan &q, int32_t N, int32_t V, int32_t d, void *ws)
    {
        Room r{static_cast<uint8_t *>(ws), 0};
        g = r.take<bf16>(q.n_pad * q.piece);
        h = r.take<bf16>(q.n_pad * d);
        sum_h = r.take<float>((int64_t)q.splits * q.m_room * q.cols * kM * q.tn_d);
        lse = r.take<float>(q.n_pad); coef = r.take<float>(q.n_pad); rest = r.take<float>(q.n_pad);
        part_p = r.take<float>(2 * (q.piece / kN) * q.n_pad);
        pos = r.take<int32_t>(N); target = r.take<int32_t>(q.n_pad); n_live = r.take<int32_t>(1); failed = r.take<uint32_t>(1 + (int64_t)q.pieces);
        first_row = r.take<uint32_t>(V);
        group_at = r.take<int32_t>((N + kGroup - 1) / kGroup + 1);
        sum_w = r.take<float>(std::min<int64_t>(q.n_pad, V) * d);
        bytes = r.used;
    }
};

bool aligned(const void *ptr, uintptr_t to) { return ptr && reinterpret_cast<uintptr_t>(ptr) % to == 0; }
bool sizes_ok(int32_t N, int32_t V, int32_t d)
{
    return N >= 0 && N <= TFE_XENT_MAX_ROWS && V >= 1 && V <= TFE_XENT_MAX_ROWS && d >= 8 && d % 8 == 0 && d <= TFE_XENT_MAX_COLS;
}
bool rows_ok(const void *at, int64_t ld, int32_t d) { return aligned(at, 16) && ld >= d && ld % 8 == 0 && ld <= (1ll << 34); }

tfe_status device_sms(int *sms)
{
    int dev = 0;
    tfe_status st = tfe_note_cuda(cudaGetDevice(&dev), "cudaGetDevice");
    return st != TFE_OK ? st : tfe_note_cuda(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev), "cudaDeviceGetAttribute");
}

tfe_status bad_map() { return tfe_note_cuda(cudaErrorInvalidValue, "cuTensorMapEncodeTiled"); }

template <int TN>
tfe_status launch_few(int grid, cudaStream_t stream, const CUtensorMap &w, const CUtensorMap &w_tail, const CUtensorMap &h, const FewParams &p)
{
    constexpr size_t smem = few_stages(TN) * few_stage(TN) + 1024;
    if (tfe_status st = tfe_note_cuda(cudaFuncSetAttribute(tfe_xent_few_kernel<TN>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem), "cross entropy attribute")) return st;
    return tfe_launch_serial(tfe_xent_few_kernel<TN>, (unsigned)grid, kFewThreads, 1, smem, stream, "cross entropy launch", w, w_tail, h, p);
}

template <int kOp>
tfe_status launch_gemm(int64_t most_units, int sms, cudaStream_t stream, const Maps &maps, const GemmParams &p)
{
    auto kernel = tfe_xent_gemm_kernel<kOp>;
    if (kOp == kLse) {                          // the registers that its warps ask for have to be there (they would wait for good)
        cudaFuncAttributes attr;
        if (tfe_status st = tfe_note_cuda(cudaFuncGetAttributes(&attr, kernel), "cross entropy attributes")) return st;
        if (attr.numRegs * kThreads < 128 * kFewRegs + 32 * kEpilogueWarps * kManyRegs) return TFE_ERR_INTERNAL;
    }
    if (tfe_status st = tfe_note_cuda(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem), "cross entropy attribute")) return st;
    const unsigned grid = (unsigned)(std::max<int64_t>(1, std::min<int64_t>(sms / kCtas, most_units)) * kCtas);
    return tfe_launch_serial(kernel, grid, kThreads, kCtas, kSmem, stream, "cross entropy launch", maps, p);
}

tfe_status launch_compact(CompactParams c, int sms, cudaStream_t stream)
{
    const bool ordered = c.first_row != nullptr;
    c.rows_per_block = (int32_t)std::max<int64_t>(8, (c.N + 2ll * sms - 1) / (2ll * sms));
    if (ordered) {                              // a power of two: no block lies in two groups
        int32_t rows = 8;
        while (rows < c.rows_per_block && rows < kGroup) rows *= 2;
        c.rows_per_block = rows;
    }
    const unsigned grid = (unsigned)std::max<int64_t>(64, ((int64_t)c.N + c.rows_per_block - 1) / c.rows_per_block);     // (few rows: zeros to write)
    return tfe_launch_serial(ordered ? tfe_xent_compact_kernel<true> : tfe_xent_compact_kernel<false>, grid, kCompactThreads, 1, 0, stream, "cross entropy rows launch", c);
}

bool touch(const void *a, int64_t a_bytes, const void *b, int64_t b_bytes)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a && b && x < y + (uintptr_t)b_bytes && y < x + (uintptr_t)a_bytes;
}

}  // namespace

extern "C" {

int64_t tfe_xent_forward_workspace_bytes(int32_t N, int32_t V, int32_t d)
{
    if (!sizes_ok(N, V, d)) return -1;
    return N == 0 ? 0 : ForwardRoom(make_plan(N, V, d), N, d, nullptr).bytes;
}

int64_t tfe_xent_backward_workspace_bytes(int32_t N, int32_t V, int32_t d)
{
    if (!sizes_ok(N, V, d)) return -1;
    return N == 0 ? 0 : BackwardRoom(make_plan(N, V, d), N, V, d, nullptr).bytes;
}

tfe_status tfe_xent_forward(const void *hidden, int64_t ld_hidden, int32_t N, const void *weight, int64_t ld_weight, int32_t V, int32_t d,
                            const int32_t *target, float *loss, float *lse, void *workspace, int64_t workspace_bytes, void *stream_)
{
    if (!sizes_ok(N, V, d)) return TFE_ERR_INVALID_ARG;
    if (N == 0) return TFE_OK;
    if (!rows_ok(hidden, ld_hidden, d) || !rows_ok(weight, ld_weight, d) || !aligned(target, 4) || !aligned(loss, 4) || !aligned(lse, 4) ||
        !aligned(workspace, 256))
        return TFE_ERR_INVALID_ARG;
    const Plan q = make_plan(N, V, d);
    const ForwardRoom room(q, N, d, workspace);
    if (workspace_bytes < room.bytes) return TFE_ERR_CAPACITY;
    const struct { const void *at; int64_t bytes; } in[] = {{hidden, ((int64_t)(N - 1) * ld_hidden + d) * 2}, {weight, ((int64_t)(V - 1) * ld_weight + d) * 2},
                                                            {target, 4ll * N}, {workspace, room.bytes}};
    for (const auto &x : in)
        if (touch(x.at, x.bytes, loss, 4ll * N) || touch(x.at, x.bytes, lse, 4ll * N)) return TFE_ERR_INVALID_ARG;
    if (touch(loss, 4ll * N, lse, 4ll * N)) return TFE_ERR_INVALID_ARG;
    for (int i = 0; i < 3; ++i)
        if (touch(in[i].at, in[i].bytes, workspace, room.bytes)) return TFE_ERR_INVALID_ARG;
    int sms = 0;
    if (tfe_status st = device_sms(&sms)) return st;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    LossParams l{};
    l.N = N; l.V = V; l.chunks = q.chunks; l.part = room.part; l.ld_part = q.n_pad; l.target = target; l.pos = room.pos;
    l.loss = loss; l.lse = lse; l.d = d;
    l.h = static_cast<const bf16 *>(hidden); l.ld_h = ld_hidden; l.w = static_cast<const bf16 *>(weight); l.ld_w = ld_weight;
    l.rows = 1;                                 // few rows: a block each
    while (l.rows < kLossRows && N / l.rows >= 2 * sms) l.rows *= 2;
    auto join = [&] { return tfe_launch_serial(tfe_xent_loss_kernel, (unsigned)((N + l.rows - 1) / l.rows), kLossThreads, 1, 0, stream, "cross entropy loss launch", l); };
    if (q.few) {
        FewParams f{};
        f.N = N; f.V = V; f.steps = (d + kStepK - 1) / kStepK;
        const int ctas = std::min(sms, kFewCtas), tn = N <= 16 ? 16 : N <= 32 ? 32 : 64;
        f.rows_per_cta = (V + ctas - 1) / ctas;
        f.rows_per_cta = (f.rows_per_cta + 7) / 8 * 8;
        f.tail_rows = f.rows_per_cta % kFewM;
        f.give_up = g_xent_give_up.load(std::memory_order_relaxed);
        f.target = target; f.part = room.part; f.ld_part = q.n_pad;
        const int grid = (V + f.rows_per_cta - 1) / f.rows_per_cta;
        CUtensorMap w, w_tail, h;
        if (!make_map(&w, weight, V, d, ld_weight, kFewM) || !make_map(&w_tail, weight, V, d, ld_weight, f.tail_rows ? (uint32_t)f.tail_rows : 8u) ||
            !make_map(&h, hidden, N, d, ld_hidden, (uint32_t)tn))
            return bad_map();
        const tfe_status st = tn == 16 ? launch_few<16>(grid, stream, w, w_tail, h, f) : tn == 32 ? launch_few<32>(grid, stream, w, w_tail, h, f) : launch_few<64>(grid, stream, w, w_tail, h, f);
        if (st != TFE_OK) return st;
        l.chunks = 4 * grid;
        return join();
    }
    if (q.gather) {
        CompactParams c{};
        c.N = N; c.V = V; c.d = d; c.h = static_cast<const bf16 *>(hidden); c.ld = ld_hidden; c.target = target;
        c.h_out = room.h; c.pos = room.pos; c.target_out = room.target; c.n_live = room.n_live; c.failed = room.failed;
        if (tfe_status st = launch_compact(c, sms, stream)) return st;
    }
    Maps maps{};
    if (!(q.gather ? make_map(&maps.a, room.h, q.n_pad, d, d, kRowsA) : make_map(&maps.a, hidden, N, d, ld_hidden, kRowsA)) ||
        !make_map(&maps.b, weight, V, d, ld_weight, (uint32_t)(q.tn / kCtas)))
        return bad_map();
    GemmParams p{};
    p.N = N; p.V = V; p.d = d; p.tn = q.tn; p.per_unit = q.per_unit; p.n_tiles = q.n_tiles; p.m_room = q.m_room;
    p.give_up = g_xent_give_up.load(std::memory_order_relaxed);
    p.n_live = room.n_live; p.target = q.gather ? room.target : target;
    p.part = room.part; p.ld_part = q.n_pad; p.failed = room.failed;
    l.failed = room.failed;
    if (!q.gather)                              // (cleared with the rows otherwise)
        if (tfe_status st = tfe_note_cuda(cudaMemsetAsync(room.failed, 0, 4, stream), "cudaMemsetAsync")) return st;
    if (tfe_status st = launch_gemm<kLse>((int64_t)q.m_room * (q.chunks / 2), sms, stream, maps, p)) return st;
    return join();
}

tfe_status tfe_xent_backward(const void *hidden, int64_t ld_hidden, int32_t N, const void *weight, int64_t ld_weight, int32_t V, int32_t d,
                             const int32_t *target, const float *lse, const float *grad_loss, void *grad_hidden, int64_t ld_grad_hidden,
                             void *grad_weight, int64_t ld_grad_weight, void *workspace, int64_t workspace_bytes, void *stream_)
{
    if (!sizes_ok(N, V, d) || (!grad_hidden && !grad_weight)) return TFE_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (grad_weight && !rows_ok(grad_weight, ld_grad_weight, d)) return TFE_ERR_INVALID_ARG;
    if (N == 0) {                               // nothing to sum: zeros
        if (!grad_weight) return TFE_OK;
        return tfe_note_cuda(cudaMemset2DAsync(grad_weight, (size_t)ld_grad_weight * 2, 0, (size_t)d * 2, (size_t)V, stream), "cudaMemset2DAsync");
    }
    if (!rows_ok(hidden, ld_hidden, d) || !rows_ok(weight, ld_weight, d) || !aligned(target, 4) || !aligned(lse, 4) || !aligned(grad_loss, 4) ||
        !aligned(workspace, 256) || (grad_hidden && !rows_ok(grad_hidden, ld_grad_hidden, d)))
        return TFE_ERR_INVALID_ARG;
    const Plan q = make_plan(N, V, d);
    const BackwardRoom room(q, N, V, d, workspace);
    if (workspace_bytes < room.bytes) return TFE_ERR_CAPACITY;
    const int64_t b_h = ((int64_t)(N - 1) * ld_hidden + d) * 2, b_w = ((int64_t)(V - 1) * ld_weight + d) * 2;
    const int64_t b_gh = ((int64_t)(N - 1) * ld_grad_hidden + d) * 2, b_gw = ((int64_t)(V - 1) * ld_grad_weight + d) * 2;
    const struct { const void *at; int64_t bytes; } in[] = {{hidden, b_h}, {weight, b_w}, {target, 4ll * N}, {lse, 4ll * N}, {grad_loss, 4ll * N}, {workspace, room.bytes}};
    for (const auto &x : in)
        if (touch(x.at, x.bytes, grad_hidden, b_gh) || touch(x.at, x.bytes, grad_weight, b_gw)) return TFE_ERR_INVALID_ARG;
    if (touch(grad_hidden, b_gh, grad_weight, b_gw)) return TFE_ERR_INVALID_ARG;
    for (int i = 0; i < 5; ++i)
        if (touch(in[i].at, in[i].bytes, workspace, room.bytes)) return TFE_ERR_INVALID_ARG;
    int sms = 0;
    if (tfe_status st = device_sms(&sms)) return st;
    CompactParams c{};
    c.N = N; c.V = V; c.d = d; c.h = static_cast<const bf16 *>(hidden); c.ld = ld_hidden; c.target = target; c.lse = lse; c.grad = grad_loss;
    c.h_out = room.h; c.pos = room.pos; c.target_out = room.target; c.n_live = room.n_live; c.lse_out = room.lse; c.coef_out = room.coef; c.failed = room.failed;
    c.counters = q.pieces; c.first_row = room.first_row; c.group_at = room.group_at;
    if (tfe_status st = launch_compact(c, sms, stream)) return st;

    // G lies in blocks of 64 columns, one below the other: whichever way a product reads it, a tile is one run of memory
    const int64_t g_rows = q.n_pad * (q.piece / 64);
    Maps probs{}, grads{};
    if (!make_map(&probs.a, room.h, q.n_pad, d, d, kRowsA) || !make_map(&probs.b, weight, V, d, ld_weight, kN / kCtas) ||
        !make_map(&probs.out, room.g, g_rows, 64, 64, 32) || !make_map(&grads.a, room.g, g_rows, 64, 64, kRowsA) ||
        !make_map(&grads.b, weight, V, d, ld_weight, 64) || !make_map(&grads.a_w, room.g, g_rows, 64, 64, 64) ||
        !make_map(&grads.b_w, room.h, q.n_pad, d, d, 64) || (grad_weight && !make_map(&grads.out, grad_weight, V, d, ld_grad_weight, 32)))
        return bad_map();
    GemmParams p{};
    p.N = N; p.V = V; p.d = d; p.n_pad = (int32_t)q.n_pad; p.m_room = q.m_room; p.splits = q.splits;
    p.want_h = grad_hidden != nullptr; p.want_w = grad_weight != nullptr;
    p.give_up = g_xent_give_up.load(std::memory_order_relaxed);
    p.n_live = room.n_live; p.target = room.target; p.lse = room.lse; p.coef = room.coef; p.sum_h = room.sum_h; p.failed = room.failed; p.rest = room.rest; p.first_row = room.first_row; p.part_p = room.part_p; p.ld_p = q.n_pad; p.sum_w = room.sum_w; p.by_id = V <= q.n_pad;
    for (int32_t i = 0; i < q.pieces; ++i) {
        p.v0 = (int32_t)(i * q.piece);
        p.width = (int32_t)std::min<int64_t>(q.piece, V - (int64_t)i * q.piece);
        p.first = i == 0;
        p.tn = kN;
        if (tfe_status st = launch_gemm<kProb>((int64_t)q.m_room * ((p.width + kN - 1) / kN), sms, stream, probs, p)) return st;
        p.tn = q.tn_d;
        p.ticket = room.failed + 1 + i;
        const int64_t most = (int64_t)q.cols * ((int64_t)p.want_h * q.m_room * q.splits + (int64_t)p.want_w * ((p.width + kM - 1) / kM));
        if (tfe_status st = launch_gemm<kGrads>(most, sms, stream, grads, p)) return st;
    }
    RestParams t{};
    t.chunks = 2 * (int32_t)((std::min<int64_t>(q.piece, V) + kN - 1) / kN); t.n_live = room.n_live; t.part_p = room.part_p; t.ld_p = q.n_pad; t.coef = room.coef; t.rest = room.rest;
    if (tfe_status st = tfe_launch_serial(tfe_xent_rest_kernel, (unsigned)((N + 31) / 32), 32 * kRestWarps, 1, 0, stream, "cross entropy targets launch", t)) return st;
    RowsParams r{};
    r.N = N; r.V = V; r.d = d; r.splits = q.splits; r.m_room = q.m_room; r.cols = q.cols; r.tn = q.tn_d; r.sum_h = room.sum_h; r.pos = room.pos;
    r.failed = room.failed; r.rest = room.rest; r.target = room.target; r.w = static_cast<const bf16 *>(weight); r.ld_weight = ld_weight; r.grad_h = static_cast<bf16 *>(grad_hidden); r.ld_h = ld_grad_hidden; r.grad_w = static_cast<bf16 *>(grad_weight); r.ld_w = ld_grad_weight;
    r.h = room.h; r.n_live = room.n_live; r.first_row = room.first_row; r.sum_w = room.sum_w; r.by_id = p.by_id;
    r.groups = (d + 31) / 32;
    r.group_at = room.group_at;
    r.slices = (d + kSlice - 1) / kSlice;
    r.id_blocks = grad_weight ? (N + kSpan - 1) / kSpan * r.slices : 0;
    const unsigned grid = (unsigned)r.id_blocks + (unsigned)(grad_hidden ? (N + 31) / 32 * r.groups : 0);
    return tfe_launch_serial(tfe_xent_rows_kernel, grid, kRowsThreads, 1, 0, stream, "cross entropy gradient launch", r);
}

tfe_status tfe_xent_status(uint32_t *device_flags, void *stream_)
{
    if (!device_flags) return TFE_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    void *at = nullptr;
    if (tfe_status st = tfe_note_cuda(cudaGetSymbolAddress(&at, g_xent_status), "cudaGetSymbolAddress")) return st;
    if (tfe_status st = tfe_note_cuda(cudaMemcpyAsync(device_flags, at, sizeof(uint32_t), cudaMemcpyDeviceToHost, stream), "cudaMemcpyAsync")) return st;
    if (tfe_status st = tfe_note_cuda(cudaStreamSynchronize(stream), "cudaStreamSynchronize")) return st;
    if (*device_flags == 0) return TFE_OK;
    tfe_xent_status_kernel<<<1, 1, 0, stream>>>(*device_flags);
    if (tfe_status st = tfe_note_cuda(cudaGetLastError(), "status launch")) return st;
    if (tfe_status st = tfe_note_cuda(cudaStreamSynchronize(stream), "cudaStreamSynchronize")) return st;
    return TFE_ERR_INTERNAL;
}

tfe_status tfe_xent_give_up(int32_t how)
{
    g_xent_give_up.store(how == 0 ? 0u : how == (int32_t)kUnderWay ? kUnderWay : kAtOnce, std::memory_order_relaxed);
    return TFE_OK;
}

}  // extern "C"

// The vocabulary product with both sides in e4m3 and an fp32 scale for each block of 128 along d: the early-exit head's
// contraction (paper Sec. 4.4) at half the bytes, and the conversion that makes its operands.
//
//   tfe_quantize_rows_kernel     activations: a scale per row and 128 columns.  16 lanes hold a group in registers, so the
//                                input is read once.
//   tfe_quantize_blocks_kernel   weights: a scale per 128 rows and 128 columns; one block holds the 128 x 128 piece.
//   tfe_matmul_fp8_kernel        out[m][n] = sum_b sa[m][b] sb[n / 128][b] (sum over the 128 k of block b of a[m][k] w[n][k])
//
// The products are persistent, warp-specialised tcgen05 kernels.  The scales change every 128 k, so an accumulator in tensor
// memory only ever holds one block's partial sum: the epilogue warps read it, multiply by the two scales and add it to fp32
// sums in registers while the next block's MMAs run into another accumulator.  The sums over blocks are thereby plain fp32
// additions whatever the precision of the tensor core's own accumulation.
//
//   tfe_matmul_fp8_few_kernel    up to 64 activation rows: the read of the weights bounds the call.  The weights' rows are the
//                                MMA's M (128), the activations' its N (16..64), so few rows waste neither tensor memory nor
//                                epilogue work, and a warp's stores of one activation row are contiguous.  The vocabulary is cut
//                                into equal row ranges, one per SM, each walked in tiles of 128.
//   tfe_matmul_fp8_many_kernel   more: the operands' way from L2 and the epilogue bound the call.  The activations' rows are the
//                                MMA's M (128), the weights' its N (256): a thread owns one activation row,
//                                so a block's scale is one number for all its columns.  Finished rows leave by asynchronous
//                                bulk copies while the next tile is summed.
//
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>

#include "../../include/tfe.h"
#include "tfe_internal.h"
#include "tfe_rows.cuh"
#include "tfe_tc.cuh"

namespace {

using tfe_rows::Elem;

// ------------------------------------------------------------------ conversion

constexpr int kQuantThreads = 256;
constexpr int kGroupLanes = 16;                 // lanes that share a group of 128 columns: 8 consecutive elements each

struct QuantParams {
    const void *x; int64_t ld;
    int32_t R, C, kb;                           // kb: groups of 128 columns
    uint8_t *q; int64_t ldq;
    float *scale;
};

__device__ __forceinline__ float scale_of(uint32_t amax_bits)
{
    // the bit pattern orders like the value, NaN above infinity: a block that holds either has that as its scale
    const float amax = __uint_as_float(amax_bits), s = __fdiv_rn(amax, 448.f);
    return amax_bits >= 0x7F800000u ? amax : fmaxf(s, 0x1p-126f);
}
// x / s correctly rounded, for the many x of a block.  Markstein's method: with r = 1 / s correctly rounded and q within one
// unit of x / s, fma(x - q s, r, q) is the correctly rounded quotient (the remainder is exact).  The product x r can be one and
// a half units off, so the step is made twice.  Where the scale's size could cost the remainder bits (or r is not finite) the
// division itself is called.  155 million quotients: the conversion of 151,936 x 1,024 weights takes 278 us with the
// division everywhere.
struct Divisor {
    float s, r;
    bool fast;
    __device__ __forceinline__ float2 two(float a, float b) const
    {
        if (!fast) return make_float2(__fdiv_rn(a, s), __fdiv_rn(b, s));
        const float2 x = make_float2(a, b), rr = make_float2(r, r), minus = make_float2(-s, -s);
        float2 q = __fmul2_rn(x, rr);           // both in one instruction
        q = __ffma2_rn(__ffma2_rn(q, minus, x), rr, q);
        return __ffma2_rn(__ffma2_rn(q, minus, x), rr, q);
    }
    __device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d) const
    {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(two(a, b), __NV_SATFINITE, __NV_E4M3), hi = __nv_cvt_float2_to_fp8x2(two(c, d), __NV_SATFINITE, __NV_E4M3);
        return lo | (hi << 16);
    }
};
__device__ __forceinline__ Divisor divisor(float s) { return {s, __fdiv_rn(1.f, s), s >= 0x1p-90f && s <= 0x1p100f}; }

// Eight elements of a group as they were read: 8 l .. 8 l + 7 for lane l (kVector: whole 16-byte vectors), or l, l + 16, ...;
// zeros beyond the row.
template <typename T>
struct Eight {
    static constexpr int kWords = (int)sizeof(T) * 2;
    uint32_t w[kWords];

    template <bool kVector>
    __device__ __forceinline__ void load(const QuantParams &p, int64_t row, int32_t c0, int l, bool any)
    {
        const T *at = static_cast<const T *>(p.x) + row * p.ld + c0;
        if constexpr (kVector) {
#pragma unroll
            for (int h = 0; h < kWords / 4; ++h) {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (any && c0 + 8 * l < p.C) v = tfe_rows::load_stream(reinterpret_cast<const uint4 *>(at + 8 * l) + h);
                w[4 * h] = v.x; w[4 * h + 1] = v.y; w[4 * h + 2] = v.z; w[4 * h + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool in = any && c0 + l + 16 * e < p.C;
                if constexpr (sizeof(T) == 4) {
                    w[e] = in ? __float_as_uint(at[l + 16 * e]) : 0u;
                } else {
                    const uint32_t x = in ? (uint32_t)__bfloat16_as_ushort(at[l + 16 * e]) : 0u;
                    w[e / 2] = e & 1 ? w[e / 2] | (x << 16) : x;
                }
            }
        }
    }
    __device__ __forceinline__ float get(int e) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
        else return __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
    }
    // the largest magnitude's bit pattern as fp32, NaN above infinity
    __device__ __forceinline__ uint32_t amax() const
    {
        uint32_t m = 0;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < kWords; ++e) m = max(m, w[e] & 0x7FFFFFFFu);
            return m;
        } else {
#pragma unroll
            for (int e = 0; e < kWords; ++e) m = __vmaxu2(m, w[e] & 0x7FFF7FFFu);
            return max(m & 0xFFFF0000u, m << 16);
        }
    }
    template <bool kVector>
    __device__ __forceinline__ void store(const QuantParams &p, int64_t row, int32_t c0, int l, const Divisor &by) const
    {
        uint8_t *at = p.q + row * p.ldq + c0;
        const uint32_t lo = by.to_e4m3x4(get(0), get(1), get(2), get(3)), hi = by.to_e4m3x4(get(4), get(5), get(6), get(7));
        if constexpr (kVector) {
            if (c0 + 8 * l < p.C) *reinterpret_cast<uint2 *>(at + 8 * l) = make_uint2(lo, hi);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c0 + l + 16 * e < p.C) at[l + 16 * e] = (uint8_t)((e < 4 ? lo : hi) >> (8 * (e & 3)));
        }
    }
};

template <typename T, bool kVector>
__global__ void __launch_bounds__(kQuantThreads)
tfe_quantize_rows_kernel(const QuantParams p)
{
    tfe_wait_for_stream();
    const int l = threadIdx.x & (kGroupLanes - 1);
    const uint32_t groups = (uint32_t)p.R * (uint32_t)p.kb;
    const uint32_t g = blockIdx.x * (kQuantThreads / kGroupLanes) + threadIdx.x / kGroupLanes;     // fits 32 bits, the thread's number does not
    if (g >= groups) return;                    // half-warps leave as a whole
    const uint32_t half = 0xFFFFu << (threadIdx.x & 16);
    const uint32_t row = g / (uint32_t)p.kb, b = g - row * (uint32_t)p.kb;
    Eight<T> x;
    x.template load<kVector>(p, row, (int32_t)(b * 128), l, true);
    uint32_t m = x.amax();
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(half, m, o));
    const float s = scale_of(m);
    x.template store<kVector>(p, row, (int32_t)(b * 128), l, divisor(s));
    if (l == 0) p.scale[g] = s;
}

// Four blocks per SM (64 registers) for bf16: 6 % faster than three; 151,936 x 1,024 take 87 us, 81 of them on the device.
template <typename T, bool kVector>
__global__ void __launch_bounds__(kQuantThreads, sizeof(T) == 2 ? 4 : 2)
tfe_quantize_blocks_kernel(const QuantParams p)
{
    constexpr int kRowsAtOnce = kQuantThreads / kGroupLanes, kTurns = 128 / kRowsAtOnce;
    __shared__ uint32_t s_max[kQuantThreads / 32];
    tfe_wait_for_stream();
    const int l = threadIdx.x & (kGroupLanes - 1), hw = threadIdx.x / kGroupLanes;
    const uint32_t rb = blockIdx.x / (uint32_t)p.kb, b = blockIdx.x - rb * (uint32_t)p.kb;
    const int64_t row0 = (int64_t)rb * 128 + hw;
    Eight<T> x[kTurns];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < kTurns; ++i) x[i].template load<kVector>(p, row0 + i * kRowsAtOnce, (int32_t)(b * 128), l, row0 + i * kRowsAtOnce < p.R);
#pragma unroll
    for (int i = 0; i < kTurns; ++i) m = max(m, x[i].amax());
    m = __reduce_max_sync(0xFFFFFFFFu, m);
    if ((threadIdx.x & 31) == 0) s_max[threadIdx.x >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kQuantThreads / 32; ++w) m = max(m, s_max[w]);
    const float s = scale_of(m);
    const Divisor by = divisor(s);
#pragma unroll
    for (int i = 0; i < kTurns; ++i)
        if (row0 + i * kRowsAtOnce < p.R) x[i].template store<kVector>(p, row0 + i * kRowsAtOnce, (int32_t)(b * 128), l, by);
    if (threadIdx.x == 0) p.scale[blockIdx.x] = s;
}

// ------------------------------------------------------------------ product

// Up to here the weights' rows are the MMA's M.  100 x 151,936 x 1,024 to fp32 takes 51.5 us that way (padded to 128 columns)
// and 48.7 us the other, 128 rows to bf16 51.6 and 45.5 us; 64 rows 38.6 and 47.5 us.
constexpr int kFewRows = 64;
constexpr int kTileRows = 128;                  // rows of a tile on that side
constexpr int kBlockK = 128;                    // bytes of a row per stage: one scale block, one 128-byte swizzle row
constexpr int kUmmaK = 32;                      // e4m3 elements per tcgen05.mma
constexpr int kMaxStages = 12;
constexpr int kScaleRing = 4;
// Few rows: scale blocks that are loaded, multiplied and read back together.  A step of the thread that issues the MMAs costs
// about 330 cycles for its waits and commits besides 60 for each MMA, and a block's share of the HBM bandwidth is 630:
// 1 x 151,936 x 1,024 takes 38 us with one block per step, 29 us with four.
__host__ __device__ constexpr int group_blocks(int tn) { return tn <= 32 ? 4 : 2; }
constexpr int kFewEpilogueWarps = 8;            // two per lane quarter of tensor memory, half of its columns each
constexpr int kFewThreads = 32 * (3 + kFewEpilogueWarps);
constexpr int kMatmulSmem = 224 * 1024;         // stages; the rest of an SM's 227 KB is the static arrays

// bits of the device status word
constexpr uint32_t kTimeoutLoader = 1u, kTimeoutMma = 2u, kTimeoutScales = 4u, kTimeoutEpilogue = 8u;
__device__ uint32_t g_matmul_status;
const float not_a_number = __builtin_nanf("");
// For tests: all waits run out at once, or those of who issues the MMAs at the end of its first tile, with copies and MMAs under way.
constexpr uint32_t kAtOnce = 1, kUnderWay = 2;
std::atomic<uint32_t> g_give_up{0};

// Only what the caller has been told goes: a bit that another stream sets meanwhile stays.
__global__ void tfe_matmul_fp8_status_kernel(uint32_t told) { atomicAnd(&g_matmul_status, ~told); }

struct MatmulParams {
    int32_t M, N, kb;                           // activation rows, weight rows, blocks of 128 along k
    int32_t stages;                             // few rows
    int32_t rows_per_cta, tail_rows;            // few rows: weight rows of a CTA, rows of its last short tile
    int32_t m_tiles;                            // many rows: tiles of activation rows
    int64_t n_units;                            // ... and all tiles
    uint32_t give_up;                           // 0, kAtOnce or kUnderWay
    const float *a_scale, *b_scale;             // [M][kb], [ceil(N / 128)][kb]
    void *out; int64_t ldo;
};

// D[tmem] (+)= A[smem] * B[smem]^T, e4m3 inputs, fp32 accumulate; issued by one thread.
__device__ __forceinline__ void umma_e4m3(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        :
        : "r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Instruction descriptor of kind::f8f6f4: D fp32 (bits [4,6) = 1), A and B e4m3 ([7,10) = [10,13) = 0), both K-major,
// N >> 3 at [17,23), M >> 4 at [24,29).
__host__ __device__ constexpr uint32_t umma_idesc_e4m3(uint32_t M, uint32_t N) { return (1u << 4) | ((N >> 3) << 17) | ((M >> 4) << 24); }

template <int TN, typename Out>
__global__ void __launch_bounds__(kFewThreads, 1)
tfe_matmul_fp8_few_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_w_tail,
                      const __grid_constant__ CUtensorMap map_a, const MatmulParams p)
{
    constexpr int kGroup = group_blocks(TN);            // scale blocks that every role takes at a time
    constexpr int kBuffers = 4;                         // sets of kGroup accumulators of TN columns
    constexpr uint32_t kTmemCols = kBuffers * kGroup * TN;      // 256 or 512
    constexpr int kEpilogueWarps = kFewEpilogueWarps, kCols = TN / 2;   // columns of an epilogue warp
    constexpr uint32_t kBlockBytes = kTileRows * 128u + TN * 128u, kStageBytes = kGroup * kBlockBytes;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t s_full[kMaxStages], s_empty[kMaxStages], s_acc_full[kBuffers], s_acc_empty[kBuffers];
    __shared__ __align__(8) uint64_t s_sc_full[kScaleRing], s_sc_empty[kScaleRing], s_drain;
    __shared__ __align__(16) float s_scale[kScaleRing][kGroup][TN];
    __shared__ uint32_t s_tmem_base;
    __shared__ volatile uint32_t s_abort, s_issued;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) { mbar_init(smem_u32(&s_full[s]), 1); mbar_init(smem_u32(&s_empty[s]), 1); }
        for (int a = 0; a < kBuffers; ++a) { mbar_init(smem_u32(&s_acc_full[a]), 1); mbar_init(smem_u32(&s_acc_empty[a]), kEpilogueWarps); }
        for (int a = 0; a < kScaleRing; ++a) { mbar_init(smem_u32(&s_sc_full[a]), 32); mbar_init(smem_u32(&s_sc_empty[a]), kEpilogueWarps); }
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
    // this CTA's weight rows, and its tiles of them
    const int64_t r0 = (int64_t)blockIdx.x * p.rows_per_cta;
    const int32_t n_rows = (int32_t)min((int64_t)p.rows_per_cta, p.N - r0), n_tiles = (n_rows + kTileRows - 1) / kTileRows;

    if (warp == 0) {
        // ============================ TMA producer ============================
        if (lane == 0) {
            const uint64_t hint_w = 0x12F0000000000000ull;          // evict first: the weights are read once
            const uint64_t hint_a = 0x14F0000000000000ull;          // evict last: the activations are read by every tile
            uint32_t stage = 0, phase = 0, issued = 0;
            bool ok = p.give_up != kAtOnce;
            for (int32_t t = 0; ok && t < n_tiles; ++t) {
                const int32_t valid = min(kTileRows, n_rows - t * kTileRows);
                // a short last tile is fetched with the short box: only its rows are read
                const bool tail = valid < kTileRows && valid == p.tail_rows;
                const uint32_t w_bytes = tail ? (uint32_t)p.tail_rows * 128u : kTileRows * 128u;
                for (int32_t kb = 0; kb < p.kb; kb += kGroup) {
                    if (!mbar_wait(smem_u32(&s_empty[stage]), phase ^ 1u, &s_abort)) {
                        atomicOr(&g_matmul_status, kTimeoutLoader);
                        s_abort = 1;
                        ok = false;
                        break;
                    }
                    const uint32_t bar = smem_u32(&s_full[stage]), dst = smem_base + stage * kStageBytes;
                    const int32_t blocks = min(kGroup, p.kb - kb);
                    mbar_expect_tx(bar, (uint32_t)blocks * (w_bytes + TN * 128u));
                    for (int32_t g = 0; g < blocks; ++g) {
                        tma_load_2d(dst + g * kBlockBytes, tail ? &map_w_tail : &map_w, bar, (kb + g) * kBlockK, (int32_t)(r0 + (int64_t)t * kTileRows), hint_w);
                        tma_load_2d(dst + g * kBlockBytes + kTileRows * 128u, &map_a, bar, (kb + g) * kBlockK, 0, hint_a);
                    }
                    ++issued;
                    if (++stage == (uint32_t)p.stages) { stage = 0; phase ^= 1u; }
                }
            }
            s_issued = issued;
        }
    } else if (warp == 1) {
        // ============================ MMA issuer ==============================
        if (lane == 0) {
            constexpr uint32_t idesc = umma_idesc_e4m3(kTileRows, TN);
            uint32_t stage = 0, phase = 0, buf = 0, buf_phase = 0;
            bool ok = p.give_up != kAtOnce;
            for (int32_t t = 0; ok && t < n_tiles; ++t) {
                for (int32_t kb = 0; kb < p.kb; kb += kGroup) {
                    if (!mbar_wait(smem_u32(&s_acc_empty[buf]), buf_phase ^ 1u, &s_abort) ||
                        !mbar_wait(smem_u32(&s_full[stage]), phase, &s_abort)) {
                        atomicOr(&g_matmul_status, kTimeoutMma);
                        s_abort = 1;
                        ok = false;
                        break;
                    }
                    tc_fence_after();
#pragma unroll
                    for (int g = 0; g < kGroup; ++g) {
                        if (g > 0 && kb + g >= p.kb) break;
                        const uint32_t w_addr = smem_base + stage * kStageBytes + g * kBlockBytes;
                        const uint64_t w_desc = umma_desc_sw128(w_addr), a_desc = umma_desc_sw128(w_addr + kTileRows * 128u);
#pragma unroll
                        for (int k = 0; k < kBlockK / kUmmaK; ++k)  // 32 bytes further along the swizzled row: +2 in the address field
                            umma_e4m3(tmem_base + (buf * kGroup + g) * TN, w_desc + (uint64_t)(2 * k), a_desc + (uint64_t)(2 * k), idesc, k > 0 ? 1u : 0u);
                    }
                    umma_commit(smem_u32(&s_empty[stage]));
                    umma_commit(smem_u32(&s_acc_full[buf]));
                    if (++stage == (uint32_t)p.stages) { stage = 0; phase ^= 1u; }
                    if (++buf == kBuffers) { buf = 0; buf_phase ^= 1u; }
                }
                if (ok && p.give_up == kUnderWay) {
                    atomicOr(&g_matmul_status, kTimeoutMma);
                    s_abort = 1;
                    ok = false;
                }
            }
        }
    } else if (warp == 2) {
        // ============================ activation scales =======================
        uint32_t st = 0, phase = 0;
        bool ok = p.give_up != kAtOnce;
        for (int32_t t = 0; ok && t < n_tiles; ++t) {
            for (int32_t kb = 0; kb < p.kb; kb += kGroup) {
                constexpr int kPer = (TN + 31) / 32;
                float v[kGroup][kPer];
#pragma unroll
                for (int g = 0; g < kGroup; ++g)
#pragma unroll
                    for (int c = 0; c < kPer; ++c)
                        v[g][c] = c * 32 + lane < p.M && kb + g < p.kb ? __ldg(p.a_scale + (int64_t)(c * 32 + lane) * p.kb + kb + g) : 0.f;
                ok = mbar_wait(smem_u32(&s_sc_empty[st]), phase ^ 1u, &s_abort);
                if (!__all_sync(0xFFFFFFFFu, ok)) {
                    if (lane == 0) atomicOr(&g_matmul_status, kTimeoutScales);
                    s_abort = 1;
                    ok = false;
                    break;
                }
#pragma unroll
                for (int g = 0; g < kGroup; ++g)
#pragma unroll
                    for (int c = 0; c < kPer; ++c)
                        if (c * 32 + lane < TN) s_scale[st][g][c * 32 + lane] = v[g][c];
                mbar_arrive(smem_u32(&s_sc_full[st]));
                if (++st == kScaleRing) { st = 0; phase ^= 1u; }
            }
        }
    } else {
        // ============================ epilogue ================================
        const uint32_t quarter = (uint32_t)warp & 3u;               // tensor-memory lanes 32 * quarter .. + 31
        const int32_t c0 = ((warp - 3) >> 2) * kCols;               // this warp's columns
        const int32_t row_in_tile = (int32_t)(quarter * 32u) + lane;
        uint32_t st = 0, phase = 0, buf = 0, buf_phase = 0;
        bool ok = p.give_up != kAtOnce;
        if (!ok && lane == 0) atomicOr(&g_matmul_status, kTimeoutEpilogue);
        int32_t t = 0;
        for (; ok && t < n_tiles; ++t) {
            const int64_t n0 = r0 + (int64_t)t * kTileRows;
            const int32_t valid = min(kTileRows, n_rows - t * kTileRows);
            float2 acc[kCols / 2];
#pragma unroll
            for (int j = 0; j < kCols / 2; ++j) acc[j] = make_float2(0.f, 0.f);
            const float *sb_row = p.b_scale + (row_in_tile < valid ? (n0 + row_in_tile) / 128 : n0 / 128) * p.kb;
            float sb_next[kGroup];                                  // loaded a group ahead
            auto fetch = [&](int32_t kb) {
#pragma unroll
                for (int g = 0; g < kGroup; ++g) sb_next[g] = kb + g < p.kb ? __ldg(sb_row + kb + g) : 0.f;
            };
            fetch(0);
            for (int32_t kb = 0; kb < p.kb; kb += kGroup) {
                float sb[kGroup];
#pragma unroll
                for (int g = 0; g < kGroup; ++g) sb[g] = sb_next[g];
                fetch(kb + kGroup);
                ok = mbar_wait(smem_u32(&s_sc_full[st]), phase, &s_abort) && mbar_wait(smem_u32(&s_acc_full[buf]), buf_phase, &s_abort);
                if (!__all_sync(0xFFFFFFFFu, ok)) {
                    if (lane == 0) atomicOr(&g_matmul_status, kTimeoutEpilogue);
                    s_abort = 1;
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint32_t taddr = tmem_base + ((quarter * 32u) << 16) + buf * kGroup * TN + (uint32_t)c0;
                uint32_t v[kGroup][kCols];                          // all of the group's reads under way together
#pragma unroll
                for (int g = 0; g < kGroup; ++g) {
                    if (g > 0 && kb + g >= p.kb) break;
                    if constexpr (kCols == 32) tmem_ld32(taddr + (uint32_t)(g * TN), v[g]);
                    else if constexpr (kCols == 16) tmem_ld16(taddr + (uint32_t)(g * TN), v[g]);
                    else tmem_ld8(taddr + (uint32_t)(g * TN), v[g]);
                }
                tmem_ld_wait();
#pragma unroll
                for (int g = 0; g < kGroup; ++g) {
                    if (g > 0 && kb + g >= p.kb) break;
                    const float2 s2 = make_float2(sb[g], sb[g]);
#pragma unroll
                    for (int j = 0; j < kCols; j += 4) {
                        const float4 sa = *reinterpret_cast<const float4 *>(&s_scale[st][g][c0 + j]);
                        const float2 lo = __fmul2_rn(make_float2(sa.x, sa.y), s2), hi = __fmul2_rn(make_float2(sa.z, sa.w), s2);
                        acc[j / 2] = __ffma2_rn(make_float2(__uint_as_float(v[g][j]), __uint_as_float(v[g][j + 1])), lo, acc[j / 2]);
                        acc[j / 2 + 1] = __ffma2_rn(make_float2(__uint_as_float(v[g][j + 2]), __uint_as_float(v[g][j + 3])), hi, acc[j / 2 + 1]);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) { mbar_arrive(smem_u32(&s_acc_empty[buf])); mbar_arrive(smem_u32(&s_sc_empty[st])); }
                if (++st == kScaleRing) { st = 0; phase ^= 1u; }
                if (++buf == kBuffers) { buf = 0; buf_phase ^= 1u; }
            }
            if (!ok) break;
            if (row_in_tile < valid) {
                Out *at = static_cast<Out *>(p.out) + (int64_t)c0 * p.ldo + n0 + row_in_tile;
                const int32_t left = p.M - c0;
#pragma unroll
                for (int j = 0; j < kCols; ++j) {
                    if (j < left) Elem<Out>::put(at, j & 1 ? acc[j / 2].y : acc[j / 2].x);
                    at += p.ldo;
                }
            }
        }
#pragma unroll 1
        for (; t < n_tiles; ++t)                                    // a wait ran out: no results, and none that look like some
            if (t * kTileRows + row_in_tile < n_rows)
#pragma unroll 1
                for (int32_t j = c0; j < min(c0 + kCols, p.M); ++j)
                    Elem<Out>::put(static_cast<Out *>(p.out) + (int64_t)j * p.ldo + r0 + (int64_t)t * kTileRows + row_in_tile, not_a_number);
    }

    tc_fence_before();
    __syncthreads();
    if (s_abort) {                              // copies and MMAs in flight end before their memory goes, whoever gave up
        if (warp == 0 && lane == 0)
            for (uint32_t s = 0; s < (uint32_t)p.stages; ++s) {
                const uint32_t fills = (s_issued + (uint32_t)p.stages - 1u - s) / (uint32_t)p.stages;
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

// ------------------------------------------------------------------ product, many activation rows

constexpr int kManyEpilogueWarps = 8;           // two per lane quarter, half of the tile's columns each
constexpr int kManyThreads = 32 * (4 + kManyEpilogueWarps);
// Registers per thread: the first four warps give most of theirs to the epilogue's.  The sum, 128 x 40 + 256 x 216, must not
// exceed what the block is launched with (384 x 168); the host checks that before the launch.
constexpr int kManyFewRegs = 40, kManyManyRegs = 216;
constexpr int kRowWords = 64;                   // 32-bit words of a thread's part of a row: 128 bf16 or 64 fp32
constexpr int kRowPitch = 4 * kRowWords + 16;   // bytes between the rows of an epilogue warp's outgoing area: 16-byte writes without conflicts

constexpr int kManyN = 256;                     // weight rows of a tile (MMA N)
constexpr int kManyCols = kManyN / 2;           // columns of an epilogue warp: one scale block of the weights
constexpr int kManyStages = 3;
constexpr uint32_t kManyStageBytes = kTileRows * 128u + kManyN * 128u;
constexpr size_t kManySmem = 1024 + (size_t)kManyStages * kManyStageBytes + (size_t)kManyEpilogueWarps * 32 * kRowPitch;

__device__ __forceinline__ void bulk_store(void *to, uint32_t from_smem, uint32_t bytes)
{
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(to), "r"(from_smem), "r"(bytes) : "memory");
}

// Part of a thread's finished output row, kCols columns in registers, to `at`.  The 16-byte blocks of the output that it covers
// whole go through the thread's own row in shared memory and an asynchronous bulk copy, which leaves the load/store path to
// others; the words are first shifted (by registers: the distance to a boundary is the thread's own) so that both sides are
// aligned.  What is left at the two ends, up to 15 bytes each, is stored directly in pieces of 2, 4 and 8 bytes.  `cols` of the
// columns exist.
template <typename Out, int kCols>
__device__ __forceinline__ void send_row(Out *at, const float2 *acc, int32_t cols, uint32_t row_smem)
{
    static_assert(kCols * sizeof(Out) == kRowWords * 4, "the columns fill the row");
    constexpr int E = 16 / (int)sizeof(Out);                                    // elements per 16 bytes
    const uint32_t past = (uint32_t)(reinterpret_cast<uintptr_t>(at) & 15u) / (uint32_t)sizeof(Out);
    const int32_t head = past ? E - (int32_t)past : 0, tail = (int32_t)past;    // (kCols is a multiple of E)
    auto element = [&](int i) { return i & 1 ? acc[i / 2].y : acc[i / 2].x; };
    if (cols < kCols) {                                                         // the last columns of the matrix
#pragma unroll
        for (int i = 0; i < kCols; ++i)
            if (i < cols) Elem<Out>::put(at + i, element(i));
        return;
    }
    const bool odd = sizeof(Out) == 2 && (head & 1);
    // word j of the part from its first 4-byte boundary on: one fp32, or two bf16 (elements 2 j + 1 and 2 j + 2 if odd)
    auto word = [&](int j) -> uint32_t {
        if (j >= kRowWords) return 0u;
        if constexpr (sizeof(Out) == 4) {
            return __float_as_uint(element(j));
        } else {
            const float second = j + 1 < kRowWords ? element((2 * j + 2) % kCols) : 0.f;
            const __nv_bfloat162 h = __floats2bfloat162_rn(odd ? element(2 * j + 1) : element(2 * j), odd ? second : element(2 * j + 1));
            return *reinterpret_cast<const uint32_t *>(&h);
        }
    };
    if constexpr (sizeof(Out) == 4) {
        if (head & 1) *reinterpret_cast<uint32_t *>(at) = word(0);
        if (head & 2) *reinterpret_cast<uint2 *>(at + (head & 1)) = head & 1 ? make_uint2(word(1), word(2)) : make_uint2(word(0), word(1));
    } else {
        if (odd) Elem<Out>::put(at, element(0));
        if (head & 2) *reinterpret_cast<uint32_t *>(at + (head & 1)) = word(0);
        if (head & 4) *reinterpret_cast<uint2 *>(at + (head & 3)) = head & 2 ? make_uint2(word(1), word(2)) : make_uint2(word(0), word(1));
    }
    const int32_t shift = head * (int32_t)sizeof(Out) / 4;                      // 0..3 words
    uint32_t w[4];                                                              // four words at a time: few registers beside the sums
#pragma unroll
    for (int c = 0; c < kRowWords; c += 4) {
        uint32_t v[6];
#pragma unroll
        for (int i = 0; i < 6; ++i) v[i] = shift & 1 ? word(c + i + 1) : word(c + i);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = shift & 2 ? v[i + 2] : v[i];
        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(row_smem + 4 * c), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    bulk_store(at + head, row_smem, past ? 4 * kRowWords - 16 : 4 * kRowWords);
    // the tail starts on a 16-byte boundary, with the last four words
    Out *end = at + kCols - tail;
    if constexpr (sizeof(Out) == 4) {
        if (tail & 2) *reinterpret_cast<uint2 *>(end) = make_uint2(w[0], w[1]);
        if (tail & 1) *reinterpret_cast<uint32_t *>(end + (tail & 2)) = tail & 2 ? w[2] : w[0];
    } else {
        if (tail & 4) *reinterpret_cast<uint2 *>(end) = make_uint2(w[0], w[1]);
        if (tail & 2) *reinterpret_cast<uint32_t *>(end + (tail & 4)) = tail & 4 ? w[2] : w[0];
        if (tail & 1) {
            const uint32_t lo = tail & 2 ? w[1] : w[0], hi = tail & 2 ? w[3] : w[2];
            end[tail - 1] = __ushort_as_bfloat16((unsigned short)(tail & 4 ? hi : lo));
        }
    }
}

template <typename Out>
__global__ void __launch_bounds__(kManyThreads, 1)
tfe_matmul_fp8_many_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_a, const MatmulParams p)
{
    constexpr int kStages = kManyStages, kN = kManyN, kCols = kManyCols, kBuffers = 512 / kN;
    constexpr int kRounds = kCols * (int)sizeof(Out) / (4 * kRowWords);         // outgoing rows full of a thread's columns
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t s_full[kStages], s_empty[kStages], s_acc_full[kBuffers], s_acc_empty[kBuffers], s_drain;
    __shared__ uint32_t s_tmem_base;
    __shared__ volatile uint32_t s_abort, s_issued;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) { mbar_init(smem_u32(&s_full[s]), 1); mbar_init(smem_u32(&s_empty[s]), 1); }
        for (int a = 0; a < kBuffers; ++a) { mbar_init(smem_u32(&s_acc_full[a]), 1); mbar_init(smem_u32(&s_acc_empty[a]), kManyEpilogueWarps); }
        mbar_init(smem_u32(&s_drain), 1);
        s_abort = s_issued = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(smem_u32(&s_tmem_base), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = s_tmem_base;
    tfe_wait_for_stream();

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kManyFewRegs));
        if (warp == 0 && lane == 0) {
            // ============================ TMA producer ============================
            const uint64_t hint = 0x14F0000000000000ull;            // evict last: both operands are read by other tiles too
            uint32_t stage = 0, phase = 0, issued = 0;
            bool ok = p.give_up != kAtOnce;
            for (int64_t u = blockIdx.x; ok && u < p.n_units; u += gridDim.x) {
                const int64_t nt = u / p.m_tiles;
                const int32_t n0 = (int32_t)(nt * kN), m0 = (int32_t)(u - nt * p.m_tiles) * kTileRows;
                for (int32_t kb = 0; kb < p.kb; ++kb) {
                    if (!mbar_wait(smem_u32(&s_empty[stage]), phase ^ 1u, &s_abort)) {
                        atomicOr(&g_matmul_status, kTimeoutLoader);
                        s_abort = 1;
                        ok = false;
                        break;
                    }
                    const uint32_t bar = smem_u32(&s_full[stage]), dst = smem_base + stage * kManyStageBytes;
                    mbar_expect_tx(bar, kManyStageBytes);
                    tma_load_2d(dst, &map_a, bar, kb * kBlockK, m0, hint);
                    tma_load_2d(dst + kTileRows * 128u, &map_w, bar, kb * kBlockK, n0, hint);
                    ++issued;
                    if (++stage == kStages) { stage = 0; phase ^= 1u; }
                }
            }
            s_issued = issued;
        } else if (warp == 1 && lane == 0) {
            // ============================ MMA issuer ==============================
            constexpr uint32_t idesc = umma_idesc_e4m3(kTileRows, kN);
            uint32_t stage = 0, phase = 0, buf = 0, buf_phase = 0;
            bool ok = p.give_up != kAtOnce;
            for (int64_t u = blockIdx.x; ok && u < p.n_units; u += gridDim.x) {
                for (int32_t kb = 0; kb < p.kb; ++kb) {
                    if (!mbar_wait(smem_u32(&s_acc_empty[buf]), buf_phase ^ 1u, &s_abort) ||
                        !mbar_wait(smem_u32(&s_full[stage]), phase, &s_abort)) {
                        atomicOr(&g_matmul_status, kTimeoutMma);
                        s_abort = 1;
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t a_addr = smem_base + stage * kManyStageBytes;
                    const uint64_t a_desc = umma_desc_sw128(a_addr), w_desc = umma_desc_sw128(a_addr + kTileRows * 128u);
#pragma unroll
                    for (int k = 0; k < kBlockK / kUmmaK; ++k)
                        umma_e4m3(tmem_base + buf * kN, a_desc + (uint64_t)(2 * k), w_desc + (uint64_t)(2 * k), idesc, k > 0 ? 1u : 0u);
                    umma_commit(smem_u32(&s_empty[stage]));
                    umma_commit(smem_u32(&s_acc_full[buf]));
                    if (++stage == kStages) { stage = 0; phase ^= 1u; }
                    if (++buf == kBuffers) { buf = 0; buf_phase ^= 1u; }
                }
                if (ok && p.give_up == kUnderWay) {
                    atomicOr(&g_matmul_status, kTimeoutMma);
                    s_abort = 1;
                    ok = false;
                }
            }
        }
        tc_fence_before();
        __syncthreads();
        if (s_abort) {                          // copies and MMAs in flight end before their memory goes, whoever gave up
            if (warp == 0 && lane == 0)
                for (uint32_t s = 0; s < kStages; ++s) {
                    const uint32_t fills = (s_issued + kStages - 1u - s) / kStages;
                    for (uint32_t t = 0; fills && t < TC_WAIT_LIMIT && !mbar_try_wait(smem_u32(&s_full[s]), (fills - 1u) & 1u); ++t) { }
                }
            if (warp == 1 && lane == 0) {
                umma_commit(smem_u32(&s_drain));
                for (uint32_t t = 0; t < TC_WAIT_LIMIT && !mbar_try_wait(smem_u32(&s_drain), 0); ++t) { }
            }
            __syncwarp();
        }
    } else {
        // ============================ epilogue ================================
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kManyManyRegs));
        const int e = warp - 4;
        const uint32_t quarter = (uint32_t)warp & 3u;               // tensor-memory lanes 32 * quarter .. + 31
        const int32_t c0 = (e >> 2) * kCols;                        // this warp's columns, all in one scale block of the weights
        const uint32_t row_smem = smem_base + kStages * kManyStageBytes + (uint32_t)((e * 32 + lane) * kRowPitch);
        uint32_t buf = 0, buf_phase = 0;
        bool ok = p.give_up != kAtOnce;
        if (!ok && lane == 0) atomicOr(&g_matmul_status, kTimeoutEpilogue);
        int64_t u = blockIdx.x;
        for (; ok && u < p.n_units; u += gridDim.x) {
            const int64_t nt = u / p.m_tiles;
            const int64_t n0 = nt * kN + c0;
            const int32_t m0 = (int32_t)(u - nt * p.m_tiles) * kTileRows + (int32_t)quarter * 32;
            const float *sa_row = p.a_scale + (int64_t)min(m0 + lane, p.M - 1) * p.kb;
            const float *sb_row = p.b_scale + min(n0, (int64_t)p.N - 1) / 128 * p.kb;
            float2 acc[kCols / 2];
#pragma unroll
            for (int j = 0; j < kCols / 2; ++j) acc[j] = make_float2(0.f, 0.f);
            // Scales of four blocks at a time, loaded while the four before are used (a register that waits for a load stalls even
            // a move, so they are touched only then).
            float scales[4], sa[4], sb[4];
            auto fetch = [&](int32_t kb) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sa[i] = kb + i < p.kb ? __ldg(sa_row + kb + i) : 0.f;
                    sb[i] = kb + i < p.kb ? __ldg(sb_row + kb + i) : 0.f;
                }
            };
            fetch(0);
            for (int32_t kb = 0; kb < p.kb; ++kb) {
                if ((kb & 3) == 0) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) scales[i] = sa[i] * sb[i];
                    fetch(kb + 4);
                }
                const float2 scale = make_float2(scales[0], scales[0]);
                scales[0] = scales[1]; scales[1] = scales[2]; scales[2] = scales[3];
                ok = mbar_wait(smem_u32(&s_acc_full[buf]), buf_phase, &s_abort);
                if (!__all_sync(0xFFFFFFFFu, ok)) {
                    if (lane == 0) atomicOr(&g_matmul_status, kTimeoutEpilogue);
                    s_abort = 1;
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint32_t taddr = tmem_base + ((quarter * 32u) << 16) + buf * kN + (uint32_t)c0;
#pragma unroll
                for (int c = 0; c < kCols; c += 16) {
                    uint32_t v[16];
                    tmem_ld16(taddr + (uint32_t)c, v);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 16; j += 2)
                        acc[(c + j) / 2] = __ffma2_rn(make_float2(__uint_as_float(v[j]), __uint_as_float(v[j + 1])), scale, acc[(c + j) / 2]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&s_acc_empty[buf]));
                if (++buf == kBuffers) { buf = 0; buf_phase ^= 1u; }
            }
            if (!ok) break;
            const int64_t left = (int64_t)p.N - n0;
#pragma unroll
            for (int round = 0; round < kRounds; ++round) {
                constexpr int kPart = kCols / kRounds;
                asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");  // this thread's last row has left its place
                if (left > round * kPart && m0 + lane < p.M)
                    send_row<Out, kPart>(static_cast<Out *>(p.out) + (int64_t)(m0 + lane) * p.ldo + n0 + round * kPart, acc + round * (kPart / 2),
                                         (int32_t)min((int64_t)kPart, left - round * kPart), row_smem);
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            }
        }
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
#pragma unroll 1
        for (; u < p.n_units; u += gridDim.x) {                     // a wait ran out: no results, and none that look like some
            const int64_t nt = u / p.m_tiles, n0 = nt * kN + c0, m = (u - nt * p.m_tiles) * kTileRows + quarter * 32u + lane;
            if (m < p.M)
#pragma unroll 1
                for (int64_t n = n0; n < min(n0 + kCols, (int64_t)p.N); ++n) Elem<Out>::put(static_cast<Out *>(p.out) + m * p.ldo + n, not_a_number);
        }
        tc_fence_before();
        __syncthreads();                        // (as the others)
    }
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tmem_base, 512);
    }
}

// ------------------------------------------------------------------ host side

// e4m3 matrix [rows][cols], rows `ld` bytes apart; box = 128 columns x box_rows rows, 128-byte swizzle, zeros outside
bool make_map_fp8(CUtensorMap *map, const void *base, int64_t rows, int64_t cols, int64_t ld, uint32_t box_rows)
{
    encode_tiled_fn enc = get_encode_tiled();
    if (!enc) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)ld};
    const cuuint32_t box[2] = {(cuuint32_t)kBlockK, box_rows};
    const cuuint32_t estr[2] = {1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int TN, typename Out>
tfe_status launch_few(int grid, cudaStream_t stream, const CUtensorMap &w, const CUtensorMap &w_tail, const CUtensorMap &a, MatmulParams p)
{
    constexpr size_t stage = (size_t)group_blocks(TN) * (kTileRows * 128 + TN * 128);
    p.stages = (int32_t)std::min<size_t>(kMaxStages, (kMatmulSmem - 1024) / stage);
    auto kernel = tfe_matmul_fp8_few_kernel<TN, Out>;
    const size_t smem = (size_t)p.stages * stage + 1024;
    if (tfe_status st = tfe_note_cuda(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem), "product attribute")) return st;
    return tfe_launch_serial(kernel, (unsigned)grid, kFewThreads, 1, smem, stream, "product launch", w, w_tail, a, p);
}

template <int TN>
tfe_status launch_few(int32_t out_dtype, int grid, cudaStream_t stream, const CUtensorMap &w, const CUtensorMap &w_tail, const CUtensorMap &a,
                      const MatmulParams &p)
{
    return out_dtype == TFE_DTYPE_BF16 ? launch_few<TN, __nv_bfloat16>(grid, stream, w, w_tail, a, p) : launch_few<TN, float>(grid, stream, w, w_tail, a, p);
}

template <typename Out>
tfe_status launch_many(int sms, cudaStream_t stream, const void *w, int64_t ldw, const void *a, int64_t lda, int32_t K, MatmulParams p)
{
    auto kernel = tfe_matmul_fp8_many_kernel<Out>;
    // the registers that its warps ask for have to be there (they would wait for good)
    cudaFuncAttributes attr;
    if (tfe_status st = tfe_note_cuda(cudaFuncGetAttributes(&attr, kernel), "product attributes")) return st;
    if (attr.numRegs * kManyThreads < 128 * kManyFewRegs + 32 * kManyEpilogueWarps * kManyManyRegs) return TFE_ERR_INTERNAL;
    if (tfe_status st = tfe_note_cuda(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kManySmem), "product attribute")) return st;
    p.m_tiles = (p.M + kTileRows - 1) / kTileRows;
    p.n_units = ((int64_t)p.N + kManyN - 1) / kManyN * p.m_tiles;
    CUtensorMap map_w, map_a;
    if (!make_map_fp8(&map_w, w, p.N, K, ldw, kManyN) || !make_map_fp8(&map_a, a, p.M, K, lda, kTileRows))
        return tfe_note_cuda(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
    return tfe_launch_serial(kernel, (unsigned)std::min<int64_t>(sms, p.n_units), kManyThreads, 1, kManySmem, stream, "product launch", map_w, map_a, p);
}

bool aligned(const void *ptr, uintptr_t to) { return ptr && reinterpret_cast<uintptr_t>(ptr) % to == 0; }

}  // namespace

extern "C" {

tfe_status tfe_quantize_fp8(const void *x, int32_t dtype, int32_t R, int32_t C, int64_t ld, int32_t block_rows, void *q, float *scale, void *stream)
{
    return tfe_quantize_fp8_ld(x, dtype, R, C, ld, block_rows, q, C, scale, stream);
}

tfe_status tfe_quantize_fp8_ld(const void *x, int32_t dtype, int32_t R, int32_t C, int64_t ld, int32_t block_rows, void *q, int64_t ldq, float *scale,
                               void *stream_)
{
    if (dtype != TFE_DTYPE_BF16 && dtype != TFE_DTYPE_F32) return TFE_ERR_INVALID_ARG;
    if (block_rows != 1 && block_rows != 128) return TFE_ERR_INVALID_ARG;
    if (R < 0 || C < 1 || C > TFE_FP8_MAX_COLS || ld < C || ld > (1ll << 34) || ldq < C || ldq > (1ll << 34)) return TFE_ERR_INVALID_ARG;
    QuantParams p{};
    p.kb = (C + 127) / 128;
    const int64_t groups = ((int64_t)R + block_rows - 1) / block_rows * p.kb;
    if (groups > 0x7FFFFFFFll) return TFE_ERR_INVALID_ARG;
    if (R == 0) return TFE_OK;
    const int es = dtype == TFE_DTYPE_BF16 ? 2 : 4;
    if (!aligned(x, es) || !q || !aligned(scale, 4)) return TFE_ERR_INVALID_ARG;
    p.x = x; p.ld = ld; p.R = R; p.C = C; p.q = static_cast<uint8_t *>(q); p.ldq = ldq; p.scale = scale;
    // 16-byte loads and 8-byte stores where every row starts on such a boundary
    const bool vec = aligned(x, 16) && ld * es % 16 == 0 && C % 8 == 0 && aligned(q, 8) && ldq % 8 == 0;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const unsigned grid = block_rows == 1 ? (unsigned)((groups * kGroupLanes + kQuantThreads - 1) / kQuantThreads) : (unsigned)groups;
    auto go = [&](auto rows_kernel, auto blocks_kernel) {
        return tfe_launch_serial(block_rows == 1 ? rows_kernel : blocks_kernel, grid, kQuantThreads, 1, 0, stream, "conversion launch", p);
    };
    if (dtype == TFE_DTYPE_BF16)
        return vec ? go(tfe_quantize_rows_kernel<__nv_bfloat16, true>, tfe_quantize_blocks_kernel<__nv_bfloat16, true>)
                   : go(tfe_quantize_rows_kernel<__nv_bfloat16, false>, tfe_quantize_blocks_kernel<__nv_bfloat16, false>);
    return vec ? go(tfe_quantize_rows_kernel<float, true>, tfe_quantize_blocks_kernel<float, true>)
               : go(tfe_quantize_rows_kernel<float, false>, tfe_quantize_blocks_kernel<float, false>);
}

tfe_status tfe_matmul_fp8(const void *a, int64_t lda, const float *a_scale, int32_t M, const void *w, int64_t ldw, const float *w_scale, int32_t N,
                          int32_t K, void *out, int32_t out_dtype, int64_t ldo, void *stream_)
{
    if (out_dtype != TFE_DTYPE_BF16 && out_dtype != TFE_DTYPE_F32) return TFE_ERR_INVALID_ARG;
    if (M < 0 || M > TFE_ROWS_MAX || N < 1 || N > TFE_ROWS_MAX || K < 1 || K > TFE_FP8_MAX_COLS) return TFE_ERR_INVALID_ARG;
    if (lda < K || lda % 16 != 0 || lda > (1ll << 34) || ldw < K || ldw % 16 != 0 || ldw > (1ll << 34) || ldo < N || ldo > (1ll << 34))
        return TFE_ERR_INVALID_ARG;
    if (M == 0) return TFE_OK;
    if (!aligned(a, 16) || !aligned(w, 16) || !aligned(a_scale, 4) || !aligned(w_scale, 4) || !aligned(out, out_dtype == TFE_DTYPE_BF16 ? 2 : 4))
        return TFE_ERR_INVALID_ARG;
    int dev = 0, sms = 0;
    if (tfe_status st = tfe_note_cuda(cudaGetDevice(&dev), "cudaGetDevice")) return st;
    if (tfe_status st = tfe_note_cuda(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev), "cudaDeviceGetAttribute")) return st;
    MatmulParams p{};
    p.M = M; p.N = N; p.kb = (K + kBlockK - 1) / kBlockK;
    p.a_scale = a_scale; p.b_scale = w_scale; p.out = out; p.ldo = ldo;
    p.give_up = g_give_up.load(std::memory_order_relaxed);
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    CUtensorMap map_w, map_a;
    if (M > kFewRows)
        return out_dtype == TFE_DTYPE_BF16 ? launch_many<__nv_bfloat16>(sms, stream, w, ldw, a, lda, K, p) : launch_many<float>(sms, stream, w, ldw, a, lda, K, p);
    const int tn = M <= 16 ? 16 : M <= 32 ? 32 : 64;
    p.rows_per_cta = (int32_t)((((int64_t)N + sms - 1) / sms + 7) / 8 * 8);
    p.tail_rows = p.rows_per_cta % kTileRows;
    const int grid = (int)(((int64_t)N + p.rows_per_cta - 1) / p.rows_per_cta);
    CUtensorMap map_w_tail;
    if (!make_map_fp8(&map_w, w, N, K, ldw, kTileRows) || !make_map_fp8(&map_w_tail, w, N, K, ldw, p.tail_rows ? (uint32_t)p.tail_rows : 8u) ||
        !make_map_fp8(&map_a, a, M, K, lda, (uint32_t)tn))
        return tfe_note_cuda(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
    switch (tn) {
    case 16: return launch_few<16>(out_dtype, grid, stream, map_w, map_w_tail, map_a, p);
    case 32: return launch_few<32>(out_dtype, grid, stream, map_w, map_w_tail, map_a, p);
    default: return launch_few<64>(out_dtype, grid, stream, map_w, map_w_tail, map_a, p);
    }
}

tfe_status tfe_matmul_fp8_status(uint32_t *device_flags, void *stream_)
{
    if (!device_flags) return TFE_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    void *at = nullptr;
    if (tfe_status st = tfe_note_cuda(cudaGetSymbolAddress(&at, g_matmul_status), "cudaGetSymbolAddress")) return st;
    if (tfe_status st = tfe_note_cuda(cudaMemcpyAsync(device_flags, at, sizeof(uint32_t), cudaMemcpyDeviceToHost, stream), "cudaMemcpyAsync")) return st;
    if (tfe_status st = tfe_note_cuda(cudaStreamSynchronize(stream), "cudaStreamSynchronize")) return st;
    if (*device_flags == 0) return TFE_OK;
    tfe_matmul_fp8_status_kernel<<<1, 1, 0, stream>>>(*device_flags);
    if (tfe_status st = tfe_note_cuda(cudaGetLastError(), "status launch")) return st;
    if (tfe_status st = tfe_note_cuda(cudaStreamSynchronize(stream), "cudaStreamSynchronize")) return st;
    return TFE_ERR_INTERNAL;
}

tfe_status tfe_matmul_fp8_give_up(int32_t how)
{
    g_give_up.store(how == 0 ? 0u : how == (int32_t)kUnderWay ? kUnderWay : kAtOnce, std::memory_order_relaxed);
    return TFE_OK;
}

}  // extern "C"

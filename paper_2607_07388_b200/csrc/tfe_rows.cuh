// Pieces shared by the kernels that walk rows of logits: 16-byte streaming loads of either element type, rows cut
// into an unaligned head, a body of 16-byte vectors and a tail, and the mask convention.
#ifndef TFE_ROWS_CUH
#define TFE_ROWS_CUH

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace tfe_rows {

// A logit at or below this is a masked one, whatever wrote it: -inf, or the lowest value of fp32 or bf16.
constexpr float kMasked = -1e30f;

template <typename T> struct Elem;
template <> struct Elem<float> {
    static constexpr int kPerVec = 4;
    static __device__ __forceinline__ void unpack(const uint4 &v, float (&f)[4])
    {
        f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[4])
    {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
    static __device__ __forceinline__ float get(const float *p) { return *p; }
    static __device__ __forceinline__ void put(float *p, float x) { *p = x; }
};
template <> struct Elem<__nv_bfloat16> {
    static constexpr int kPerVec = 8;
    static __device__ __forceinline__ void unpack(const uint4 &v, float (&f)[8])
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[8])
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&h);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ float get(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
    static __device__ __forceinline__ void put(__nv_bfloat16 *p, float x) { *p = __float2bfloat16_rn(x); }
};

// [0, head) elements before the first 16-byte boundary, then n_vec whole vectors, then the tail up to n.
struct Cut { int64_t head, n_vec; };
template <typename T>
__device__ __forceinline__ Cut cut_row(const T *row, int64_t n)
{
    const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(row) & 15u);
    int64_t head = off ? (int64_t)((16u - off) / sizeof(T)) : 0;
    head = head < n ? head : n;
    return {head, (n - head) / Elem<T>::kPerVec};
}

__device__ __forceinline__ uint4 load_stream(const uint4 *p)      // read once: not kept in L1
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

__device__ __forceinline__ float exp2_approx(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

}  // namespace tfe_rows

#endif

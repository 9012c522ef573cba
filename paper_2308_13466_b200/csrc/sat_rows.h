// Rows of fp32, bf16 or fp16 elements, taken 16 bytes at a time and worked on in fp32; sums over the threads of a row.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "sat_internal.h"

// element types of an entry point that takes rows of several
static inline bool ok_type(int type) { return type == SAT_F32 || type == SAT_BF16 || type == SAT_F16; }
static inline int32_t type_bytes(int type) { return type == SAT_F32 ? 4 : 2; }
// row stride in elements: at least the width, a multiple of 16 bytes
static inline bool ok_ld_of(int type, int32_t ld, int32_t d) { return ld >= d && ((ld * (int64_t)type_bytes(type)) & 15) == 0; }

#ifdef __CUDACC__
template <typename T>
struct RowVec;   // V elements in 16 bytes
template <>
struct RowVec<float> {
    static constexpr int V = 4;
    static __device__ __forceinline__ void unpack(const uint4 &u, float (&f)[4])
    {
        f[0] = __uint_as_float(u.x), f[1] = __uint_as_float(u.y), f[2] = __uint_as_float(u.z), f[3] = __uint_as_float(u.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[4])
    {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
    static __device__ __forceinline__ float from(float x) { return x; }
    static __device__ __forceinline__ float to(float x) { return x; }
};
template <>
struct RowVec<__nv_bfloat16> {
    static constexpr int V = 8;
    static __device__ __forceinline__ void unpack(const uint4 &u, float (&f)[8])
    {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) f[2 * i] = __uint_as_float(w[i] << 16), f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[8])   // to nearest, ties to even
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&p);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ float from(__nv_bfloat16 x) { return __bfloat162float(x); }
    static __device__ __forceinline__ __nv_bfloat16 to(float x) { return __float2bfloat16_rn(x); }
};
template <>
struct RowVec<__half> {
    static constexpr int V = 8;
    static __device__ __forceinline__ void unpack(const uint4 &u, float (&f)[8])
    {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 p = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
            f[2 * i] = p.x, f[2 * i + 1] = p.y;
        }
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[8])
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __half2 p = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&p);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ float from(__half x) { return __half2float(x); }
    static __device__ __forceinline__ __half to(float x) { return __float2half_rn(x); }
};

// Elements [col, col + V) of a row of d: one access where all of them are there, element by element at the row's end (what lies behind it is
// neither read nor written: it may be another matrix's).
template <typename T>
__device__ __forceinline__ uint4 row_load_raw(const T *__restrict__ row, int32_t col, int32_t d)
{
    constexpr int V = RowVec<T>::V;
    uint4 u = make_uint4(0u, 0u, 0u, 0u);
    if (col + V <= d) {
        u = __ldg(reinterpret_cast<const uint4 *>(row + col));
    } else if (col < d) {
        uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < V - 1; ++i) {
            if (col + i >= d) break;
            if (sizeof(T) == 4) w[i % 4] = __ldg(reinterpret_cast<const uint32_t *>(row + col + i));
            else w[i / 2] |= (uint32_t)__ldg(reinterpret_cast<const uint16_t *>(row + col + i)) << (16 * (i & 1));
        }
        u = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return u;
}
template <typename T>
__device__ __forceinline__ void row_load(const T *__restrict__ row, int32_t col, int32_t d, float (&f)[RowVec<T>::V])
{
    RowVec<T>::unpack(row_load_raw(row, col, d), f);
}
template <typename T>
__device__ __forceinline__ void row_store(T *__restrict__ row, int32_t col, int32_t d, const float (&f)[RowVec<T>::V])
{
    constexpr int V = RowVec<T>::V;
    if (col + V <= d) {
        *reinterpret_cast<uint4 *>(row + col) = RowVec<T>::pack(f);
    } else {
#pragma unroll
        for (int i = 0; i < V - 1; ++i)
            if (col + i < d) row[col + i] = RowVec<T>::to(f[i]);
    }
}
// V consecutive fp32 parameters (of d), `other` where there are none
template <int V>
__device__ __forceinline__ void param_load(const float *__restrict__ p, int32_t col, int32_t d, float other, float (&f)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = other;
    if (!p) return;
    if (col + V <= d) {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const float4 v = __ldg(reinterpret_cast<const float4 *>(p + col + i));
            f[i] = v.x, f[i + 1] = v.y, f[i + 2] = v.z, f[i + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < V - 1; ++i)
            if (col + i < d) f[i] = __ldg(p + col + i);
    }
}

// Sums over the TPR threads of a row (a power of two; up to 32 of them lie in one warp, more are the whole block), the same in all of them.
// `red` takes two floats a warp; calls alternate between two of these (`turn`), so that one barrier a call is enough.
template <int TPR>
__device__ __forceinline__ float2 row_sum2(float a, float b, float2 (*red)[32], int &turn)
{
#pragma unroll
    for (int o = (TPR < 32 ? TPR : 32) / 2; o > 0; o >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, o);
        b += __shfl_xor_sync(0xffffffffu, b, o);
    }
    if (TPR > 32) {
        constexpr int W = TPR / 32;
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        if (lane == 0) red[turn][warp] = make_float2(a, b);
        __syncthreads();
        const float2 v = lane < W ? red[turn][lane] : make_float2(0.f, 0.f);
        a = v.x, b = v.y;
#pragma unroll
        for (int o = W / 2; o > 0; o >>= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, o);
            b += __shfl_xor_sync(0xffffffffu, b, o);
        }
        a = __shfl_sync(0xffffffffu, a, 0);
        b = __shfl_sync(0xffffffffu, b, 0);
        turn ^= 1;
    }
    return make_float2(a, b);
}
#endif

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
    static __device__ __forceinline__ uint4 lowest() { return make_uint4(0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u); }   // all -inf
    static __device__ __forceinline__ uint4 cut(const uint4 &u, int32_t n)   // -inf from the n-th element on
    {
        return make_uint4(n > 0 ? u.x : 0xFF800000u, n > 1 ? u.y : 0xFF800000u, n > 2 ? u.z : 0xFF800000u, n > 3 ? u.w : 0xFF800000u);
    }
    static __device__ __forceinline__ uint4 trim(const uint4 &u, int32_t n)   // zeros from the n-th element on
    {
        return make_uint4(n > 0 ? u.x : 0u, n > 1 ? u.y : 0u, n > 2 ? u.z : 0u, n > 3 ? u.w : 0u);
    }
    static __device__ __forceinline__ float largest(const uint4 &u)
    {
        return fmaxf(fmaxf(__uint_as_float(u.x), __uint_as_float(u.y)), fmaxf(__uint_as_float(u.z), __uint_as_float(u.w)));
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
    static __device__ __forceinline__ uint4 lowest() { return make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u); }
    static __device__ __forceinline__ uint4 cut(const uint4 &u, int32_t n)
    {
        uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (2 * i >= n) w[i] = (w[i] & 0xFFFF0000u) | 0xFF80u;
            if (2 * i + 1 >= n) w[i] = (w[i] & 0xFFFFu) | 0xFF800000u;
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ uint4 trim(const uint4 &u, int32_t n)
    {
        uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (2 * i >= n) w[i] &= 0xFFFF0000u;
            if (2 * i + 1 >= n) w[i] &= 0xFFFFu;
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ float largest(const uint4 &u)
    {
        auto two = [](uint32_t w) { return *reinterpret_cast<const __nv_bfloat162 *>(&w); };
        const float2 m = __bfloat1622float2(__hmax2(__hmax2(two(u.x), two(u.y)), __hmax2(two(u.z), two(u.w))));
        return fmaxf(m.x, m.y);
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
    static __device__ __forceinline__ uint4 lowest() { return make_uint4(0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u); }
    static __device__ __forceinline__ uint4 cut(const uint4 &u, int32_t n)
    {
        uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (2 * i >= n) w[i] = (w[i] & 0xFFFF0000u) | 0xFC00u;
            if (2 * i + 1 >= n) w[i] = (w[i] & 0xFFFFu) | 0xFC000000u;
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ uint4 trim(const uint4 &u, int32_t n)
    {
        uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (2 * i >= n) w[i] &= 0xFFFF0000u;
            if (2 * i + 1 >= n) w[i] &= 0xFFFFu;
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ float largest(const uint4 &u)
    {
        auto two = [](uint32_t w) { return *reinterpret_cast<const __half2 *>(&w); };
        const float2 m = __half22float2(__hmax2(__hmax2(two(u.x), two(u.y)), __hmax2(two(u.z), two(u.w))));
        return fmaxf(m.x, m.y);
    }
    static __device__ __forceinline__ float from(__half x) { return __half2float(x); }
    static __device__ __forceinline__ __half to(float x) { return __float2half_rn(x); }
};

// Elements [col, col + V) of a row of d, col a multiple of V: 16 bytes, of which those behind the row's end (another matrix's, or padding) are read and
// mean nothing.  Plain loads: a row's results may go where it lies.
template <typename T>
__device__ __forceinline__ uint4 row_load_raw(const T *row, int32_t col, int32_t d)
{
    return col < d ? *reinterpret_cast<const uint4 *>(row + col) : make_uint4(0u, 0u, 0u, 0u);
}
// ... as numbers, zeros behind the end
template <typename T>
__device__ __forceinline__ void row_unpack(const uint4 &u, int32_t col, int32_t d, float (&f)[RowVec<T>::V])
{
    RowVec<T>::unpack(u, f);
    if (col + RowVec<T>::V > d) {
#pragma unroll
        for (int i = 0; i < RowVec<T>::V; ++i)
            if (col + i >= d) f[i] = 0.f;
    }
}
template <typename T>
__device__ __forceinline__ void row_load(const T *row, int32_t col, int32_t d, float (&f)[RowVec<T>::V])
{
    row_unpack<T>(row_load_raw(row, col, d), col, d, f);
}
// results: what lies behind the row's end is left as it is
template <typename T>
__device__ __forceinline__ void row_store(T *row, int32_t col, int32_t d, const float (&f)[RowVec<T>::V])
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
// V fp32 results, whatever V
template <int V>
__device__ __forceinline__ void row_store_f32(float *row, int32_t col, int32_t d, const float (&f)[V])
{
#pragma unroll
    for (int i = 0; i < V; i += 4) {
        const float v[4] = {f[i], f[i + 1], f[i + 2], f[i + 3]};
        if (col + i < d) row_store(row, col + i, d, v);
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

// two fp32 operations in one instruction
__device__ __forceinline__ uint64_t f2_pack(float a, float b)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 f2_unpack(uint64_t v)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ uint64_t f2_add(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t f2_mul(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t f2_fma(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t f2_ex2(uint64_t a)
{
    const float2 v = f2_unpack(a);
    return f2_pack(ex2_fast(v.x), ex2_fast(v.y));
}

// rows by pairs of elements: 16 bytes of one, zeros behind its end; parameters; results
template <typename T>
__device__ __forceinline__ void pair_unpack(uint4 u, int32_t col, int32_t d, uint64_t (&f)[RowVec<T>::V / 2])
{
    constexpr int V = RowVec<T>::V;
    if (col + V > d) u = RowVec<T>::trim(u, d - col);
    float v[V];
    RowVec<T>::unpack(u, v);
#pragma unroll
    for (int i = 0; i < V / 2; ++i) f[i] = f2_pack(v[2 * i], v[2 * i + 1]);
}
template <int V>
__device__ __forceinline__ void pair_param(const float *__restrict__ p, int32_t col, int32_t d, float other, uint64_t (&f)[V / 2])
{
    float v[V];
    param_load<V>(p, col, d, other, v);
#pragma unroll
    for (int i = 0; i < V / 2; ++i) f[i] = f2_pack(v[2 * i], v[2 * i + 1]);
}
template <int V>
__device__ __forceinline__ void pair_floats(const uint64_t (&f)[V / 2], float (&v)[V])
{
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        const float2 x = f2_unpack(f[i]);
        v[2 * i] = x.x, v[2 * i + 1] = x.y;
    }
}
__device__ __forceinline__ uint64_t f2_all(float a) { return f2_pack(a, a); }
__device__ __forceinline__ float f2_sum(uint64_t a) { return f2_unpack(a).x + f2_unpack(a).y; }

// Sums over the TPR threads of a row (a power of two; up to 32 of them lie in one warp, more are the whole block and meet at its barrier), the same in all of them.
// `red` takes a pair a warp; calls alternate between two of these (`turn`), so that one barrier a call is enough.
template <int TPR>
__device__ __forceinline__ float row_sum(float a, float2 (*red)[32], int &turn)
{
#pragma unroll
    for (int o = (TPR < 32 ? TPR : 32) / 2; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
    if constexpr (TPR > 32) {
        constexpr int W = TPR / 32;
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        if (lane == 0) red[turn][warp].x = a;
        __syncthreads();
        a = red[turn][lane % W].x;
#pragma unroll
        for (int o = W / 2; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
        turn ^= 1;
    }
    return a;
}
// Two sums at once: half of the lanes add up one, half the other, which takes little more than one of them alone.
template <int TPR>
__device__ __forceinline__ float2 row_sum2(float a, float b, float2 (*red)[32], int &turn)
{
    constexpr int L = TPR < 32 ? TPR : 32, HALF = L / 2;
    const int lane = threadIdx.x & 31;
    const bool upper = (lane & HALF) != 0;
    float v = upper ? b : a;
    v += __shfl_xor_sync(0xffffffffu, upper ? a : b, HALF);
#pragma unroll
    for (int o = HALF / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if constexpr (TPR > 32) {
        constexpr int W = TPR / 32, P = W < 16 ? W : 16;   // (32 warps: a lane takes two)
        const int warp = threadIdx.x >> 5;
        if ((lane & 15) == 0) (upper ? red[turn][warp].y : red[turn][warp].x) = v;
        __syncthreads();
        const float *from = &red[turn][0].x + (upper ? 1 : 0);
        v = from[2 * (lane % P)];
        if (W == 32) v += from[2 * (lane % P + 16)];
#pragma unroll
        for (int o = P / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        turn ^= 1;
    }
    return make_float2(__shfl_sync(0xffffffffu, v, 0, L), __shfl_sync(0xffffffffu, v, HALF, L));
}
#endif

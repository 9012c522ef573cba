// Microscaled matrices: layout and the two formats, shared by their kernels (sat_mx.cu, sat_mx_tc.cu).
#pragma once

#include "sat_internal.h"

#define MX_GROUP 32
#define MX_MAX (INT32_MAX - 255)   /* rows and columns: the kernels count in 32 bits, up to a tile past the end */

static inline int32_t mx_groups(int32_t d) { return (d + MX_GROUP - 1) / MX_GROUP; }
// bytes of codes in a row, the last group filled up
static inline int32_t mx_row_bytes(const sat_mx_matrix *q) { return mx_groups(q->d) * (q->format == SAT_MX8 ? 32 : 16); }

// The matrix as kernels take it
struct MxView {
    uint8_t *codes, *scales;
    int64_t ld_codes, ld_scales;
};
static inline MxView mx_view(const sat_mx_matrix *q) { return MxView{q->codes, q->scales, q->ld_codes, q->ld_scales}; }

// =====================================================================================
// the two formats
// =====================================================================================
// Scale byte of a group from the bits of its largest magnitude: the exponent that brings it to [largest / 2, largest], rounded up from the
// fraction's compare with 1.75 (448 = 1.75 2^8) or 1.5 (6 = 1.5 2^2) by a carry; 255 where that magnitude is no finite number.
template <int FMT>
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t amax)
{
    if (amax >= 0x7F800000u) return 255u;
    const int32_t e = (int32_t)((amax + (FMT == SAT_MX8 ? 0x1FFFFFu : 0x3FFFFFu)) >> 23) - (FMT == SAT_MX8 ? 8 : 2);
    return e > 0 ? (uint32_t)e : 0u;
}
// 2^(127 - byte), which is never subnormal: bytes go up to 253, and NaN's comes out as 0.  (x 2^-e is rounded only where it is below
// 2^-126, far under half a step of either format.)
__device__ __forceinline__ float mx_inverse(uint32_t byte) { return byte == 255u ? 0.f : __uint_as_float((254u - byte) << 23); }
// 2^(byte - 127); byte 0 is a subnormal number, 255 stands for NaN
__device__ __forceinline__ float mx_power(uint32_t byte)
{
    return byte == 255u ? __uint_as_float(0x7FFFFFFFu) : byte == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(byte << 23);
}
// four elements -> four bytes (SAT_MX8) or two (SAT_MX4), the first element lowest
template <int FMT>
__device__ __forceinline__ uint32_t mx_encode4(float a, float b, float c, float d)
{
    uint32_t r;
    if (FMT == SAT_MX8)
        asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\tmov.b32 %0, {l, h};\n\t}"
            : "=r"(r)
            : "f"(a), "f"(b), "f"(c), "f"(d));
    else
        asm("{\n\t.reg .b8 l, h, z;\n\tcvt.rn.satfinite.e2m1x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 h, %4, %3;\n\tmov.b32 %0, {l, h, l, h};\n\t}"
            : "=r"(r)
            : "f"(a), "f"(b), "f"(c), "f"(d));
    return r;
}
// a group of 32 elements -> 32 or 16 bytes of codes; the scale byte
template <int FMT>
__device__ __forceinline__ uint32_t mx_quantise32(const float4 (&v)[8], uint32_t (&code)[FMT])
{
    uint32_t top[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        top[i] = max(max(__float_as_uint(v[i].x) & 0x7FFFFFFFu, __float_as_uint(v[i].y) & 0x7FFFFFFFu), max(__float_as_uint(v[i].z) & 0x7FFFFFFFu, __float_as_uint(v[i].w) & 0x7FFFFFFFu));
    const uint32_t byte = mx_scale_byte<FMT>(max(max(max(top[0], top[1]), max(top[2], top[3])), max(max(top[4], top[5]), max(top[6], top[7]))));
    const float f = mx_inverse(byte);
    uint32_t c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = byte == 255u ? 0u : mx_encode4<FMT>(v[i].x * f, v[i].y * f, v[i].z * f, v[i].w * f);
#pragma unroll
    for (int i = 0; i < FMT; ++i) code[i] = FMT == SAT_MX8 ? c[i] : (c[(2 * i) & 7] & 0xFFFFu) | c[(2 * i + 1) & 7] << 16;
    return byte;
}
// two elements as a pair of halves, without the scale
template <int FMT>
__device__ __forceinline__ uint32_t mx_decode2(uint32_t code)
{
    uint32_t r;
    if (FMT == SAT_MX8)
        asm("{\n\t.reg .b16 t;\n\tcvt.u16.u32 t, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, t;\n\t}" : "=r"(r) : "r"(code));
    else
        asm("{\n\t.reg .b8 t;\n\tcvt.u8.u32 t, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, t;\n\t}" : "=r"(r) : "r"(code));
    return r;
}
__device__ __forceinline__ float2 mx_unpack(uint32_t halves)
{
    float2 f;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, h;\n\t}" : "=f"(f.x), "=f"(f.y) : "r"(halves));
    return f;
}
// element (r, c)
template <int FMT>
__device__ __forceinline__ float mx_element(const MxView &q, int64_t r, int32_t c)
{
    const float s = mx_power(__ldg(q.scales + r * q.ld_scales + (c >> 5)));
    if (FMT == SAT_MX8) return mx_unpack(mx_decode2<FMT>(__ldg(q.codes + r * q.ld_codes + c))).x * s;
    const float2 p = mx_unpack(mx_decode2<FMT>(__ldg(q.codes + r * q.ld_codes + (c >> 1))));
    return ((c & 1) ? p.y : p.x) * s;
}

// columns of a tile: as few tiles of at most 256 as possible, of equal width, whole groups
static inline int32_t mx_tile_columns(int32_t n)
{
    const int32_t tiles = (n + 255) / 256;
    return ((n + tiles - 1) / tiles + MX_GROUP - 1) / MX_GROUP * MX_GROUP;
}

// Contractions on the tensor cores (sat_mx_nt.cu, sat_mx_tc.cu); shapes are checked by the callers and not empty
sat_status sat_mx_tc_nn(sat_ctx *ctx, int64_t m, const float *A, int32_t lda, const sat_mx_matrix *W, float *C, int32_t ldc);
sat_status sat_mx_tc_tn(sat_ctx *ctx, const sat_mx_matrix *A, int32_t n, const float *B, int32_t ldb, float *C, float *colsum, int accumulate);
// A (quantised, and kept in Aq where given) or, without it, Aq
sat_status sat_mx_tc_nt(sat_ctx *ctx, int64_t m, const float *A, int32_t lda, const sat_mx_matrix *Aq, const sat_mx_matrix *W, const float *bias, float *C, int32_t ldc);

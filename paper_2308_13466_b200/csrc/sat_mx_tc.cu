// Contractions of fp32 rows with microscaled matrices on the 5th-generation tensor cores.
//     k_mx_gemm<true>    C[q.d x n] = Q^^T X     sat_mx_dense_tn: the terms run over the rows of both, split over CTAs
//     k_mx_gemm<false>   C[m x q.d] = X Q^       sat_mx_dense_nn: the terms run over the columns of X and the rows of Q
// What a code stands for has four significant bits and a power of two, so it is a bf16 number.  An fp32 operand is cut into three bf16
// terms by taking the upper half of its bits off twice, which is exact: x = hi + mid + lo, eight bits each.  Three MMAs of
// kind::f16 with bf16 operands then give exact products, and all that is rounded is the sum.
//
// The tensor core chops its running sum at every instruction (16 products), always towards zero, so a sum in one accumulator drifts:
// about a third of a unit of 2^-23 per instruction.  Only the products with hi matter for that; those with mid and lo are 2^-8 of them and
// have an accumulator of their own.  The hi accumulator is taken out after MX_FLUSH stages (24 instructions) and added up in registers,
// rounded to nearest; relative error 3e-7 to 1e-6, about that of an fp32 FMA loop.
//
// One CTA per SM, 20 warps, two of them idle.  Warps 0..15 convert a stage of 32 terms (raw fp32 and codes in shared memory, brought by TMA, to
// swizzled bf16 tiles) and hold the sums; warp 16 issues the MMAs; warp 17 issues the TMA loads and adds up the columns of X where
// the bias gradient is asked for.  The fp32 operand is the M side (128 lanes of TMEM), the codes are the N side (up to 256 columns).
#include "sat_mx.h"
#include "sat_ptx.h"

#include <algorithm>

#define MXT_WORKERS 16
#define MXT_THREADS ((MXT_WORKERS + 4) * 32)   /* five whole warpgroups, see k_mx_gemm */
#define MXT_KB 32                    /* terms per stage */
#define MXT_OP 3                     /* stages of converted tiles */
#define MXT_RAW 4                    /* stages of raw tiles */
#define MXT_FLUSH 12                 /* stages between two reads of the hi accumulator */
#define MXT_X_PLANE (128 * MXT_KB * 2)
#define MXT_Q_TILE (256 * MXT_KB * 2)
#define MXT_STAGE (3 * MXT_X_PLANE + MXT_Q_TILE)
#define MXT_X_RAW (128 * MXT_KB * 4)
#define MXT_Q_RAW (256 * MXT_KB)
#define MXT_RAW_STAGE (MXT_X_RAW + MXT_Q_RAW)

struct MxtShared {
    uint64_t raw_full[MXT_RAW], raw_empty[MXT_RAW];   // TMA bytes have landed; the workers (and the column sums) have read them
    uint64_t op_full[MXT_OP], op_empty[MXT_OP];       // the workers have written the tiles; the MMAs have read them
    uint64_t acc_full, acc_empty;                     // the hi accumulator is to be taken out; has been
    uint64_t turned;                                  // (NN) the results have left the operand stages
    uint32_t tmem_base;
    int dead;
};
#define MXT_SMEM (1024 + MXT_OP * MXT_STAGE + MXT_RAW * MXT_RAW_STAGE + (int)sizeof(MxtShared))
static_assert(MXT_SMEM <= 227 * 1024, "shared memory");
static_assert(MXT_OP * MXT_STAGE >= MXT_WORKERS * 32 * 36 * 4, "the results are turned around in the operand stages");

struct MxtArgs {
    const uint8_t *scales;
    int64_t ld_scales;
    int32_t groups;            // of a row of Q
    int32_t M, N;              // rows of the tile grid: columns of X (TN) or rows of X (NN); columns of Q
    int32_t K, kps;            // terms, and terms of a split (a multiple of MXT_KB)
    int32_t bn, tiles_m, tiles_n;
    int32_t items;             // tiles times splits, the tiles of a split next to each other
    float *C;                  // TN: [splits][N][M] partial sums, or with one split the result; NN: [M x ldc]
    int64_t ldc;
    float *colsum;             // TN: [splits][M] column sums of X, or none
    int direct, accumulate;    // TN with one split: C and colsum are the results, and are added to
    int *status;
};
// A tile and its terms [k0, k1)
struct MxtItem {
    int32_t m0, n0, split, k0, k1, stages;
};
__device__ __forceinline__ MxtItem mxt_item(const MxtArgs &a, int32_t i)
{
    MxtItem t;
    const int32_t tiles = a.tiles_m * a.tiles_n, tile = i % tiles;
    t.split = i / tiles;
    t.m0 = tile / a.tiles_n * 128;
    t.n0 = tile % a.tiles_n * a.bn;
    t.k0 = t.split * a.kps;
    t.k1 = a.K - t.k0 < a.kps ? a.K : t.k0 + a.kps;
    t.stages = (t.k1 - t.k0 + MXT_KB - 1) / MXT_KB;
    return t;
}

// ---- formats to bf16 ------------------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t bf16x2_mul(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// A code's bits moved to bf16's exponent and fraction are the number times 2^-120 (e4m3) or 2^-126 (e2m1), subnormal codes included; one
// exact product with a power of two puts that and the group's scale right.  Scales above 2^7 (2^1) need a second one.
// Integer logic runs at half the rate of multiply-adds, so the bits are moved by the latter: with a code in the low byte of a half-word,
// code 2^s has its exponent and fraction in place, and (sign bit) (2^t - 2^s) more moves the sign up to bit 15.
template <int FMT>
struct MxtScale {
    uint32_t first, second;   // pairs of bf16
    bool two;
    __device__ __forceinline__ explicit MxtScale(uint32_t byte)
    {
        constexpr uint32_t bias = FMT == SAT_MX8 ? 120u : 126u;
        const uint32_t e = byte + bias;                       // exponent of the whole factor + 127
        two = e > 254u;
        const uint32_t f = byte == 255u ? 0x7FFFu : two ? 254u << 7 : e << 7;
        first = f * 0x10001u;
        second = byte == 255u ? 0x3F803F80u : ((e - 127u) << 7) * 0x10001u;   // what is left of it: e - 127 - 127, plus 127
    }
};
// eight elements (two words of e4m3 or one of e2m1) as four pairs of bf16, in order
template <int FMT>
__device__ __forceinline__ uint4 mxt_decode8(uint32_t lo, uint32_t hi, const MxtScale<FMT> &sc)
{
    uint32_t x[4];
    if (FMT == SAT_MX8) {
        x[0] = __byte_perm(lo, 0, 0x4140);
        x[1] = __byte_perm(lo, 0, 0x4342);
        x[2] = __byte_perm(hi, 0, 0x4140);
        x[3] = __byte_perm(hi, 0, 0x4342);
    } else {
        const uint32_t even = lo & 0x0F0F0F0Fu, odd = (lo >> 4) & 0x0F0F0F0Fu;
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            // byte i of either, and their sign bits, which are zero, above them
            asm("prmt.b32 %0, %1, %2, %3;" : "=r"(x[i]) : "r"(even), "r"(odd), "r"(0xC480u + 0x1111u * i));
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t sign = x[i] & (FMT == SAT_MX8 ? 0x00800080u : 0x00080008u);
        x[i] = bf16x2_mul(x[i] * (FMT == SAT_MX8 ? 16u : 64u) + sign * (FMT == SAT_MX8 ? 256u - 16u : 4096u - 64u), sc.first);
    }
    return make_uint4(x[0], x[1], x[2], x[3]);
}
__device__ __forceinline__ uint4 bf16x8_mul(const uint4 &v, uint32_t s)
{
    return make_uint4(bf16x2_mul(v.x, s), bf16x2_mul(v.y, s), bf16x2_mul(v.z, s), bf16x2_mul(v.w, s));
}
// eight fp32 values -> eight bf16 each of hi, mid, lo (upper halves; what is left after two of them fits a third)
__device__ __forceinline__ void mxt_split8(const float4 &a, const float4 &b, uint4 &hi, uint4 &mid, uint4 &lo)
{
    const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    uint32_t h[4], m[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        h[i] = __byte_perm(__float_as_uint(x[2 * i]), __float_as_uint(x[2 * i + 1]), 0x7632);
        const float r0 = x[2 * i] - __uint_as_float(h[i] * 0x10000u), r1 = x[2 * i + 1] - __uint_as_float(h[i] & 0xFFFF0000u);
        m[i] = __byte_perm(__float_as_uint(r0), __float_as_uint(r1), 0x7632);
        const float s0 = r0 - __uint_as_float(m[i] * 0x10000u), s1 = r1 - __uint_as_float(m[i] & 0xFFFF0000u);
        l[i] = __byte_perm(__float_as_uint(s0), __float_as_uint(s1), 0x7632);
    }
    hi = make_uint4(h[0], h[1], h[2], h[3]);
    mid = make_uint4(m[0], m[1], m[2], m[3]);
    lo = make_uint4(l[0], l[1], l[2], l[3]);
}

__device__ __forceinline__ void tc_ld16(uint32_t taddr, uint32_t *r)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr)
                 : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// bf16 operands, fp32 accumulation; Q is MN-major (its tile has a row per term), X is with TN
template <bool TN>
__device__ __forceinline__ uint32_t mxt_idesc(int32_t bn)
{
    return 1u << 4 | 1u << 7 | 1u << 10 | (TN ? 1u << 15 : 0u) | 1u << 16 | (uint32_t)(bn >> 3) << 17 | (128u >> 4) << 24;
}

// ---- the roles --------------------------------------------------------------------------------------------------------------
struct MxtMem {
    uint8_t *op, *raw;
    MxtShared *sh;
    uint32_t tmem;
};

template <bool TN>
__device__ __forceinline__ void mxt_mma(const MxtArgs &a, const MxtMem &s, int32_t first, int32_t step)
{
    volatile int *dead = &s.sh->dead;
    const uint32_t idesc = mxt_idesc<TN>(a.bn);
    // MN-major tiles: blocks of 64 columns (128 bytes a term, 128-byte swizzle) MXT_KB x 128 bytes apart, groups of eight terms 1024 bytes
    // apart; an instruction takes 16 terms.  K-major (X without TN): a row's 32 terms are 64 bytes, 64-byte swizzle, eight rows 512 apart.
    const uint64_t q0 = make_desc(smem_u32(s.op) + 3 * MXT_X_PLANE, MXT_KB * 128, 1024, 2);
    const uint64_t x0 = TN ? make_desc(smem_u32(s.op), MXT_KB * 128, 1024, 2) : make_desc(smem_u32(s.op), 16, 512, 4);
    constexpr uint32_t x_step = (TN ? 2048 : 32) >> 4, q_step = 2048 >> 4, plane = MXT_X_PLANE >> 4;
    uint32_t st = 0, ph = 0, taken = 0;   // taken: times the accumulators were handed over so far
    for (int32_t i = first; i < a.items; i += step) {
        const int32_t stages = mxt_item(a, i).stages;
        int32_t in_run = 0;               // stages since the hi accumulator was last handed over
        for (int32_t k = 0; k < stages; ++k) {
            if (!mbar_wait_all(&s.sh->op_full[st], ph, dead, a.status)) return;
            tc_fence_after();
            const uint64_t x = x0 + (uint64_t)(st * (MXT_STAGE >> 4)), q = q0 + (uint64_t)(st * (MXT_STAGE >> 4));
            // (acc_empty's phase `taken - 1` completes when the workers have read what was handed over last)
            if (k == 0 && taken > 0) {
                if (!mbar_wait_all(&s.sh->acc_empty, (taken - 1) & 1u, dead, a.status)) return;
                tc_fence_after();
            }
            if (elect_one()) {
#pragma unroll
                for (uint32_t ks = 0; ks < MXT_KB / 16; ++ks)
#pragma unroll
                    for (uint32_t t = 1; t < 3; ++t)
                        tc_mma_f16<0, 1>(s.tmem + 256u, x + ks * x_step + t * plane, q + ks * q_step, idesc, k > 0 || ks > 0 || t > 1 ? 1u : 0u);
            }
            __syncwarp();
            if (in_run == 0 && k > 0) {
                if (!mbar_wait_all(&s.sh->acc_empty, (taken - 1) & 1u, dead, a.status)) return;
                tc_fence_after();
            }
            const bool hand_over = ++in_run == MXT_FLUSH || k + 1 == stages;
            if (elect_one()) {
#pragma unroll
                for (uint32_t ks = 0; ks < MXT_KB / 16; ++ks)
                    tc_mma_f16<0, 1>(s.tmem, x + ks * x_step, q + ks * q_step, idesc, in_run > 1 || ks > 0 ? 1u : 0u);
                tc_commit<1>(&s.sh->op_empty[st]);
                if (hand_over) tc_commit<1>(&s.sh->acc_full);
            }
            __syncwarp();
            if (hand_over) ++taken, in_run = 0;
            if (++st == MXT_OP) st = 0, ph ^= 1u;
        }
    }
}

// TMA loads, up to MXT_RAW stages ahead of the workers; the column sums of X in doubles, four columns a lane
template <bool TN, int FMT>
__device__ __forceinline__ void mxt_load(const MxtArgs &a, const MxtMem &s, const CUtensorMap *map_x, const CUtensorMap *map_q, int32_t first, int32_t step, int lane)
{
    volatile int *dead = &s.sh->dead;
    int32_t ahead = first;              // what is loaded next
    int32_t ahead_k = 0;
    MxtItem at{};
    if (ahead < a.items) at = mxt_item(a, ahead);
    uint32_t lst = 0, lph = 0;
    auto load = [&]() -> bool {
        if (ahead >= a.items) return true;
        if (!mbar_wait_all(&s.sh->raw_empty[lst], lph ^ 1u, dead, a.status)) return false;
        if (lane == 0) {
            uint8_t *x = s.raw + (size_t)lst * MXT_RAW_STAGE, *q = x + MXT_X_RAW;
            uint64_t *bar = &s.sh->raw_full[lst];
            const int32_t k = at.k0 + ahead_k * MXT_KB;
            const int32_t boxes = TN ? (a.M - at.m0 + 31) / 32 < 4 ? (a.M - at.m0 + 31) / 32 : 4 : 1;
            mbar_expect_tx(bar, (TN ? (uint32_t)boxes * 4096u : (uint32_t)MXT_X_RAW) + (uint32_t)(a.bn * MXT_KB * FMT / 8));
            if (TN)
                for (int b = 0; b < boxes; ++b) tma_load_2d(x + b * 4096, map_x, bar, at.m0 + 32 * b, k);
            else tma_load_2d(x, map_x, bar, k, at.m0);
            tma_load_2d(q, map_q, bar, at.n0 * FMT / 8, k);
        }
        __syncwarp();
        if (++lst == MXT_RAW) lst = 0, lph ^= 1u;
        if (++ahead_k == at.stages) {
            ahead_k = 0;
            ahead += step;
            if (ahead < a.items) at = mxt_item(a, ahead);
        }
        return true;
    };
    for (int i = 0; i < MXT_RAW - 1; ++i)
        if (!load()) return;
    uint32_t st = 0, ph = 0;
    for (int32_t i = first; i < a.items; i += step) {
        const MxtItem it = mxt_item(a, i);
        const bool sums = TN && a.colsum && it.n0 == 0;
        double c[4] = {0., 0., 0., 0.};
        for (int32_t k = 0; k < it.stages; ++k) {
            if (!load()) return;
            if (!TN) continue;
            if (!mbar_wait_all(&s.sh->raw_full[st], ph, dead, a.status)) return;
            if (sums && it.m0 + (lane >> 3) * 32 < a.M) {
                const uint8_t *x = s.raw + (size_t)st * MXT_RAW_STAGE + (lane >> 3) * 4096;
                float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
                for (int r = 0; r < MXT_KB; ++r) {
                    const float4 v = *reinterpret_cast<const float4 *>(x + r * 128 + (((lane & 7) ^ (r & 7)) << 4));
                    t.x += v.x;
                    t.y += v.y;
                    t.z += v.z;
                    t.w += v.w;
                }
                c[0] += t.x;
                c[1] += t.y;
                c[2] += t.z;
                c[3] += t.w;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&s.sh->raw_empty[st]);
            if (++st == MXT_RAW) st = 0, ph ^= 1u;
        }
        if (sums)
            for (int j = 0; j < 4; ++j) {
                const int32_t col = it.m0 + 4 * lane + j;
                if (col >= a.M) continue;
                float *out = a.colsum + (int64_t)it.split * a.M + col;
                *out = a.direct && a.accumulate ? (float)((double)*out + c[j]) : (float)c[j];
            }
    }
}

template <bool TN, int FMT>
__device__ __forceinline__ void mxt_work(const MxtArgs &a, const MxtMem &s, int32_t first, int32_t step, int warp, int lane)
{
    volatile int *dead = &s.sh->dead;
    // Eight values of X and 16 elements of Q per thread and stage.  Terms of Q (and of X with TN): `term`; the places along a row go over the
    // lanes so that eight lanes in turn touch all banks, in the raw rows as in the swizzled ones.
    const int j = (lane >> 2) & 1, term = 2 * warp + (j ^ ((lane >> 3) & 1)), place = (lane & 3) | j << 2 | (lane >> 4) << 3;
    const int row = TN ? 0 : 8 * warp + (lane >> 2), quad = lane & 3;     // (NN) row of X and which eight of its 32 terms
    const uint32_t x_raw = TN ? (uint32_t)(place >> 2) * 4096u + (uint32_t)term * 128u : (uint32_t)row * 128u;
    const uint32_t x_at = (uint32_t)((2 * (TN ? place & 3 : quad)) ^ ((TN ? term : row) & 7)) << 4;
    const uint32_t x_op = TN ? (uint32_t)(place >> 3) * (MXT_KB * 128) + (uint32_t)term * 128u + (uint32_t)(((place & 7) ^ (term & 7)) << 4)
                             : (uint32_t)row * 64u + (uint32_t)((quad ^ ((row >> 1) & 3)) << 4);
    const uint32_t q_raw = MXT_X_RAW + (uint32_t)(term * a.bn + 16 * place) * FMT / 8;
    const uint32_t q_op = 3 * MXT_X_PLANE + (uint32_t)(place >> 2) * (MXT_KB * 128) + (uint32_t)term * 128u;
    const uint32_t q_at = (uint32_t)((2 * (place & 3)) ^ (term & 7)) << 4;
    const bool has_q = 16 * place < a.bn;
    const int chunks = a.bn / 32;

    // scale bytes come two stages ahead: `left` more terms of the item ahead, the byte of its next stage at `next`
    int32_t ahead = first, left = 0;
    const uint8_t *next = a.scales;
    bool in_range = false;
    const int64_t stage_scales = a.ld_scales * MXT_KB;
    auto scale = [&]() -> uint32_t {
        if (left <= 0) {
            if (ahead >= a.items) return 127u;
            const MxtItem t = mxt_item(a, ahead);
            const int32_t g = (t.n0 + 16 * place) / MX_GROUP;
            in_range = has_q && g < a.groups;
            next = a.scales + (int64_t)(t.k0 + term) * a.ld_scales + g;
            left = t.k1 - t.k0;
            ahead += step;
        }
        uint32_t byte = 127u;
        if (in_range && term < left) byte = __ldg(next);
        next += stage_scales;
        left -= MXT_KB;
        return byte;
    };
    uint32_t b0 = scale(), b1 = scale();
    uint32_t rst = 0, rph = 0, ost = 0, oph = 0, taken = 0, turned = 0;
    const uint32_t lanes = s.tmem + ((uint32_t)((warp & 3) * 32) << 16);
    for (int32_t i = first; i < a.items; i += step) {
        const MxtItem it = mxt_item(a, i);
        const bool has_x = !TN || it.m0 + 8 * place < a.M;
        float acc[2][32];
#pragma unroll
        for (int c = 0; c < 64; ++c) acc[c >> 5][c & 31] = 0.f;
        auto take = [&](uint32_t base) {
#pragma unroll
            for (int c = 0; c < 2; ++c)
                if ((warp >> 2) + 4 * c < chunks) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t r[16];
                        tc_ld16(lanes + base + (uint32_t)((warp >> 2) + 4 * c) * 32u + 16u * h, r);
#pragma unroll
                        for (int e = 0; e < 16; ++e) acc[c][16 * h + e] += __uint_as_float(r[e]);
                    }
                }
        };
        auto hand_back = [&]() {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&s.sh->acc_empty);
            ++taken;
        };
        int32_t in_run = 0;
#pragma unroll 1
        for (int32_t k = 0; k < it.stages; ++k) {
            const uint32_t byte = b0;
            b0 = b1;
            b1 = scale();
            if (!mbar_wait_all(&s.sh->raw_full[rst], rph, dead, a.status)) return;
            const uint8_t *raw = s.raw + (size_t)rst * MXT_RAW_STAGE;
            float4 xa = make_float4(0.f, 0.f, 0.f, 0.f), xb = xa;
            if (has_x) {
                xa = *reinterpret_cast<const float4 *>(raw + x_raw + x_at);
                xb = *reinterpret_cast<const float4 *>(raw + x_raw + (x_at ^ 16u));
            }
            uint32_t c[4] = {0u, 0u, 0u, 0u};
            if (has_q) {
                if (FMT == SAT_MX8) {
                    const uint4 t = *reinterpret_cast<const uint4 *>(raw + q_raw);
                    c[0] = t.x, c[1] = t.y, c[2] = t.z, c[3] = t.w;
                } else {
                    const uint2 t = *reinterpret_cast<const uint2 *>(raw + q_raw);
                    c[0] = t.x, c[1] = t.y;
                }
            }
            uint4 h, m, l;
            mxt_split8(xa, xb, h, m, l);
            const MxtScale<FMT> sc(byte);
            uint4 v0 = mxt_decode8<FMT>(c[0], c[1], sc), v1 = FMT == SAT_MX8 ? mxt_decode8<FMT>(c[2], c[3], sc) : mxt_decode8<FMT>(c[1], 0u, sc);
            if (sc.two) v0 = bf16x8_mul(v0, sc.second), v1 = bf16x8_mul(v1, sc.second);
            __syncwarp();
            if (lane == 0) mbar_arrive(&s.sh->raw_empty[rst]);
            if (++rst == MXT_RAW) rst = 0, rph ^= 1u;
            if (!mbar_wait_all(&s.sh->op_empty[ost], oph ^ 1u, dead, a.status)) return;
            uint8_t *op = s.op + (size_t)ost * MXT_STAGE;
            if (has_x) {
                *reinterpret_cast<uint4 *>(op + x_op) = h;
                *reinterpret_cast<uint4 *>(op + x_op + MXT_X_PLANE) = m;
                *reinterpret_cast<uint4 *>(op + x_op + 2 * MXT_X_PLANE) = l;
            }
            if (has_q) {
                *reinterpret_cast<uint4 *>(op + q_op + q_at) = v0;
                *reinterpret_cast<uint4 *>(op + q_op + (q_at ^ 16u)) = v1;
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&s.sh->op_full[ost]);
            if (++ost == MXT_OP) ost = 0, oph ^= 1u;
            // taken out one stage late, so that the MMAs have something to do meanwhile
            if (in_run == MXT_FLUSH) {
                if (!mbar_wait_all(&s.sh->acc_full, taken & 1u, dead, a.status)) return;
                tc_fence_after();
                take(0u);
                hand_back();
                in_run = 0;
            }
            ++in_run;
        }
        if (!mbar_wait_all(&s.sh->acc_full, taken & 1u, dead, a.status)) return;
        tc_fence_after();
        take(0u);
        take(256u);
        hand_back();
        const int32_t q32 = (warp & 3) * 32;
        if (TN) {
            // a lane has a column of X, a register a column of Q: consecutive lanes write consecutive floats
            const int32_t col = it.m0 + q32 + lane;
            float *C = a.C + (int64_t)it.split * a.M * a.N;
            if (col < a.M)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int32_t r0 = it.n0 + ((warp >> 2) + 4 * c) * 32;
                    if ((warp >> 2) + 4 * c < chunks)
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (r0 + e < a.N) {
                                float *o = C + (int64_t)(r0 + e) * a.M + col;
                                *o = a.direct && a.accumulate ? *o + acc[c][e] : acc[c][e];
                            }
                }
        } else {
            // a lane has a row: blocks of 32 x 32 are turned around in the operand stages, which every MMA has left
            float *tb = reinterpret_cast<float *>(s.op) + warp * (32 * 36);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int32_t col = it.n0 + ((warp >> 2) + 4 * c) * 32 + 4 * (lane & 7);
                if ((warp >> 2) + 4 * c < chunks) {
#pragma unroll
                    for (int e = 0; e < 32; e += 4)
                        *reinterpret_cast<float4 *>(tb + lane * 36 + e) = make_float4(acc[c][e], acc[c][e + 1], acc[c][e + 2], acc[c][e + 3]);
                    __syncwarp();
#pragma unroll
                    for (int r = 0; r < 32; r += 4) {
                        const int32_t row_out = it.m0 + q32 + r + (lane >> 3);
                        const float4 v = *reinterpret_cast<const float4 *>(tb + (r + (lane >> 3)) * 36 + 4 * (lane & 7));
                        if (row_out < a.M && col < a.N) {
                            float *o = a.C + (int64_t)row_out * a.ldc + col;
                            if (col + 4 <= a.N) {
                                *reinterpret_cast<float4 *>(o) = v;
                            } else {
                                o[0] = v.x;
                                if (col + 1 < a.N) o[1] = v.y;
                                if (col + 2 < a.N) o[2] = v.z;
                            }
                        }
                    }
                    __syncwarp();
                }
            }
            // every warp has before the first of them converts into the stages again
            if (lane == 0) mbar_arrive(&s.sh->turned);
            if (!mbar_wait_all(&s.sh->turned, turned & 1u, dead, a.status)) return;
            ++turned;
        }
    }
}

template <bool TN, int FMT>
__global__ void __launch_bounds__(MXT_THREADS, 1)
k_mx_gemm(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ MxtArgs a)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    MxtMem s;
    s.op = smem;
    s.raw = smem + MXT_OP * MXT_STAGE;
    s.sh = (MxtShared *)(s.raw + MXT_RAW * MXT_RAW_STAGE);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < MXT_RAW; ++i) {
            mbar_init(&s.sh->raw_full[i], 1);
            mbar_init(&s.sh->raw_empty[i], MXT_WORKERS + (TN ? 1 : 0));
        }
        for (int i = 0; i < MXT_OP; ++i) {
            mbar_init(&s.sh->op_full[i], MXT_WORKERS);
            mbar_init(&s.sh->op_empty[i], 1);
        }
        mbar_init(&s.sh->acc_full, 1);
        mbar_init(&s.sh->acc_empty, MXT_WORKERS);
        mbar_init(&s.sh->turned, MXT_WORKERS);
        s.sh->dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == MXT_WORKERS) tc_alloc<1>(&s.sh->tmem_base, 512u);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    s.tmem = s.sh->tmem_base;
    sat_grid_wait();   // everything above is set-up of this block; no global memory has been touched
    // 640 threads start with 96 registers each; the four warpgroups of workers, which hold 64 sums a thread, go to 104 and the fifth one
    // to 64: 4 x 104 + 64 = 5 x 96
    if (warp < MXT_WORKERS) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
        mxt_work<TN, FMT>(a, s, blockIdx.x, gridDim.x, warp, lane);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (warp == MXT_WORKERS) mxt_mma<TN>(a, s, blockIdx.x, gridDim.x);
        else if (warp == MXT_WORKERS + 1) mxt_load<TN, FMT>(a, s, &map_x, &map_q, blockIdx.x, gridDim.x, lane);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == MXT_WORKERS) {
        tc_fence_after();
        tc_dealloc<1>(s.tmem, 512u);
    }
}

static sat_status mxt_map_q(sat_ctx *ctx, CUtensorMap *map, const sat_mx_matrix *q, int32_t bn)
{
    return sat_tensor_map(ctx, map, CU_TENSOR_MAP_DATA_TYPE_UINT8, q->codes, mx_row_bytes(q), q->rows, q->ld_codes, bn * q->format / 8, MXT_KB, CU_TENSOR_MAP_SWIZZLE_NONE);
}

template <bool TN, int FMT>
static sat_status mxt_launch(sat_ctx *ctx, const CUtensorMap &map_x, const CUtensorMap &map_q, const MxtArgs &a)
{
    static PerDeviceOnce attr;
    if (attr.need(ctx->device)) {
        SAT_CUDA(ctx, cudaFuncSetAttribute(k_mx_gemm<TN, FMT>, cudaFuncAttributeMaxDynamicSharedMemorySize, MXT_SMEM));
        attr.mark(ctx->device);
    }
    sat_pdl(ctx->stream, k_mx_gemm<TN, FMT>, (unsigned)std::min<int64_t>(a.items, ctx->sms), MXT_THREADS, MXT_SMEM)(map_x, map_q, a);
    SAT_LAUNCHED(ctx);
    return SAT_OK;
}

sat_status sat_mx_tc_nn(sat_ctx *ctx, int64_t m, const float *A, int32_t lda, const sat_mx_matrix *W, float *C, int32_t ldc)
{
    MxtArgs a{};
    a.scales = W->scales;
    a.ld_scales = W->ld_scales;
    a.groups = mx_groups(W->d);
    a.M = (int32_t)m;
    a.N = W->d;
    a.K = a.kps = (int32_t)W->rows;
    a.bn = mx_tile_columns(a.N);
    a.tiles_m = (int32_t)cdiv64(m, 128);
    a.tiles_n = (int32_t)cdiv64(a.N, a.bn);
    if ((int64_t)a.tiles_m * a.tiles_n > INT32_MAX / 2) return sat_fail(ctx, SAT_EINVAL, "sat_mx_dense_nn: shape is too large");
    a.items = a.tiles_m * a.tiles_n;
    a.C = C;
    a.ldc = ldc;
    a.status = ctx->d_flag + 1;
    CUtensorMap map_x, map_q;
    SAT_TRY(sat_tensor_map(ctx, &map_x, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, A, W->rows, m, (int64_t)lda * 4, MXT_KB, 128, CU_TENSOR_MAP_SWIZZLE_128B));
    SAT_TRY(mxt_map_q(ctx, &map_q, W, a.bn));
    return W->format == SAT_MX8 ? mxt_launch<false, SAT_MX8>(ctx, map_x, map_q, a) : mxt_launch<false, SAT_MX4>(ctx, map_x, map_q, a);
}

sat_status sat_mx_tc_tn(sat_ctx *ctx, const sat_mx_matrix *A, int32_t n, const float *B, int32_t ldb, float *C, float *colsum, int accumulate)
{
    MxtArgs a{};
    a.scales = A->scales;
    a.ld_scales = A->ld_scales;
    a.groups = mx_groups(A->d);
    a.M = n;
    a.N = A->d;
    a.K = (int32_t)A->rows;
    a.bn = mx_tile_columns(a.N);
    a.tiles_m = (int32_t)cdiv64(n, 128);
    a.tiles_n = (int32_t)cdiv64(a.N, a.bn);
    const int64_t tiles = (int64_t)a.tiles_m * a.tiles_n, stages = cdiv64(a.K, MXT_KB);
    if (tiles > INT32_MAX / 2) return sat_fail(ctx, SAT_EINVAL, "sat_mx_dense_tn: shape is too large");
    const int64_t splits = std::max<int64_t>(1, std::min<int64_t>(ctx->sms / tiles, cdiv64(stages, 4)));
    a.kps = (int32_t)std::min<int64_t>(cdiv64(stages, splits) * MXT_KB, INT32_MAX & ~(MXT_KB - 1));
    const int64_t n_splits = cdiv64(a.K, a.kps);
    a.items = (int32_t)(tiles * n_splits);
    a.direct = n_splits == 1;
    a.accumulate = accumulate;
    a.status = ctx->d_flag + 1;
    if (a.direct) {
        a.C = C;
        a.colsum = colsum;
    } else {
        SAT_TRY(sat_ensure(ctx, ctx->buf_splitk, (size_t)n_splits * ((size_t)a.N * n + n) * sizeof(float)));
        a.C = (float *)ctx->buf_splitk.p;
        a.colsum = colsum ? a.C + (size_t)n_splits * a.N * n : nullptr;
    }
    CUtensorMap map_x, map_q;
    SAT_TRY(sat_tensor_map(ctx, &map_x, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, B, n, A->rows, (int64_t)ldb * 4, 32, MXT_KB, CU_TENSOR_MAP_SWIZZLE_128B));
    SAT_TRY(mxt_map_q(ctx, &map_q, A, a.bn));
    SAT_TRY((A->format == SAT_MX8 ? mxt_launch<true, SAT_MX8>(ctx, map_x, map_q, a) : mxt_launch<true, SAT_MX4>(ctx, map_x, map_q, a)));
    if (a.direct) return SAT_OK;
    return sat_splitk_reduce(ctx, a.C, (int64_t)a.N * n, (int32_t)n_splits, accumulate, C, n, n, a.colsum, n, colsum);
}

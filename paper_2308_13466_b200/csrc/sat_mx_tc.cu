// Contractions of fp32 rows with microscaled matrices on the 5th-generation tensor cores.
//     k_mx_gemm<true>    C[q.d x n] = Q^^T X     sat_mx_dense_tn: the terms run over the rows of both, split over CTA pairs
//     k_mx_gemm<false>   C[m x q.d] = X Q^       sat_mx_dense_nn: the terms run over the columns of X and the rows of Q
// What a code stands for has four significant bits and a power of two, so it is a bf16 number.  An fp32 operand is cut into three bf16
// terms by taking the upper half of its bits off twice, which is exact: x = hi + mid + lo, eight bits each.  Three MMAs of
// kind::f16 with bf16 operands then give exact products, and all that is rounded is the sum.
//
// The tensor core chops its running sum at every instruction (16 terms), always towards zero, so a sum in one accumulator drifts:
// about a third of a unit of 2^-23 per instruction.  Only the products with hi matter for that; those with mid and lo are 2^-8 of them and
// have an accumulator of their own.  The hi accumulator is taken out after MXT_FLUSH stages (24 instructions) and added up in registers,
// rounded to nearest; relative error 3e-7 to 1e-6, about that of an fp32 FMA loop.
//
// A pair of CTAs shares a tile of 256 columns of Q (the M side, 128 lanes of TMEM in either CTA) by up to 256 columns (TN) or rows (NN) of
// X.  What bounds it besides memory is shared memory, at 128 bytes a clock: per stage of 32 terms a CTA takes in 16 KB of X and 4 KB of codes
// (written by TMA, read once), writes 24 KB and 8 KB of bf16, and the tensor core reads 32 KB (each CTA holds one half of X, and a tile of Q
// stays in the operand collector for its three products): 104 KB, 830 clocks, against 768 for the MMAs.  With single CTAs and X as the M side it
// was 183 KB for as many products.
//
// 20 warps.  Warps 0..15 convert, in two groups on alternate stages, and hold the sums; warp 16 of the first CTA issues the MMAs; warp 17 the
// loads; warps 18 and 19 add up the columns of X where the bias gradient is asked for.
#include "sat_mx.h"
#include "sat_ptx.h"

#include <algorithm>

#define MXT_WORKERS 16
#define MXT_THREADS ((MXT_WORKERS + 4) * 32)   /* five whole warpgroups, see k_mx_gemm */
#define MXT_KB 32                    /* terms per stage */
#define MXT_RAW 6                    /* stages of raw tiles; an even number, so that either group keeps to its own */
#define MXT_OP 3                     /* stages of converted tiles */
#define MXT_FLUSH 12                 /* stages between two reads of the hi accumulator */
#define MXT_Q_TILE (128 * MXT_KB * 2)
#define MXT_X_PLANE (128 * MXT_KB * 2)
#define MXT_STAGE (MXT_Q_TILE + 3 * MXT_X_PLANE)
#define MXT_X_RAW (128 * MXT_KB * 4)
#define MXT_Q_RAW (128 * MXT_KB)
#define MXT_RAW_STAGE (MXT_X_RAW + MXT_Q_RAW)
#define MXT_SCALES (MXT_KB * 4)       /* of a stage: four groups a term */

struct MxtShared {
    double sums[128];
    uint64_t sums_full, sums_empty;
    uint8_t scales[MXT_RAW][MXT_SCALES];
    uint64_t raw_full[MXT_RAW], raw_empty[MXT_RAW];   // TMA bytes and scales have landed; a group of workers (and the column sums) has read them
    uint64_t op_full[MXT_OP], op_empty[MXT_OP];     // (first CTA) both CTAs' workers have written the tiles; the MMAs have read them
    uint64_t acc_full, acc_empty;                       // the hi accumulator is to be taken out; (first CTA) both CTAs have
    uint32_t tmem_base;
    int dead;
};
#define MXT_SMEM (1024 + MXT_OP * MXT_STAGE + MXT_RAW * MXT_RAW_STAGE + (int)sizeof(MxtShared))
static_assert(MXT_SMEM <= 227 * 1024, "shared memory");

struct MxtArgs {
    const uint8_t *scales;
    int64_t ld_scales;
    int32_t groups;            // of a row of Q
    int32_t D, N;              // columns of Q; columns (TN) or rows (NN) of X
    int32_t K, kps;            // terms, and terms of a split (a multiple of MXT_KB)
    int32_t bn, tiles_d, tiles_n;
    int32_t items;             // tiles times splits, the tiles of a split next to each other
    float *C;                  // element (column j of Q, column or row i of X) of split z at C + z split + i by_x + j by_q
    int64_t split, by_x, by_q;
    float *colsum;             // TN: [splits][N] column sums of X, or none
    int add;                   // to what is there
    int *status;
};
// A tile and its terms [k0, k1)
struct MxtItem {
    int32_t d0, n0, split, k0, k1, stages;
};
__device__ __forceinline__ MxtItem mxt_item(const MxtArgs &a, int32_t i)
{
    MxtItem t;
    const int32_t tiles = a.tiles_d * a.tiles_n, tile = i % tiles;
    t.split = i / tiles;
    t.d0 = tile % a.tiles_d * 256;
    t.n0 = tile / a.tiles_d * a.bn;
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
    return 1u << 4 | 1u << 7 | 1u << 10 | 1u << 15 | (TN ? 1u << 16 : 0u) | (uint32_t)(bn >> 3) << 17 | (256u >> 4) << 24;
}

// Waits like mbar_wait_all, but the hardware may put the warp aside for up to a microsecond a time: what waits here would take issue slots
// from the warps that convert, which are bound by them
__device__ __forceinline__ bool mxt_wait(uint64_t *bar, uint32_t parity, volatile int *dead, int *status)
{
    const uint32_t addr = smem_u32(bar);
    for (uint32_t it = 0; it < TC_WAIT_LIMIT; ++it) {
        uint32_t ok;
        asm volatile(
            "{\n\t"
            ".reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t"
            "}"
            : "=r"(ok)
            : "r"(addr), "r"(parity), "r"(1000u)
            : "memory");
        if (__all_sync(0xffffffffu, ok)) return true;
        if (__any_sync(0xffffffffu, *dead)) return false;
    }
    *dead = 1;
    atomicOr(status, 1);
    return false;
}

// ---- the roles --------------------------------------------------------------------------------------------------------------
struct MxtMem {
    uint8_t *op, *raw;
    MxtShared *sh;
    uint32_t tmem;
    int32_t rank;              // CTA of the pair
    int32_t unit, units;       // pair, and pairs
};

template <bool TN>
__device__ __forceinline__ void mxt_mma(const MxtArgs &a, const MxtMem &s)
{
    volatile int *dead = &s.sh->dead;
    const uint32_t idesc = mxt_idesc<TN>(a.bn), hi = s.tmem, rest = s.tmem + 256u;
    // MN-major tiles: blocks of 64 columns (128 bytes a term, 128-byte swizzle) MXT_KB x 128 bytes apart, groups of eight terms 1024 bytes
    // apart; an instruction takes 16 terms.  K-major (X without TN): a row's 32 terms are 64 bytes, 64-byte swizzle, eight rows 512 apart.
    const uint64_t q0 = make_desc(smem_u32(s.op), MXT_KB * 128, 1024, 2);
    const uint64_t x0 = TN ? make_desc(smem_u32(s.op) + MXT_Q_TILE, MXT_KB * 128, 1024, 2) : make_desc(smem_u32(s.op) + MXT_Q_TILE, 16, 512, 4);
    constexpr uint32_t x_step = (TN ? 2048 : 32) >> 4, q_step = 2048 >> 4, plane = MXT_X_PLANE >> 4;
    uint32_t st = 0, ph = 0, taken = 0;   // taken: times the accumulators were handed over
    for (int32_t i = s.unit; i < a.items; i += s.units) {
        const int32_t stages = mxt_item(a, i).stages;
        int32_t in_run = 0;               // stages since the hi accumulator was last handed over
        for (int32_t k = 0; k < stages; ++k) {
            if (!mxt_wait(&s.sh->op_full[st], ph, dead, a.status)) return;
            // (acc_empty's phase `taken - 1` completes when the workers have read what was handed over last)
            if (k == 0 && taken > 0 && !mxt_wait(&s.sh->acc_empty, (taken - 1) & 1u, dead, a.status)) return;
            tc_fence_after();
            const uint64_t q = q0 + (uint64_t)(st * (MXT_STAGE >> 4)), x = x0 + (uint64_t)(st * (MXT_STAGE >> 4));
            const bool run_starts = in_run == 0 && k > 0, hand_over = ++in_run == MXT_FLUSH || k + 1 == stages;
            if (!run_starts) {
                if (elect_one()) {
#pragma unroll
                    for (uint32_t ks = 0; ks < MXT_KB / 16; ++ks) {   // the tile of Q stays in the collector for its three products
                        tc_mma_f16<1, 2>(rest, q + ks * q_step, x + ks * x_step + plane, idesc, k > 0 || ks > 0 ? 1u : 0u);
                        tc_mma_f16<3, 2>(rest, q + ks * q_step, x + ks * x_step + 2 * plane, idesc, 1u);
                        tc_mma_f16<2, 2>(hi, q + ks * q_step, x + ks * x_step, idesc, k > 0 || ks > 0 ? 1u : 0u);
                    }
                }
            } else {   // mid and lo go ahead while the hi accumulator is still being read
                if (elect_one()) {
#pragma unroll
                    for (uint32_t ks = 0; ks < MXT_KB / 16; ++ks) {
                        tc_mma_f16<1, 2>(rest, q + ks * q_step, x + ks * x_step + plane, idesc, 1u);
                        tc_mma_f16<2, 2>(rest, q + ks * q_step, x + ks * x_step + 2 * plane, idesc, 1u);
                    }
                }
                __syncwarp();
                if (!mxt_wait(&s.sh->acc_empty, (taken - 1) & 1u, dead, a.status)) return;
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (uint32_t ks = 0; ks < MXT_KB / 16; ++ks) tc_mma_f16<0, 2>(hi, q + ks * q_step, x + ks * x_step, idesc, ks > 0 ? 1u : 0u);
                }
            }
            __syncwarp();
            if (elect_one()) {
                tc_commit<2>(&s.sh->op_empty[st]);
                if (hand_over) tc_commit<2>(&s.sh->acc_full);
            }
            __syncwarp();
            if (hand_over) ++taken, in_run = 0;
            if (++st == MXT_OP) st = 0, ph ^= 1u;
        }
    }
}

// TMA loads and, a term per lane, asynchronous copies of the scales, up to MXT_RING stages ahead of the workers
template <bool TN, int FMT>
__device__ __forceinline__ void mxt_load(const MxtArgs &a, const MxtMem &s, const CUtensorMap *map_x, const CUtensorMap *map_q, int lane)
{
    volatile int *dead = &s.sh->dead;
    const int32_t half = a.bn / 2;
    uint32_t st = 0, ph = 0, total = 0;
    for (int32_t i = s.unit; i < a.items; i += s.units) {
        const MxtItem it = mxt_item(a, i);
        const int32_t x0 = it.n0 + s.rank * half, q0 = it.d0 + s.rank * 128;
        const int32_t boxes = x0 >= a.N ? 0 : !TN ? 1 : min((a.N - x0 + 31) / 32, half / 32);
        const bool has_q = q0 < a.D;
        const uint32_t bytes = (uint32_t)boxes * (TN ? 4096u : (uint32_t)half * 128u) + (has_q ? 128u * MXT_KB * FMT / 8 : 0u);
        const uint8_t *scales = a.scales + (int64_t)(it.k0 + lane) * a.ld_scales + q0 / MX_GROUP;   // four bytes, of which some may lie behind the row's last
        for (int32_t k = it.k0; k < it.k1; k += MXT_KB, ++total, scales += MXT_KB * a.ld_scales) {
            if (!mxt_wait(&s.sh->raw_empty[st], ph ^ 1u, dead, a.status)) return;
            uint64_t *bar = &s.sh->raw_full[st];
            if (lane == 0) {
                uint8_t *x = s.raw + (size_t)st * MXT_RAW_STAGE;
                mbar_expect_tx(bar, bytes);
                if (TN)
                    for (int b = 0; b < boxes; ++b) tma_load_2d(x + b * 4096, map_x, bar, x0 + 32 * b, k);
                else if (boxes) tma_load_2d(x, map_x, bar, k, x0);
                if (has_q) tma_load_2d(x + MXT_X_RAW, map_q, bar, q0 / 8 * FMT, k);
            }
            __syncwarp();
            const bool there = has_q && k + lane < it.k1;   // (else four zero bytes and nothing read)
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(s.sh->scales[st] + 4 * lane)), "l"(there ? scales : a.scales), "r"(there ? 4u : 0u) : "memory");
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
            if (++st == MXT_RAW) st = 0, ph ^= 1u;
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    // the pair's MMAs have signalled every stage: nothing arrives here any more once both CTAs may exit
    for (uint32_t i = 0; i < MXT_OP; ++i) {
        const uint32_t uses = (total + MXT_OP - 1 - i) / MXT_OP;
        if (uses > 0 && !mxt_wait(&s.sh->op_empty[i], (uses - 1) & 1u, dead, a.status)) return;
    }
}

// The column sums of X (TN), four columns a lane: half a stage in fp32, the stages in doubles.  Two warps, with one half of every stage's terms each
// (one alone took longer over a stage than everything else); the second one leaves its sums to the first.
__device__ __forceinline__ void mxt_sums(const MxtArgs &a, const MxtMem &s, int part, int lane)
{
    volatile int *dead = &s.sh->dead;
    const int32_t half = a.bn / 2, mine = (lane >> 3) * 32;
    uint32_t st = 0, ph = 0, turn = 0;
    for (int32_t i = s.unit; i < a.items; i += s.units) {
        const MxtItem it = mxt_item(a, i);
        const int32_t x0 = it.n0 + s.rank * half;
        const bool sums = it.d0 == 0, here = sums && mine < half && x0 + mine < a.N;
        double c[4] = {0., 0., 0., 0.};
        for (int32_t k = 0; k < it.stages; ++k) {
            if (!mxt_wait(&s.sh->raw_full[st], ph, dead, a.status)) return;
            if (here) {
                const uint8_t *x = s.raw + st * MXT_RAW_STAGE + (lane >> 3) * 4096 + part * (MXT_KB / 2 * 128);
                float2 t = make_float2(0.f, 0.f), u = t;
#pragma unroll
                for (int r = 0; r < MXT_KB / 2; ++r) {
                    const float4 v = *reinterpret_cast<const float4 *>(x + r * 128 + (((lane & 7) ^ (r & 7)) << 4));
                    t = __fadd2_rn(t, make_float2(v.x, v.y));
                    u = __fadd2_rn(u, make_float2(v.z, v.w));
                }
                c[0] += t.x;
                c[1] += t.y;
                c[2] += u.x;
                c[3] += u.y;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&s.sh->raw_empty[st]);
            if (++st == MXT_RAW) st = 0, ph ^= 1u;
        }
        if (!sums) continue;
        double *slot = s.sh->sums + 4 * lane;
        if (part == 1) {
            if (!mxt_wait(&s.sh->sums_empty, (turn & 1u) ^ 1u, dead, a.status)) return;
            for (int j = 0; j < 4; ++j) slot[j] = c[j];
            __syncwarp();
            if (lane == 0) mbar_arrive(&s.sh->sums_full);
        } else {
            if (!mxt_wait(&s.sh->sums_full, turn & 1u, dead, a.status)) return;
            for (int j = 0; j < 4; ++j) {
                const int32_t col = x0 + 4 * lane + j;
                const double both = c[j] + slot[j];
                if (!here || 4 * lane + j >= half || col >= a.N) continue;
                float *out = a.colsum + (int64_t)it.split * a.N + col;
                *out = a.add ? (float)((double)*out + both) : (float)both;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&s.sh->sums_empty);
        }
        ++turn;
    }
}

template <bool TN, int FMT>
__device__ __forceinline__ void mxt_work(const MxtArgs &a, const MxtMem &s, int warp, int lane)
{
    volatile int *dead = &s.sh->dead;
    const uint32_t group = (uint32_t)warp >> 3;
    const int w = warp & 7;
    const int32_t half = a.bn / 2;
    // 16 elements of Q and twice eight values of X per thread and stage.  Terms and places along a row go over the lanes so that eight
    // lanes in turn touch all banks, in the raw rows as in the swizzled ones.
    const int j = (lane >> 2) & 1, term = 4 * w + 2 * (lane >> 4) + (j ^ ((lane >> 3) & 1)), place = (lane & 3) | j << 2;
    const uint32_t q_raw = MXT_X_RAW + (uint32_t)(term * 128 + 16 * place) * FMT / 8;
    const uint32_t q_op = (uint32_t)(place >> 2) * (MXT_KB * 128) + (uint32_t)term * 128u + ((uint32_t)((2 * (place & 3)) ^ (term & 7)) << 4);
    // TN: columns 8 place .. of the term, and 64 columns on.  NN: terms 8 (lane % 4) .. of a row, and of the row 64 on.
    const int row = 8 * w + (lane >> 2), quad = lane & 3;
    const uint32_t x_raw = TN ? (uint32_t)(place >> 2) * 4096u + (uint32_t)term * 128u + ((uint32_t)((2 * (place & 3)) ^ (term & 7)) << 4)
                              : (uint32_t)row * 128u + ((uint32_t)((2 * quad) ^ (row & 7)) << 4);
    const uint32_t x_op = MXT_Q_TILE + (TN ? (uint32_t)term * 128u + ((uint32_t)(place ^ (term & 7)) << 4) : (uint32_t)row * 64u + ((uint32_t)(quad ^ ((row >> 1) & 3)) << 4));
    constexpr uint32_t x_raw2 = 8192u, x_op2 = 4096u;    // the second eight: two boxes, or 64 rows, further on
    const int32_t x_first = TN ? 8 * place : row;        // its index within the CTA's half; the second is 64 further on
    const int32_t chunks = a.bn / 32, slice = warp >> 2; // 32 columns of the accumulators each: chunks slice and slice + 4 are this warp's
    const uint32_t lanes = s.tmem + ((uint32_t)((warp & 3) * 32) << 16);

    float acc[2][32];
#pragma unroll
    for (int c = 0; c < 64; ++c) acc[c >> 5][c & 31] = 0.f;
    uint32_t taken = 0;
    auto take = [&](bool last) -> bool {
        if (!mxt_wait(&s.sh->acc_full, taken & 1u, dead, a.status)) return false;
        tc_fence_after();
#pragma unroll
        for (int c = 0; c < 2; ++c)
            if (slice + 4 * c < chunks) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t r[16];
                    tc_ld16(lanes + (uint32_t)(slice + 4 * c) * 32u + 16u * h, r);
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[c][16 * h + e] += __uint_as_float(r[e]);
                    if (last) {
                        tc_ld16(lanes + 256u + (uint32_t)(slice + 4 * c) * 32u + 16u * h, r);
#pragma unroll
                        for (int e = 0; e < 16; ++e) acc[c][16 * h + e] += __uint_as_float(r[e]);
                    }
                }
            }
        tc_fence_before();
        mbar_arrive_warp<2>(&s.sh->acc_empty, lane);
        ++taken;
        return true;
    };
    // A lane has a column of Q, a register a column or row of X: consecutive lanes write consecutive floats
    auto finish = [&](int32_t item) -> bool {
        if (!take(true)) return false;
        const MxtItem it = mxt_item(a, item);
        const int32_t col = it.d0 + s.rank * 128 + (warp & 3) * 32 + lane;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int32_t first = it.n0 + (slice + 4 * c) * 32;
            float *o = a.C + it.split * a.split + first * a.by_x + col * a.by_q;
            if (slice + 4 * c < chunks && col < a.D) {
                if (first + 32 <= a.N && !(TN && a.add)) {
#pragma unroll
                    for (int e = 0; e < 32; ++e, o += a.by_x) *o = acc[c][e];
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e, o += a.by_x)
                        if (first + e < a.N) *o = TN && a.add ? *o + acc[c][e] : acc[c][e];
                }
            }
#pragma unroll
            for (int e = 0; e < 32; ++e) acc[c][e] = 0.f;
        }
        return true;
    };

    uint32_t base = 0;      // parity of the stages before this item
    uint32_t rs = group, rph = 0, os = group, oph = 0;
    int32_t pending = -1;   // the item that is to be finished
    for (int32_t i = s.unit;; i += s.units) {
        MxtItem it{};       // (no stages behind the last one)
        if (i < a.items) it = mxt_item(a, i);
        const bool has_q = it.d0 + s.rank * 128 + 16 * place < a.D;
        const int32_t x0 = it.n0 + s.rank * half + x_first;
        const bool has_x = x_first < half && x0 < a.N, has_x2 = x_first + 64 < half && x0 + 64 < a.N;
        int32_t run_end = MXT_FLUSH;
#pragma unroll 1
        for (int32_t k = (int32_t)(group ^ base);; k += 2) {
            if (k < it.stages) {
                if (!mxt_wait(&s.sh->raw_full[rs], rph, dead, a.status)) return;
                if (!mxt_wait(&s.sh->op_empty[os], oph ^ 1u, dead, a.status)) return;
                const uint8_t *raw = s.raw + rs * MXT_RAW_STAGE;
                uint8_t *op = s.op + os * MXT_STAGE;
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if (h ? has_x2 : has_x) {
                        uint4 hi, mid, lo;
                        mxt_split8(*reinterpret_cast<const float4 *>(raw + x_raw + h * x_raw2), *reinterpret_cast<const float4 *>(raw + (x_raw ^ 16u) + h * x_raw2), hi, mid, lo);
                        uint8_t *o = op + x_op + h * x_op2;
                        *reinterpret_cast<uint4 *>(o) = hi;
                        *reinterpret_cast<uint4 *>(o + MXT_X_PLANE) = mid;
                        *reinterpret_cast<uint4 *>(o + 2 * MXT_X_PLANE) = lo;
                    }
                if (has_q) {
                    const MxtScale<FMT> sc(s.sh->scales[rs][4 * term + (place >> 1)]);
                    uint4 v0, v1;
                    if (FMT == SAT_MX8) {
                        const uint4 c = *reinterpret_cast<const uint4 *>(raw + q_raw);
                        v0 = mxt_decode8<FMT>(c.x, c.y, sc), v1 = mxt_decode8<FMT>(c.z, c.w, sc);
                    } else {
                        const uint2 c = *reinterpret_cast<const uint2 *>(raw + q_raw);
                        v0 = mxt_decode8<FMT>(c.x, 0u, sc), v1 = mxt_decode8<FMT>(c.y, 0u, sc);
                    }
                    if (sc.two) v0 = bf16x8_mul(v0, sc.second), v1 = bf16x8_mul(v1, sc.second);
                    *reinterpret_cast<uint4 *>(op + q_op) = v0;
                    *reinterpret_cast<uint4 *>(op + (q_op ^ 16u)) = v1;
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&s.sh->raw_empty[rs]);
                mbar_arrive_warp<2>(&s.sh->op_full[os], lane);
                if ((rs += 2) >= MXT_RAW) rs -= MXT_RAW, rph ^= 1u;
                if ((os += 2) >= MXT_OP) os -= MXT_OP, oph ^= 1u;
            }
            // Accumulators are taken out a stage late, so that the MMAs have something to do meanwhile
            if (pending >= 0) {
                if (!finish(pending)) return;
                pending = -1;
            }
            for (; run_end < it.stages && run_end <= k; run_end += MXT_FLUSH)
                if (!take(false)) return;
            if (k >= it.stages) break;
        }
        if (i >= a.items) return;
        base ^= (uint32_t)it.stages & 1u;
        pending = i;
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
    s.rank = (int32_t)(blockIdx.x & 1u);
    s.unit = (int32_t)(blockIdx.x >> 1);
    s.units = (int32_t)(gridDim.x >> 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < MXT_RAW; ++i) {
            mbar_init(&s.sh->raw_full[i], 1 + 32);            // the TMA's issuer and the scales' lanes
            mbar_init(&s.sh->raw_empty[i], MXT_WORKERS / 2 + (TN && a.colsum ? 2 : 0));
        }
        for (int i = 0; i < MXT_OP; ++i) {
            mbar_init(&s.sh->op_full[i], MXT_WORKERS);        // a group of either CTA
            mbar_init(&s.sh->op_empty[i], 1);
        }
        mbar_init(&s.sh->acc_full, 1);
        mbar_init(&s.sh->sums_full, 1);
        mbar_init(&s.sh->sums_empty, 1);
        mbar_init(&s.sh->acc_empty, 2 * MXT_WORKERS);
        s.sh->dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == MXT_WORKERS) tc_alloc<2>(&s.sh->tmem_base, 512u);
    tc_fence_before();
    __syncthreads();
    cluster_sync();   // the other CTA's barriers are initialised and its TMEM is allocated
    tc_fence_after();
    s.tmem = s.sh->tmem_base;
    sat_grid_wait();   // everything above is set-up of this block; no global memory has been touched
    // 640 threads start with 96 registers each; the four warpgroups of workers, which hold 64 sums a thread, go to 104 and the fifth one
    // to 64: 4 x 104 + 64 = 5 x 96
    if (warp < MXT_WORKERS) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
        mxt_work<TN, FMT>(a, s, warp, lane);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (warp == MXT_WORKERS && s.rank == 0) mxt_mma<TN>(a, s);
        else if (warp == MXT_WORKERS + 1) mxt_load<TN, FMT>(a, s, &map_x, &map_q, lane);
        else if (TN && warp >= MXT_WORKERS + 2 && a.colsum) mxt_sums(a, s, warp - (MXT_WORKERS + 2), lane);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    cluster_sync();   // neither CTA's shared memory or TMEM is in use by the other any more
    if (warp == MXT_WORKERS) {
        tc_fence_after();
        tc_dealloc<2>(s.tmem, 512u);
    }
}

// C[j][i] (+)= sum over the splits of part[z][i][j], cs[i] (+)= that of part_cs[z][i], in a fixed order: 32 columns of Q by eight of X per block,
// four threads to an element
__global__ void __launch_bounds__(1024)
k_mx_reduce(const float *__restrict__ part, const float *__restrict__ part_cs, int32_t splits, int32_t D, int32_t N, int add, float *__restrict__ C, float *__restrict__ colsum)
{
    sat_grid_wait();
    __shared__ float red[4][8][33];
    const int lane = threadIdx.x & 31, i = (threadIdx.x >> 5) & 7, z4 = threadIdx.x >> 8;
    const int32_t col = (int32_t)blockIdx.x * 32 + lane, row = (int32_t)blockIdx.y * 8 + i;
    const int64_t plane = (int64_t)D * N;
    float t = 0.f;
    if (col < D && row < N) {
        const float *p = part + (int64_t)row * D + col;
#pragma unroll 8
        for (int32_t z = z4; z < splits; z += 4) t += __ldg(p + z * plane);
    }
    red[z4][i][lane] = t;
    __syncthreads();
    if (threadIdx.x < 256) {
        const int jj = threadIdx.x >> 3, ii = threadIdx.x & 7;   // eight lanes write eight consecutive floats of a row of C
        const int32_t c = (int32_t)blockIdx.x * 32 + jj, r = (int32_t)blockIdx.y * 8 + ii;
        if (c < D && r < N) {
            const float sum = (red[0][ii][jj] + red[1][ii][jj]) + (red[2][ii][jj] + red[3][ii][jj]);
            float *o = C + (int64_t)c * N + r;
            *o = add ? *o + sum : sum;
        }
    } else if (threadIdx.x < 264 && blockIdx.x == 0 && colsum) {
        const int32_t r = (int32_t)blockIdx.y * 8 + (int32_t)threadIdx.x - 256;
        if (r < N) {
            double sum = 0.;
            for (int32_t z = 0; z < splits; ++z) sum += (double)__ldg(part_cs + (int64_t)z * N + r);
            colsum[r] = add ? (float)((double)colsum[r] + sum) : (float)sum;
        }
    }
}

template <bool TN, int FMT>
static sat_status mxt_launch(sat_ctx *ctx, const CUtensorMap &map_x, const CUtensorMap &map_q, const MxtArgs &a)
{
    static PerDeviceOnce attr;
    if (attr.need(ctx->device)) {
        SAT_CUDA(ctx, cudaFuncSetAttribute(k_mx_gemm<TN, FMT>, cudaFuncAttributeMaxDynamicSharedMemorySize, MXT_SMEM));
        attr.mark(ctx->device);
    }
    sat_pdl(ctx->stream, k_mx_gemm<TN, FMT>, 2u * (unsigned)std::min(a.items, ctx->sms / 2), MXT_THREADS, MXT_SMEM, 2)(map_x, map_q, a);
    SAT_LAUNCHED(ctx);
    return SAT_OK;
}

// what both have in common
static sat_status mxt_args(sat_ctx *ctx, const sat_mx_matrix *q, int64_t n, int32_t bn, MxtArgs *a, CUtensorMap *map_q)
{
    a->scales = q->scales;
    a->ld_scales = q->ld_scales;
    a->groups = mx_groups(q->d);
    a->D = q->d;
    a->N = (int32_t)n;
    a->K = a->kps = (int32_t)q->rows;
    a->bn = bn;
    a->tiles_d = (int32_t)cdiv64(q->d, 256);
    a->tiles_n = (int32_t)cdiv64(n, bn);
    if ((int64_t)a->tiles_d * a->tiles_n > INT32_MAX / 2) return sat_fail(ctx, SAT_EINVAL, "microscaled contraction: shape is too large");
    a->items = a->tiles_d * a->tiles_n;
    a->status = ctx->d_flag + 1;
    return sat_tensor_map(ctx, map_q, CU_TENSOR_MAP_DATA_TYPE_UINT8, q->codes, mx_row_bytes(q), q->rows, q->ld_codes, 128 * q->format / 8, MXT_KB, CU_TENSOR_MAP_SWIZZLE_NONE);
}

sat_status sat_mx_tc_nn(sat_ctx *ctx, int64_t m, const float *A, int32_t lda, const sat_mx_matrix *W, float *C, int32_t ldc)
{
    // 256 rows a tile, or fewer where that leaves pairs of SMs without one
    int32_t bn = 256;
    while (bn > 64 && cdiv64(W->d, 256) * cdiv64(m, bn) < ctx->sms / 2) bn /= 2;
    MxtArgs a{};
    CUtensorMap map_x, map_q;
    SAT_TRY(mxt_args(ctx, W, m, bn, &a, &map_q));
    a.C = C;
    a.by_x = ldc;
    a.by_q = 1;
    SAT_TRY(sat_tensor_map(ctx, &map_x, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, A, W->rows, m, (int64_t)lda * 4, MXT_KB, bn / 2, CU_TENSOR_MAP_SWIZZLE_128B));
    return W->format == SAT_MX8 ? mxt_launch<false, SAT_MX8>(ctx, map_x, map_q, a) : mxt_launch<false, SAT_MX4>(ctx, map_x, map_q, a);
}

sat_status sat_mx_tc_tn(sat_ctx *ctx, const sat_mx_matrix *A, int32_t n, const float *B, int32_t ldb, float *C, float *colsum, int accumulate)
{
    const int32_t tiles_n = (int32_t)cdiv64(n, 256), bn = (int32_t)cdiv64(cdiv64(n, tiles_n), 64) * 64;
    MxtArgs a{};
    CUtensorMap map_x, map_q;
    SAT_TRY(mxt_args(ctx, A, n, bn, &a, &map_q));
    // Row splits: what takes the fewest stages in a row on the busiest pair, a split costing about six stages to set up and to add up
    const int64_t units = ctx->sms / 2, tiles = a.items, stages = cdiv64(A->rows, MXT_KB);
    int64_t best = 1, best_cost = INT64_MAX;
    for (int64_t s = 1; s <= std::min<int64_t>(2 * units / tiles + 1, cdiv64(stages, 4)); ++s) {
        const int64_t cost = cdiv64(tiles * s, units) * (cdiv64(stages, s) + 6);
        if (cost < best_cost) best = s, best_cost = cost;
    }
    a.kps = (int32_t)std::min<int64_t>(cdiv64(stages, best) * MXT_KB, INT32_MAX & ~(MXT_KB - 1));
    const int32_t splits = (int32_t)cdiv64(A->rows, a.kps);
    a.items *= splits;
    if (splits == 1) {
        a.C = C;
        a.by_x = 1;
        a.by_q = n;
        a.add = accumulate;
        a.colsum = colsum;
    } else {
        a.split = (int64_t)a.D * n;
        SAT_TRY(sat_ensure(ctx, ctx->buf_splitk, (size_t)splits * (size_t)(a.split + n) * sizeof(float)));
        a.C = (float *)ctx->buf_splitk.p;
        a.by_x = a.D;
        a.by_q = 1;
        a.colsum = colsum ? a.C + splits * a.split : nullptr;
    }
    SAT_TRY(sat_tensor_map(ctx, &map_x, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, B, n, A->rows, (int64_t)ldb * 4, 32, MXT_KB, CU_TENSOR_MAP_SWIZZLE_128B));
    SAT_TRY((A->format == SAT_MX8 ? mxt_launch<true, SAT_MX8>(ctx, map_x, map_q, a) : mxt_launch<true, SAT_MX4>(ctx, map_x, map_q, a)));
    if (splits == 1) return SAT_OK;
    if (cdiv64(n, 8) > 65535) return sat_fail(ctx, SAT_EINVAL, "sat_mx_dense_tn: shape is too large");
    sat_pdl(ctx->stream, k_mx_reduce, dim3((unsigned)cdiv64(a.D, 32), (unsigned)cdiv64(n, 8)), 1024, 0)(a.C, a.colsum, splits, a.D, n, accumulate, C, colsum);
    SAT_LAUNCHED(ctx);
    return SAT_OK;
}

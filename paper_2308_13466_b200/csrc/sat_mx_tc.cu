// Contractions of fp32 rows with microscaled matrices on the 5th-generation tensor cores.
//     k_mx_gemm<true>    C[q.d x n] = Q^^T X     sat_mx_dense_tn: the terms run over the rows of both, split over CTA pairs
//     k_mx_gemm<false>   C[m x q.d] = X Q^       sat_mx_dense_nn: the terms run over the columns of X and the rows of Q
// What a code stands for has four significant bits and a power of two, so it is a bf16 number.  An fp32 operand is cut into three bf16
// terms by taking the upper half of its bits off twice, which is exact: x = hi + mid + lo, eight bits each.  Three MMAs of
// kind::f16 with bf16 operands then give exact products, and all that is rounded is the sum.
//
// The tensor core chops its running sum at every instruction (16 terms), always towards zero, so a sum in one accumulator drifts: 612257 terms in 74
// splits were off by 1e-5 of the result.  Only the products with hi matter for that; those with mid and lo, 2^-8 of them, have an accumulator of their own,
// and the one of hi is taken out every 12 stages (24 instructions; NN: 16) and added up in registers, rounded to nearest: 5e-7 (2-norm against
// 64 bits; an fp32 product of the library 9e-7).
// The other one follows every 32 runs: a million terms of one sign in one split were off by 4e-5 where it was taken out at their end only.
//
// A pair of CTAs shares a tile of 256 columns of Q (the M side, 128 lanes of TMEM in either CTA) by up to 256 columns (TN) or rows (NN) of
// X.  What bounds it besides memory is shared memory, at 128 bytes a clock: per stage of 32 terms a CTA takes in 16 KB of X and 4 KB of codes
// (written by TMA, read once), writes 24 KB and 8 KB of bf16, and the tensor core reads 32 KB (each CTA holds one half of X, and a tile of Q
// stays in the operand collector for its three products): 104 KB, 830 clocks, against 768 for the MMAs.  (With single CTAs and X as the M side it
// was 183 KB for as many products.  Loading straight into registers takes 40 KB less, but what it can keep in flight does not cover the latency.)
// Measured: 1,020 clocks a stage with TN, 1,130 without, the tensor pipe busy 72 and 64 % of the time; what fills the rest is the chain from a load to its MMAs, which
// is as long for narrow tiles (no counter names one part of it).  612257 x 256 by 256 226 us, 179250 x 512 x 512 278, back to back under the power limit; 199 and 239
// with pauses.
//
// (For NN, one accumulator of all three products, two of them by turns, taken out by four warps that write at once: 90000 x 512 x 512 108 us instead of 128, but
// 96 chopped additions, 1.3e-6.)
//
// Two groups of four warps convert stages in turn; eight warps take the accumulators out and hold the sums of the runs (converters that held them as well had no
// registers left to work with); one, of the first CTA, issues the MMAs, one the loads, and with TN one adds up the column sums that the converters made on the
// way.
#include "sat_mx.h"
#include "sat_ptx.h"

#include <algorithm>

#define MXT_SLOTS 4                  /* stages of raw and of converted tiles */
#define MXT_KB 32                    /* terms per stage */
#define MXT_Q_TILE (128 * MXT_KB * 2)
#define MXT_X_PLANE (128 * MXT_KB * 2)
#define MXT_STAGE (MXT_Q_TILE + 3 * MXT_X_PLANE)
#define MXT_X_RAW (128 * MXT_KB * 4)
#define MXT_Q_RAW (128 * MXT_KB)
#define MXT_RAW_STAGE (MXT_X_RAW + MXT_Q_RAW)
#define MXT_SCALES (MXT_KB * 4)       /* of a stage: four groups a term */
#define MXT_GROUPS 2                 /* groups of four converting warps, a divisor of the slots */
template <bool TN> constexpr int32_t MXT_RUN = TN ? 12 : 16;   /* stages between two reads of the hi accumulator: 24 instructions, or 32 (one read for 512 terms) */
#define MXT_REST 32                  /* runs between two reads of the accumulator of mid and lo, which starts anew then */
#define MXT_TOTAL 32                 /* stages of a group whose column sums are added up by themselves: 256 terms a thread */
#define MXT_WORKERS (4 * MXT_GROUPS)
#define MXT_TAKERS 8                 /* warps that add up the runs, behind the converters; then one for the MMAs, for the loads, for the column sums */
#define MXT_MMA (MXT_WORKERS + MXT_TAKERS)
#define MXT_THREADS ((MXT_MMA + 4) * 32)

struct MxtShared {
    float sums[MXT_WORKERS][128];
    uint64_t sums_full, sums_empty;
    uint8_t scales[MXT_SLOTS][MXT_SCALES];
    uint64_t raw_full[MXT_SLOTS], raw_empty[MXT_SLOTS];   // TMA bytes and scales have landed; the group has read them
    uint64_t op_full[MXT_SLOTS], op_empty[MXT_SLOTS];     // (first CTA) both CTAs' groups have written the tiles; the MMAs have read them
    uint64_t acc_full, acc_empty;                           // the hi accumulator holds a run; (first CTA) both CTAs have taken it out
    uint32_t tmem_base;
    int dead;
};
#define MXT_SMEM (1024 + MXT_SLOTS * (MXT_STAGE + MXT_RAW_STAGE) + (int)sizeof(MxtShared))
static_assert(MXT_SMEM <= 227 * 1024, "shared memory");

struct MxtArgs {
    const uint8_t *scales;
    int64_t ld_scales;
    int32_t D, N;              // columns of Q; columns (TN) or rows (NN) of X
    int32_t K, kps;            // terms, and terms of a split (a multiple of MXT_KB)
    int32_t bn, tiles_d, tiles_n;
    int32_t items;             // tiles times splits, the tiles of a split next to each other
    float *C;                  // element (column j of Q, column or row i of X) of split z at C + z split + i by_x + j
    int64_t split, by_x;
    float *colsum;             // TN: [splits][N] column sums of X, or none
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
// four fp32 values -> four bf16 each of hi, mid, lo (upper halves; what is left after two of them fits a third)
__device__ __forceinline__ float2 mxt_left(const float2 &x, uint32_t upper)   // x - its upper halves, by a packed multiply-add
{
    return __ffma2_rn(make_float2(__uint_as_float(upper * 0x10000u), __uint_as_float(upper & 0xFFFF0000u)), make_float2(-1.f, -1.f), x);
}
__device__ __forceinline__ uint32_t mxt_upper(const float2 &x) { return __byte_perm(__float_as_uint(x.x), __float_as_uint(x.y), 0x7632); }
__device__ __forceinline__ void mxt_split4(const float4 &x, uint2 &hi, uint2 &mid, uint2 &lo)
{
    float2 a = make_float2(x.x, x.y), b = make_float2(x.z, x.w);
    hi = make_uint2(mxt_upper(a), mxt_upper(b));
    a = mxt_left(a, hi.x);
    b = mxt_left(b, hi.y);
    mid = make_uint2(mxt_upper(a), mxt_upper(b));
    lo = make_uint2(mxt_upper(mxt_left(a, mid.x)), mxt_upper(mxt_left(b, mid.y)));
}

__device__ __forceinline__ void tc_ld16(uint32_t taddr, uint32_t *r)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr)
                 : "memory");
}
__device__ __forceinline__ void tc_ld8(uint32_t taddr, uint32_t *r)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr)
                 : "memory");
}
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// Shared memory by its own addresses (through generic pointers, a conversion took a third more instructions)
__device__ __forceinline__ float4 lds_f4(uint32_t at)
{
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ uint4 lds_u4(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ uint2 lds_u2(uint32_t at)
{
    uint2 v;
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds_u1(uint32_t at)
{
    uint32_t v;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void sts_u2(uint32_t at, const uint2 &v) { asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at), "r"(v.x), "r"(v.y) : "memory"); }
__device__ __forceinline__ void sts_u4(uint32_t at, const uint4 &v) { asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory"); }

// e4m3's codes of no number (seven ones behind the sign), which the conversion above takes for 480: NaN in their places among the two times 16 elements that
// a thread of mxt_work converts.  Codes of sat_mx_quantise have none.
__device__ __forceinline__ void mxt_no_numbers(uint32_t raw, uint32_t op, int32_t other)
{
#pragma unroll 1
    for (int32_t i = 0; i < 32; ++i) {
        const uint32_t e = i & 15, h = i >> 4;
        if ((lds_u1(raw + h * (16 * 128) + e) & 0x7Fu) != 0x7Fu) continue;
        asm volatile("st.shared.u16 [%0], %1;" ::"r"((op ^ (((e >> 3) ^ (uint32_t)other) << 4)) + h * 2048 + 2 * (e & 7)), "h"((uint16_t)0x7FFF) : "memory");
    }
}

// bf16 operands, fp32 accumulation; Q is MN-major (its tile has a row per term), X is with TN
template <bool TN>
__device__ __forceinline__ uint32_t mxt_idesc(int32_t bn)
{
    return 1u << 4 | 1u << 7 | 1u << 10 | 1u << 15 | (TN ? 1u << 16 : 0u) | (uint32_t)(bn >> 3) << 17 | (256u >> 4) << 24;
}

// Waits like mbar_wait_all in as few instructions as possible (what waits takes issue slots from the warps that convert, which are bound by them): the
// hardware may put the warp aside for up to a microsecond a time, and whether others have given up is looked at every sixteenth time.
template <int SLEEP_NS = 0>
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
        if ((it & 15u) == 15u && __any_sync(0xffffffffu, *dead)) return false;
        if (SLEEP_NS > 0) __nanosleep(SLEEP_NS);
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
// Tensor memory: the accumulator of the products with hi, from column 256 on that of the rest, which is taken out with every MXT_REST-th run and the last
// one of an item
template <bool TN>
__device__ __forceinline__ void mxt_mma(const MxtArgs &a, const MxtMem &s)
{
    volatile int *dead = &s.sh->dead;
    const uint32_t idesc = mxt_idesc<TN>(a.bn);
    // MN-major tiles: blocks of 64 columns (128 bytes a term, 128-byte swizzle) MXT_KB x 128 bytes apart, groups of eight terms 1024 bytes
    // apart; an instruction takes 16 terms.  K-major (X without TN): a row's 32 terms are 64 bytes, 64-byte swizzle, eight rows 512 apart.
    const uint64_t q0 = make_desc(smem_u32(s.op), MXT_KB * 128, 1024, 2);
    const uint64_t x0 = TN ? make_desc(smem_u32(s.op) + MXT_Q_TILE, MXT_KB * 128, 1024, 2) : make_desc(smem_u32(s.op) + MXT_Q_TILE, 16, 512, 4);
    constexpr uint32_t x_step = (TN ? 2048 : 32) >> 4, q_step = 2048 >> 4, plane = MXT_X_PLANE >> 4;
    uint32_t st = 0, ph = 0, run = 0;
    for (int32_t i = s.unit; i < a.items; i += s.units) {
        const int32_t stages = mxt_item(a, i).stages;
        for (int32_t k0 = 0; k0 < stages; k0 += MXT_RUN<TN>, ++run) {
            const uint32_t hi = s.tmem, rest = s.tmem + 256u, taken = (run & 1u) ^ 1u;   // phase of acc_empty in which what was there before has been taken out
            const bool wait_late = k0 % (MXT_REST * MXT_RUN<TN>) != 0;   // else both start anew; mid and lo go ahead while the hi accumulator is still being read
            if (!wait_late && !mxt_wait(&s.sh->acc_empty, taken, dead, a.status)) return;
            const int32_t n = min(stages - k0, MXT_RUN<TN>);
            for (int32_t k = 0; k < n; ++k) {
                if (!mxt_wait(&s.sh->op_full[st], ph, dead, a.status)) return;
                tc_fence_after();
                const uint64_t q = q0 + (uint64_t)(st * (MXT_STAGE >> 4)), x = x0 + (uint64_t)(st * (MXT_STAGE >> 4));
                if (!wait_late || k > 0) {
                    if (elect_one()) {
#pragma unroll
                        for (uint32_t ks = 0; ks < MXT_KB / 16; ++ks) {   // the tile of Q stays in the collector for its three products
                            tc_mma_f16<1, 2>(rest, q + ks * q_step, x + ks * x_step + 2 * plane, idesc, wait_late || k > 0 || ks > 0 ? 1u : 0u);
                            tc_mma_f16<3, 2>(rest, q + ks * q_step, x + ks * x_step + plane, idesc, 1u);
                            tc_mma_f16<2, 2>(hi, q + ks * q_step, x + ks * x_step, idesc, k > 0 || ks > 0 ? 1u : 0u);
                        }
                    }
                } else {
                    if (elect_one()) {
#pragma unroll
                        for (uint32_t ks = 0; ks < MXT_KB / 16; ++ks) {
                            tc_mma_f16<1, 2>(rest, q + ks * q_step, x + ks * x_step + 2 * plane, idesc, 1u);
                            tc_mma_f16<2, 2>(rest, q + ks * q_step, x + ks * x_step + plane, idesc, 1u);
                        }
                    }
                    __syncwarp();
                    if (!mxt_wait(&s.sh->acc_empty, taken, dead, a.status)) return;
                    tc_fence_after();
                    if (elect_one()) {
#pragma unroll
                        for (uint32_t ks = 0; ks < MXT_KB / 16; ++ks) tc_mma_f16<0, 2>(hi, q + ks * q_step, x + ks * x_step, idesc, ks > 0 ? 1u : 0u);
                    }
                }
                __syncwarp();
                if (elect_one()) {
                    tc_commit<2>(&s.sh->op_empty[st]);
                    if (k + 1 == n) tc_commit<2>(&s.sh->acc_full);
                }
                __syncwarp();
                if (++st == MXT_SLOTS) st = 0, ph ^= 1u;
            }
        }
    }
}

// TMA loads and, a term per lane, asynchronous copies of the scales, as soon as a group has read what it had
template <bool TN, int FMT>
__device__ __forceinline__ void mxt_load(const MxtArgs &a, const MxtMem &s, const CUtensorMap *map_x, const CUtensorMap *map_q, int lane)
{
    volatile int *dead = &s.sh->dead;
    const int32_t half = a.bn / 2;
    uint32_t st = 0, ph = 0, issued = 0;
    if (lane == 0) tma_prefetch(map_x), tma_prefetch(map_q);
    for (int32_t i = s.unit; i < a.items; i += s.units) {
        const MxtItem it = mxt_item(a, i);
        const int32_t x0 = it.n0 + s.rank * half, q0 = it.d0 + s.rank * 128;
        const bool has_x = x0 < a.N, has_q = q0 < a.D;
        const uint32_t bytes = (has_x ? (uint32_t)half * 128u : 0u) + (has_q ? 128u * MXT_KB * FMT / 8 : 0u);
        const uint8_t *scales = a.scales + (int64_t)(it.k0 + lane) * a.ld_scales + q0 / MX_GROUP;   // four bytes, of which some may lie behind the row's last
        for (int32_t k = it.k0; k < it.k1; k += MXT_KB, scales += MXT_KB * a.ld_scales) {
            if (!mxt_wait<100>(&s.sh->raw_empty[st], ph ^ 1u, dead, a.status)) {
                asm volatile("cp.async.wait_all;" ::: "memory");
                return mbar_settle(s.sh->raw_full, MXT_SLOTS, issued);
            }
            if (i == s.unit && k == it.k0) sat_grid_wait();   // (what comes before is set-up; the converters and the MMAs touch no global memory, the other roles wait as well)
            uint64_t *bar = &s.sh->raw_full[st];
            if (lane == 0) {
                uint8_t *x = s.raw + st * MXT_RAW_STAGE;
                mbar_expect_tx(bar, bytes);
                if (has_x) tma_load_2d(x, map_x, bar, TN ? x0 : k, TN ? k : x0);
                if (has_q) tma_load_2d(x + MXT_X_RAW, map_q, bar, q0 / 8 * FMT, k);
            }
            __syncwarp();
            const bool there = has_q && k + lane < it.k1;   // (else four zero bytes and nothing read)
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(s.sh->scales[st] + 4 * lane)), "l"(there ? scales : a.scales), "r"(there ? 4u : 0u) : "memory");
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
            if (++st == MXT_SLOTS) st = 0, ph ^= 1u;
            ++issued;
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (*dead) mbar_settle(s.sh->raw_full, MXT_SLOTS, issued);
}

template <bool TN, int FMT>
__device__ __forceinline__ void mxt_work(const MxtArgs &a, const MxtMem &s, int warp, int lane)
{
    volatile int *dead = &s.sh->dead;
    const int32_t group = warp >> 2, w = warp & 3, half = a.bn / 2;
    // Per thread and stage: eight times four values of X and two times 16 elements of Q (all places relative to the stage's).
    // TN: columns 4 lane .. of the terms w + 4 i; a warp reads a term's 512 bytes, half of it writes 128 of a block of 64 columns.
    // NN: terms 4 (lane % 8) .. of the rows 4 w + lane / 8 + 16 i; eight lanes read 128 bytes of a row and write its 64.
    const int32_t x_row = TN ? w : 4 * w + (lane >> 3), x_col = TN ? 4 * lane : 4 * (lane & 7);
    constexpr int32_t x_apart = TN ? 4 : 16;
    const uint32_t x_next = (uint32_t)x_apart * (TN ? (uint32_t)half * 4u : 128u);
    const uint32_t x_raw = smem_u32(s.raw) + (uint32_t)x_row * (TN ? (uint32_t)half * 4u : 128u) + (uint32_t)x_col * 4u;
    const uint32_t x_op = smem_u32(s.op) + MXT_Q_TILE + (TN ? (uint32_t)(lane >> 4) * (MXT_KB * 128) + (uint32_t)x_row * 128u + ((uint32_t)(((lane & 15) >> 1) ^ x_row) << 4)
                                                            : (uint32_t)x_row * 64u + ((uint32_t)(((lane & 7) >> 1) ^ ((x_row >> 1) & 3)) << 4)) + (uint32_t)(lane & 1) * 8u;
    // Q: elements 16 place .. of the terms term + 16 i.  Eight lanes write a term's two halves of 128 bytes: those of the second half its 16-byte pieces in
    // the other order, so that they meet no bank twice
    const int32_t place = lane & 7, term = 4 * w + (lane >> 3), other = place >> 2;
    const uint32_t q_raw = smem_u32(s.raw) + MXT_X_RAW + (uint32_t)(term * 128 + 16 * place) * FMT / 8;
    const uint32_t scales = smem_u32(s.sh->scales[0]) + 4u * (uint32_t)term + ((uint32_t)place >> 1);
    const uint32_t q_op = smem_u32(s.op) + (uint32_t)other * (MXT_KB * 128) + (uint32_t)term * 128u + ((uint32_t)((2 * (place & 3) + other) ^ (term & 7)) << 4);

    uint32_t st = (uint32_t)group, ph = 0, turn = 0;
    int32_t base = 0;   // stages before this item, modulo the groups
    for (int32_t i = s.unit; i < a.items; i += s.units) {
        const MxtItem it = mxt_item(a, i);
        const int32_t x0 = it.n0 + s.rank * half;
        const bool sums = TN && a.colsum && it.d0 == 0, has_q = it.d0 + s.rank * 128 + 16 * place < a.D;
        // how many of this thread's rows there are (NN), or whether its columns are (TN)
        const int32_t end = min(half, a.N - x0), has_x = TN ? (x_col < end ? 8 : 0) : (x_row < end ? (end - 1 - x_row) / x_apart + 1 : 0);
        // column sums: of up to MXT_TOTAL stages of this group, and of those before, so that no chain of additions is long
        float2 total[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)}, before[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll 1
        for (int32_t k = (group - base) & (MXT_GROUPS - 1); k < it.stages; k += MXT_GROUPS) {
            if (!mxt_wait<20>(&s.sh->raw_full[st], ph, dead, a.status)) return;
            if (!mxt_wait<20>(&s.sh->op_empty[st], ph ^ 1u, dead, a.status)) return;
            const uint32_t raw = st * MXT_RAW_STAGE, op = st * MXT_STAGE;
            float4 x[4];   // four in flight
#pragma unroll
            for (int h = 0; h < 4; ++h)
                if (h < has_x) x[h] = lds_f4(x_raw + raw + h * x_next);
#pragma unroll
            for (int h = 0; h < 8; ++h)
                if (h < has_x) {
                    uint2 hi, mid, lo;
                    const float4 v = x[h & 3];
                    if (h + 4 < 8 && h + 4 < has_x) x[h & 3] = lds_f4(x_raw + raw + (h + 4) * x_next);
                    mxt_split4(v, hi, mid, lo);
                    if (sums) {
                        total[0] = __fadd2_rn(total[0], make_float2(v.x, v.y));
                        total[1] = __fadd2_rn(total[1], make_float2(v.z, v.w));
                    }
                    // TN: the term four on has the other half of a row's swizzle
                    const uint32_t o = op + (TN ? (x_op ^ (uint32_t)((h & 1) << 6)) + h * 512 : x_op + h * 1024);
                    sts_u2(o, hi);
                    sts_u2(o + MXT_X_PLANE, mid);
                    sts_u2(o + 2 * MXT_X_PLANE, lo);
                }
            if (has_q) {
                uint32_t c[2][4], byte[2], odd = 0u;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    byte[h] = lds_u1(scales + st * MXT_SCALES + 64 * h);
                    if (FMT == SAT_MX8) {
                        const uint4 t = lds_u4(q_raw + raw + h * (16 * 128));
                        c[h][0] = t.x, c[h][1] = t.y, c[h][2] = t.z, c[h][3] = t.w;
#pragma unroll
                        for (int e = 0; e < 4; ++e) odd |= c[h][e] ^ (c[h][e] + 0x01010101u);   // a byte's top bit changes where the others are all ones
                    } else {
                        const uint2 t = lds_u2(q_raw + raw + h * (16 * 64));
                        c[h][0] = t.x, c[h][2] = t.y, c[h][1] = c[h][3] = 0u;
                    }
                }
                const bool no_numbers = FMT == SAT_MX8 && (odd & 0x80808080u);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const MxtScale<FMT> sc(byte[h]);
                    // the half that is written first: the upper one for lanes of the second block
                    uint4 v0 = mxt_decode8<FMT>(other ? c[h][2] : c[h][0], other ? c[h][3] : c[h][1], sc), v1 = mxt_decode8<FMT>(other ? c[h][0] : c[h][2], other ? c[h][1] : c[h][3], sc);
                    if (sc.two) v0 = bf16x8_mul(v0, sc.second), v1 = bf16x8_mul(v1, sc.second);
                    sts_u4(q_op + op + h * 2048, v0);
                    sts_u4((q_op ^ 16u) + op + h * 2048, v1);
                }
                if (no_numbers) mxt_no_numbers(q_raw + raw, q_op + op, other);
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&s.sh->raw_empty[st]);
            mbar_arrive_warp<2>(&s.sh->op_full[st], lane);
            if (sums && (k + MXT_GROUPS) % (MXT_GROUPS * MXT_TOTAL) < MXT_GROUPS) {
#pragma unroll
                for (int h = 0; h < 2; ++h) before[h] = __fadd2_rn(before[h], total[h]), total[h] = make_float2(0.f, 0.f);
            }
            if ((st += MXT_GROUPS) >= MXT_SLOTS) st -= MXT_SLOTS, ph ^= 1u;
        }
        base += it.stages;
        if (sums) {   // the warps' sums of a column are added up by the warp that writes them
            if (!mxt_wait(&s.sh->sums_empty, (turn & 1u) ^ 1u, dead, a.status)) return;
            *reinterpret_cast<float4 *>(s.sh->sums[warp] + 4 * lane) = make_float4(before[0].x + total[0].x, before[0].y + total[0].y, before[1].x + total[1].x, before[1].y + total[1].y);
            __syncwarp();
            if (lane == 0) mbar_arrive(&s.sh->sums_full);
            ++turn;
        }
    }
    // the pair's MMAs have signalled this group's stages: nothing arrives here any more once both CTAs may exit
    for (int h = 0; h < MXT_SLOTS; h += MXT_GROUPS) {
        if (!mxt_wait(&s.sh->op_empty[st], ph ^ 1u, dead, a.status)) return;
        if ((st += MXT_GROUPS) >= MXT_SLOTS) st -= MXT_SLOTS, ph ^= 1u;
    }
}

// Adds up the runs: a lane has a column of Q, a register a column or row of X, so that consecutive lanes write consecutive floats.  Eight warps, two to a
// quarter of the lanes, with half the columns each.
template <bool TN>
__device__ __forceinline__ void mxt_runs(const MxtArgs &a, const MxtMem &s, int warp, int lane)
{
    volatile int *dead = &s.sh->dead;
    const int32_t c0 = (warp >> 2) * 128, here = min(8, (a.bn - c0) / 16);   // 16 columns at a time
    const uint32_t lanes = s.tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)c0;
    uint32_t run = 0;
    sat_grid_wait();
    uint32_t acc[128];   // bits of the sums
    for (int32_t i = s.unit; i < a.items; i += s.units) {
        const int32_t stages = mxt_item(a, i).stages;
#pragma unroll 1
        for (int32_t k0 = 0; k0 < stages; k0 += MXT_RUN<TN>, ++run) {
            if (!mxt_wait<60>(&s.sh->acc_full, run & 1u, dead, a.status)) return;
            tc_fence_after();
            const bool with_rest = k0 + MXT_RUN<TN> >= stages || (k0 / MXT_RUN<TN> + 1) % MXT_REST == 0;
            if (k0 == 0) {   // straight to where it stays
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    if (c < here) tc_ld16(lanes + 16u * c, acc + 16 * c);
                tc_wait_ld();
            }
#pragma unroll
            for (int half = 0; half < 2; ++half)   // the run, then the rest
                if (half ? with_rest : k0 > 0) {
#pragma unroll
                    for (int c = 0; c < 16; ++c)
                        if (c < 2 * here) {
                            uint32_t r[8];
                            tc_ld8(lanes + 256u * half + 8u * c, r);
                            tc_wait_ld();
#pragma unroll
                            for (int e = 0; e < 8; ++e) acc[8 * c + e] = __float_as_uint(__uint_as_float(acc[8 * c + e]) + __uint_as_float(r[e]));
                        }
                }
            tc_fence_before();
            mbar_arrive_warp<2>(&s.sh->acc_empty, lane);
        }
        const MxtItem it = mxt_item(a, i);
        const int32_t col = it.d0 + s.rank * 128 + (warp & 3) * 32 + lane, n = min(a.bn, a.N - it.n0) - c0;
        float *o = a.C + it.split * a.split + (it.n0 + c0) * a.by_x + col;
        if (col >= a.D) continue;
        // 16 at a time, those that are there: one warp a scheduler waits for every instruction, so what does not have to be looked at counts (301 x 100 by 301 x 47:
        // 8100 clocks of 18000 went by here while each of the 128 was asked whether it is there)
#pragma unroll
        for (int c = 0; c < 8; ++c, o += 16 * a.by_x) {
            if (16 * c >= n) break;
            float *e = o;
            if (16 * c + 16 <= n) {
#pragma unroll
                for (int h = 0; h < 16; ++h, e += a.by_x) *e = __uint_as_float(acc[16 * c + h]);
            } else {
#pragma unroll
                for (int h = 0; h < 16; ++h, e += a.by_x)
                    if (16 * c + h < n) *e = __uint_as_float(acc[16 * c + h]);
            }
        }
    }
}

// (TN) The column sums of an item
__device__ __forceinline__ void mxt_totals(const MxtArgs &a, const MxtMem &s, int lane)
{
    const int32_t half = a.bn / 2;
    uint32_t turn = 0;
    sat_grid_wait();
    for (int32_t i = s.unit; i < a.items; i += s.units) {
        const MxtItem it = mxt_item(a, i);
        if (it.d0 != 0) continue;
        if (!mxt_wait<1000>(&s.sh->sums_full, turn & 1u, &s.sh->dead, a.status)) return;
        for (int32_t c = lane; c < half; c += 32) {
            double sum = 0.;
            for (int h = 0; h < MXT_WORKERS; ++h) sum += (double)s.sh->sums[h][c];
            const int32_t at = it.n0 + s.rank * half + c;
            if (at >= a.N) continue;
            float *out = a.colsum + (int64_t)it.split * a.N + at;
            *out = (float)sum;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&s.sh->sums_empty);
        ++turn;
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
    s.raw = smem + MXT_SLOTS * MXT_STAGE;
    s.sh = (MxtShared *)(s.raw + MXT_SLOTS * MXT_RAW_STAGE);
    s.rank = (int32_t)(blockIdx.x & 1u);
    s.unit = (int32_t)(blockIdx.x >> 1);
    s.units = (int32_t)(gridDim.x >> 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < MXT_SLOTS; ++i) {
            mbar_init(&s.sh->raw_full[i], 1 + 32);   // the TMA's issuer and the scales' lanes
            mbar_init(&s.sh->raw_empty[i], 4);
            mbar_init(&s.sh->op_full[i], 2 * 4);     // a group of either CTA
            mbar_init(&s.sh->op_empty[i], 1);
        }
        mbar_init(&s.sh->acc_full, 1);
        mbar_init(&s.sh->acc_empty, 2 * MXT_TAKERS);
        mbar_init(&s.sh->sums_full, MXT_WORKERS);
        mbar_init(&s.sh->sums_empty, 1);
        s.sh->dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == MXT_MMA) tc_alloc<2>(&s.sh->tmem_base, 512u);
    tc_fence_before();
    __syncthreads();
    cluster_sync();   // the other CTA's barriers are initialised and its TMEM is allocated
    tc_fence_after();
    s.tmem = s.sh->tmem_base;
    // 640 threads start with 96 registers each; the two warpgroups that add up the runs, 128 sums a thread, go to 160, the converters' two to 64 and the fifth
    // one to 32: 2 x 160 + 2 x 64 + 32 = 5 x 96
    if (warp < MXT_WORKERS) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        mxt_work<TN, FMT>(a, s, warp, lane);
    } else if (warp < MXT_MMA) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 160;");
        mxt_runs<TN>(a, s, warp - MXT_WORKERS, lane);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 32;");
        if (warp == MXT_MMA) {
            if (s.rank == 0) mxt_mma<TN>(a, s);
        } else if (warp == MXT_MMA + 1) mxt_load<TN, FMT>(a, s, &map_x, &map_q, lane);
        else if (TN && warp == MXT_MMA + 2 && a.colsum) mxt_totals(a, s, lane);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    cluster_sync();   // neither CTA's shared memory or TMEM is in use by the other any more
    if (warp == MXT_MMA) {
        tc_fence_after();
        tc_dealloc<2>(s.tmem, 512u);
    }
}

// C[j][i] (+)= sum over the splits of part[z][i][j], cs[i] (+)= that of part_cs[z][i], in a fixed order: 128 columns of Q by R of X per block, four columns to
// a lane, every 16 / R-th split to a warp.  Bound by the L2 and its latency: R = 1 where
// splits are many, for more loads at once, else 4, for longer pieces of C.  Measured with 1 / 4, gradient included: 73 splits of 256 x 256 19.0 / 22.3 us, of 100 x 128
// 80.0 / 83.9; 24 splits of 602 x 256 63.7 / 63.7, 9 of 1024 x 512 152.3 / 147.5.
template <int R>
__global__ void __launch_bounds__(512)
k_mx_reduce(const float *__restrict__ part, const float *__restrict__ part_cs, int32_t splits, int32_t D, int32_t N, int64_t ld, int add, float *__restrict__ C,
            float *__restrict__ colsum)
{
    constexpr int Z = 16 / R;
    sat_grid_wait();
    __shared__ float red[Z][R][132];
    const int lane = threadIdx.x & 31, i = (threadIdx.x >> 5) % R, z0 = (threadIdx.x >> 5) / R;
    const int32_t tiles = (D + 127) / 128, tile = (int32_t)(blockIdx.x % (uint32_t)tiles), col = tile * 128 + 4 * lane, row0 = (int32_t)(blockIdx.x / (uint32_t)tiles) * R, row = row0 + i;
    const int64_t plane = ld * N;
    float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
    if (col < D && row < N) {
        const float *p = part + (int64_t)row * ld + col;
#pragma unroll 8
        for (int32_t z = z0; z < splits; z += Z) {
            const float4 v = __ldg(reinterpret_cast<const float4 *>(p + z * plane));
            t = make_float4(t.x + v.x, t.y + v.y, t.z + v.z, t.w + v.w);
        }
    }
    *reinterpret_cast<float4 *>(&red[z0][i][4 * lane]) = t;
    if (z0 == Z - 1 && tile == 0 && colsum && row < N) {   // a warp a column (one thread that took the splits in turn was what the launch waited for)
        double sum = 0.;
        for (int32_t z = lane; z < splits; z += 32) sum += (double)__ldg(part_cs + (int64_t)z * N + row);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) colsum[row] = add ? (float)((double)colsum[row] + sum) : (float)sum;
    }
    __syncthreads();
    const int j = threadIdx.x / R, ii = threadIdx.x % R;   // R lanes write R consecutive floats of a row of C
    const int32_t c = tile * 128 + j, r = row0 + ii;
    if (j < 128 && c < D && r < N) {
        float sum = 0.f;
#pragma unroll
        for (int z = 0; z < Z; ++z) sum += red[z][ii][j];
        float *o = C + (int64_t)c * N + r;
        *o = add ? *o + sum : sum;
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
    // Rows a tile: what ends first.  A round of tiles of 256 rows takes a third longer than one of 64, since the codes are converted for either
    // (512 terms: 14.6 and 11.5 us).  Measured with 64 / 256 rows: 2000 rows by 256 columns 11.8 / 15.1 us, 5000 rows 19.0 / 15.5 (128 rows: 14.0), 18944 rows 38.0 / 18.6.
    int32_t bn = 64;
    int64_t best = INT64_MAX;
    for (int32_t b = 64; b <= 256; b *= 2) {
        const int64_t cost = cdiv64(cdiv64(W->d, 256) * cdiv64(m, b), ctx->sms / 2) * (512 + b);
        if (cost < best) bn = b, best = cost;
    }
    MxtArgs a{};
    CUtensorMap map_x, map_q;
    SAT_TRY(mxt_args(ctx, W, m, bn, &a, &map_q));
    a.C = C;
    a.by_x = ldc;
    SAT_TRY(sat_tensor_map(ctx, &map_x, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, A, W->rows, m, (int64_t)lda * 4, MXT_KB, bn / 2, CU_TENSOR_MAP_SWIZZLE_NONE));
    return W->format == SAT_MX8 ? mxt_launch<false, SAT_MX8>(ctx, map_x, map_q, a) : mxt_launch<false, SAT_MX4>(ctx, map_x, map_q, a);
}

sat_status sat_mx_tc_tn(sat_ctx *ctx, const sat_mx_matrix *A, int32_t n, const float *B, int32_t ldb, float *C, float *colsum, int accumulate)
{
    const int32_t tiles_n = (int32_t)cdiv64(n, 256), bn = (int32_t)cdiv64(cdiv64(n, tiles_n), 64) * 64;
    MxtArgs a{};
    CUtensorMap map_x, map_q;
    SAT_TRY(mxt_args(ctx, A, n, bn, &a, &map_q));
    // Row splits: what takes the fewest stages in a row on the busiest pair, a split costing about six stages to set up and to add up
    // (150000 rows of 602 by 256: 138.8 us, 139.4 where a split is taken to cost one stage; nothing in it from 20000 rows down)
    const int64_t units = ctx->sms / 2, tiles = a.items, stages = cdiv64(A->rows, MXT_KB);
    int64_t best = 1, best_cost = INT64_MAX;
    for (int64_t s = 1; s <= std::min<int64_t>(2 * units / tiles + 1, cdiv64(stages, 4)); ++s) {
        const int64_t cost = cdiv64(tiles * s, units) * (cdiv64(stages, s) + 6);
        if (cost < best_cost) best = s, best_cost = cost;
    }
    a.kps = (int32_t)std::min<int64_t>(cdiv64(stages, best) * MXT_KB, INT32_MAX & ~(MXT_KB - 1));
    const int32_t splits = (int32_t)cdiv64(A->rows, a.kps);
    a.items *= splits;
    // One split goes through memory as well, as Q^^T X turned round: a lane holds a column of Q, so writing C itself takes 32 pieces of 32 lines an instruction (40 rows
    // of 256 by 256: 30 us against 9.7; 30 of 100 by 18 5.0 against 6.3)
    a.by_x = (a.D + 3) & ~3;
    a.split = a.by_x * n;
    SAT_TRY(sat_ensure(ctx, ctx->buf_splitk, (size_t)splits * (size_t)(a.split + n) * sizeof(float)));
    a.C = (float *)ctx->buf_splitk.p;
    a.colsum = colsum ? a.C + splits * a.split : nullptr;
    SAT_TRY(sat_tensor_map(ctx, &map_x, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, B, n, A->rows, (int64_t)ldb * 4, bn / 2, MXT_KB, CU_TENSOR_MAP_SWIZZLE_NONE));
    SAT_TRY((A->format == SAT_MX8 ? mxt_launch<true, SAT_MX8>(ctx, map_x, map_q, a) : mxt_launch<true, SAT_MX4>(ctx, map_x, map_q, a)));
    if (splits > 32)
        sat_pdl(ctx->stream, k_mx_reduce<1>, (unsigned)(cdiv64(a.D, 128) * n), 512, 0)(a.C, a.colsum, splits, a.D, n, a.by_x, accumulate, C, colsum);
    else
        sat_pdl(ctx->stream, k_mx_reduce<4>, (unsigned)(cdiv64(a.D, 128) * cdiv64(n, 4)), 512, 0)(a.C, a.colsum, splits, a.D, n, a.by_x, accumulate, C, colsum);
    SAT_LAUNCHED(ctx);
    return SAT_OK;
}

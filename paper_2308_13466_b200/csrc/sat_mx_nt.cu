// Product of 4-bit operands on the 5th-generation tensor cores (sat_mx_dense_nt):
//     C[m x n] = A^[m x k] W^[n x k]^T + bias,   A fp32 and quantised on the way in, or stored
// kind::mxf4 with a scale per 32 terms: the tensor core multiplies e2m1 by e2m1, applies both powers of two and adds in fp32; a product
// has at most six significant bits, so sums are exact or nearly so.  What bounds it is memory: 4 bytes an element of A in, 4 bytes an element of
// C out, each once; the contraction is a quarter of that time at the widths of a layer
// (169343 x 256 by 256: 67 us, 79 % of the copy rate).
//
// One CTA per SM walks tiles of 128 rows by up to 256 columns.  24 warps: 0..15 quantise (a warpgroup per 32 of a stage's 128 terms, a
// thread per row and group, so that a group's maximum needs no exchange), 16..19 the epilogue, 20 MMAs, 21 TMA loads of A, 22 W's codes (TMA) and
// scales.  Scales lie in shared memory as the tensor core wants them, row r and group g of a stage at (r % 32) 16 + (r / 32) 4 + g, and are
// copied to TMEM (four columns per 128 rows) in front of the stage's two MMAs.
#include "sat_mx.h"
#include "sat_ptx.h"

#include <algorithm>

#define NT_THREADS (24 * 32)
#define NT_KB 128                       /* terms per stage: 64 bytes of codes, 64-byte swizzle */
#define NT_OP 2                         /* stages of operand tiles */
#define NT_RAW 2                        /* boxes of 128 rows x 32 floats per warpgroup in flight */
#define NT_A_TILE (128 * NT_KB / 2)
#define NT_W_TILE (256 * NT_KB / 2)
#define NT_SFA (NT_A_TILE + NT_W_TILE)  /* scales of A: 512 bytes, of W: 1024 */
#define NT_SFW (NT_SFA + 512)
#define NT_STAGE (26 * 1024)
#define NT_BOX (128 * 32 * 4)
#define NT_OUT (4 * 2 * 4096)            /* results on their way out: two blocks of 32 x 32 per warp */
#define NT_BIAS (4 * 256 * 4)

struct NtShared {
    uint64_t raw_full[4][NT_RAW], raw_empty[4][NT_RAW];   // per warpgroup
    uint64_t op_full[NT_OP], op_empty[NT_OP];             // 16 quantising warps, W's warp and W's TMA bytes; the MMAs have read them
    uint64_t acc_full, acc_empty;
    uint32_t tmem_base;
    int dead;
};
#define NT_SMEM (1024 + NT_OP * NT_STAGE + 4 * NT_RAW * NT_BOX + NT_OUT + NT_BIAS + (int)sizeof(NtShared))
static_assert(NT_SFW + 1024 <= NT_STAGE && NT_SMEM <= 227 * 1024, "shared memory");

struct NtArgs {
    MxView a, w;                 // a: where A comes from or is kept, or null
    int64_t ldc;
    int32_t m, n, k, groups, stages;
    int32_t bn, tiles_n, tiles;
    const float *bias;
    float *C;
    int *status;
};

// kind::mxf4, e2m1 by e2m1, e8m0 scales; `pair`: which two of a stage's four scales
__device__ __forceinline__ uint32_t nt_idesc(int32_t bn, uint32_t pair)
{
    return (2u * pair) << 4 | 1u << 7 | 1u << 10 | (uint32_t)(bn >> 3) << 17 | 1u << 23 | (128u >> 4) << 24 | (2u * pair) << 29;
}
__device__ __forceinline__ void nt_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate)
{
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t"
        "}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void nt_copy_scales(uint32_t taddr, uint64_t desc)
{
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}

struct NtMem {
    uint8_t *op, *raw, *out;
    NtShared *sh;
    uint32_t tmem;
};

__device__ __forceinline__ void nt_issue(const NtArgs &p, const NtMem &s)
{
    volatile int *dead = &s.sh->dead;
    const uint64_t a0 = make_desc(smem_u32(s.op), 16, 512, 4), w0 = make_desc(smem_u32(s.op) + NT_A_TILE, 16, 512, 4);
    const uint64_t f0 = make_desc(smem_u32(s.op) + NT_SFA, 16, 128, 0);
    uint32_t st = 0, ph = 0, done = 0;
    for (int32_t t = blockIdx.x; t < p.tiles; t += gridDim.x, ++done) {
        if (!mbar_wait_all(&s.sh->acc_empty, (done & 1u) ^ 1u, dead, p.status)) return;
        tc_fence_after();
        for (int32_t k = 0; k < p.stages; ++k) {
            if (!mbar_wait_all(&s.sh->op_full[st], ph, dead, p.status)) return;
            tc_fence_after();
            if (elect_one()) {
                const uint64_t off = (uint64_t)(st * (NT_STAGE >> 4));
                const uint32_t sfa = s.tmem + 256u + 16u * st, sfw = sfa + 4u;   // a stage has its own columns: nothing is overwritten in use
                nt_copy_scales(sfa, f0 + off);
                nt_copy_scales(sfw, f0 + off + (512 >> 4));
                if (p.bn > 128) nt_copy_scales(sfw + 4u, f0 + off + (1024 >> 4));
#pragma unroll
                for (uint32_t h = 0; h < 2; ++h)   // 64 terms, 32 bytes of a row
                    nt_mma(s.tmem, a0 + off + 2 * h, w0 + off + 2 * h, nt_idesc(p.bn, h), sfa, sfw, k > 0 || h > 0 ? 1u : 0u);
                tc_commit<1>(&s.sh->op_empty[st]);
                if (k + 1 == p.stages) tc_commit<1>(&s.sh->acc_full);
            }
            __syncwarp();
            if (++st == NT_OP) st = 0, ph ^= 1u;
        }
    }
}

__device__ __forceinline__ void nt_load_a(const NtArgs &p, const NtMem &s, const CUtensorMap *map_a)
{
    volatile int *dead = &s.sh->dead;
    uint32_t slot = 0, ph = 0, issued = 0;
    auto settle = [&](int g0) {   // the rings below g0 have had one more
        for (int g = 0; g < 4; ++g) mbar_settle(s.sh->raw_full[g], NT_RAW, issued + (g < g0 ? 1u : 0u));
    };
    for (int32_t t = blockIdx.x; t < p.tiles; t += gridDim.x) {
        const int32_t m0 = t / p.tiles_n * 128;
        for (int32_t k = 0; k < p.stages; ++k, ++issued) {
            for (int g = 0; g < 4; ++g) {
                if (!mbar_wait(&s.sh->raw_empty[g][slot], ph ^ 1u, dead, p.status)) return settle(g);
                mbar_expect_tx(&s.sh->raw_full[g][slot], NT_BOX);
                tma_load_2d(s.raw + (g * NT_RAW + slot) * NT_BOX, map_a, &s.sh->raw_full[g][slot], k * NT_KB + 32 * g, m0);
            }
            if (++slot == NT_RAW) slot = 0, ph ^= 1u;
        }
    }
    if (*dead) settle(0);
}

__device__ __forceinline__ void nt_load_w(const NtArgs &p, const NtMem &s, const CUtensorMap *map_w, int lane)
{
    volatile int *dead = &s.sh->dead;
    uint32_t st = 0, ph = 0, issued = 0;
    for (int32_t t = blockIdx.x; t < p.tiles; t += gridDim.x) {
        const int32_t n0 = t % p.tiles_n * p.bn;
        for (int32_t k = 0; k < p.stages; ++k, ++issued) {
            // four scales of each of up to eight rows; one where there is no such row or group
            uint32_t f[8];
            const int32_t left = p.groups - 4 * k;
            const uint32_t keep = left >= 4 ? 0xFFFFFFFFu : (1u << 8 * left) - 1u;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int32_t r = 32 * i + lane;
                f[i] = 0x7F7F7F7Fu;
                if (r < p.bn && n0 + r < p.n) f[i] = (__ldg(reinterpret_cast<const uint32_t *>(p.w.scales + (int64_t)(n0 + r) * p.w.ld_scales) + k) & keep) | (0x7F7F7F7Fu & ~keep);
            }
            if (!mbar_wait_all(&s.sh->op_empty[st], ph ^ 1u, dead, p.status)) return mbar_settle(s.sh->op_full, NT_OP, issued);
            uint8_t *op = s.op + st * NT_STAGE;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (32 * i < p.bn) *reinterpret_cast<uint32_t *>(op + NT_SFW + (i >> 2) * 512 + lane * 16 + (i & 3) * 4) = f[i];
            fence_async_smem();
            __syncwarp();
            if (lane == 0) {
                mbar_expect_tx(&s.sh->op_full[st], (uint32_t)p.bn * 64u);
                tma_load_2d(op + NT_A_TILE, map_w, &s.sh->op_full[st], k * (NT_KB / 2), n0);
            }
            if (++st == NT_OP) st = 0, ph ^= 1u;
        }
    }
    if (*dead) mbar_settle(s.sh->op_full, NT_OP, issued);
}

template <bool STORED>
__device__ __forceinline__ void nt_rows(const NtArgs &p, const NtMem &s, int warp, int lane)
{
    volatile int *dead = &s.sh->dead;
    const int g = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t at = (uint32_t)row * 64u + (uint32_t)((g ^ ((row >> 1) & 3)) << 4), sf_at = NT_SFA + (row & 31) * 16 + (row >> 5) * 4 + g;
    uint32_t slot = 0, rph = 0, st = 0, ph = 0;
    for (int32_t t = blockIdx.x; t < p.tiles; t += gridDim.x) {
        const int64_t r = (int64_t)(t / p.tiles_n) * 128 + row;
        const bool keep = !STORED && p.a.codes && t % p.tiles_n == 0 && r < p.m;
        for (int32_t k = 0; k < p.stages; ++k) {
            uint32_t c[4] = {0u, 0u, 0u, 0u};
            uint32_t byte = 127u;
            const int32_t group = 4 * k + g;
            if (STORED) {
                if (r < p.m && group < p.groups) {
                    const uint4 t = __ldg(reinterpret_cast<const uint4 *>(p.a.codes + r * p.a.ld_codes) + group);
                    c[0] = t.x, c[1] = t.y, c[2] = t.z, c[3] = t.w;
                    byte = __ldg(p.a.scales + r * p.a.ld_scales + group);
                }
            } else {
                if (!mbar_wait_all(&s.sh->raw_full[g][slot], rph, dead, p.status)) return;
                const uint8_t *x = s.raw + (g * NT_RAW + slot) * NT_BOX + row * 128;
                float4 v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const float4 *>(x + ((i ^ (row & 7)) << 4));
                byte = mx_quantise32<SAT_MX4>(v, c);
                fence_async_smem();   // the loads are done before the TMA writes there again (an arrival alone lets it overtake them)
                __syncwarp();
                if (lane == 0) mbar_arrive(&s.sh->raw_empty[g][slot]);
                if (++slot == NT_RAW) slot = 0, rph ^= 1u;
                if (keep && group < p.groups) {
                    *(reinterpret_cast<uint4 *>(p.a.codes + r * p.a.ld_codes) + group) = make_uint4(c[0], c[1], c[2], c[3]);
                    p.a.scales[r * p.a.ld_scales + group] = (uint8_t)byte;
                }
            }
            if (!mbar_wait_all(&s.sh->op_empty[st], ph ^ 1u, dead, p.status)) return;
            uint8_t *op = s.op + st * NT_STAGE;
            *reinterpret_cast<uint4 *>(op + at) = make_uint4(c[0], c[1], c[2], c[3]);
            op[sf_at] = (uint8_t)byte;
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&s.sh->op_full[st]);
            if (++st == NT_OP) st = 0, ph ^= 1u;
        }
    }
}

// A lane has a row of a block of 32 x 32; it goes to shared memory (128 bytes a row, swizzled) and from there out by TMA, which leaves out
// what lies behind the edges
__device__ __forceinline__ void nt_results(const NtArgs &p, const NtMem &s, const CUtensorMap *map_c, int warp, int lane)
{
    volatile int *dead = &s.sh->dead;
    float *bias = reinterpret_cast<float *>(s.out + NT_OUT) + warp * 256;
    const uint32_t lanes = s.tmem + ((uint32_t)(warp * 32) << 16);
    uint32_t done = 0, buf = 0;
    int32_t bias_of = -1;
    for (int32_t t = blockIdx.x; t < p.tiles; t += gridDim.x, ++done) {
        const int32_t m0 = t / p.tiles_n * 128 + warp * 32, n0 = t % p.tiles_n * p.bn;
        if (p.bias && n0 != bias_of) {
            for (int32_t c = lane; c < p.bn; c += 32) bias[c] = n0 + c < p.n ? __ldg(p.bias + n0 + c) : 0.f;
            __syncwarp();
            bias_of = n0;
        }
        if (!mbar_wait_all(&s.sh->acc_full, done & 1u, dead, p.status)) break;
        tc_fence_after();
        for (int32_t c = 0; c < p.bn; c += 32) {
            uint32_t r[32];
            tc_ld32(lanes + (uint32_t)c, r);
            if (c + 32 >= p.bn) {   // the accumulator has been read
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&s.sh->acc_empty);
            }
            if (m0 >= p.m || n0 + c >= p.n) continue;
            uint8_t *o = s.out + (2 * warp + buf) * 4096;
            if (lane == 0) tma_store_wait_read<1>();
            __syncwarp();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float4 v = make_float4(__uint_as_float(r[4 * e]), __uint_as_float(r[4 * e + 1]), __uint_as_float(r[4 * e + 2]), __uint_as_float(r[4 * e + 3]));
                if (p.bias) {
                    const float4 b = *reinterpret_cast<const float4 *>(bias + c + 4 * e);
                    v = make_float4(v.x + b.x, v.y + b.y, v.z + b.z, v.w + b.w);
                }
                *reinterpret_cast<float4 *>(o + lane * 128 + ((e ^ (lane & 7)) << 4)) = v;
            }
            if (n0 + c + 32 > p.n && (p.n & 3)) {   // a bulk store writes the last 16 bytes of a row whole
                __syncwarp();
                for (int i = 0; i < 32; ++i)
                    if (m0 + i < p.m && n0 + c + lane < p.n)
                        p.C[(int64_t)(m0 + i) * p.ldc + n0 + c + lane] = *reinterpret_cast<const float *>(o + i * 128 + (((lane >> 2) ^ (i & 7)) << 4) + (lane & 3) * 4);
                __syncwarp();
                continue;
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) tma_store_2d(map_c, o, n0 + c, m0);
            buf ^= 1u;
        }
        __syncwarp();   // (the bias of another tile is not written while a lane still reads this one's)
    }
    if (lane == 0) tma_store_wait_all();
}

template <bool STORED>
__global__ void __launch_bounds__(NT_THREADS, 1)
k_mx_nt(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_c,
        const __grid_constant__ NtArgs p)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    NtMem s;
    s.op = smem;
    s.raw = smem + NT_OP * NT_STAGE;
    s.out = s.raw + 4 * NT_RAW * NT_BOX;
    s.sh = reinterpret_cast<NtShared *>(s.out + NT_OUT + NT_BIAS);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int g = 0; g < 4; ++g)
            for (int i = 0; i < NT_RAW; ++i) {
                mbar_init(&s.sh->raw_full[g][i], 1);
                mbar_init(&s.sh->raw_empty[g][i], 4);
            }
        for (int i = 0; i < NT_OP; ++i) {
            mbar_init(&s.sh->op_full[i], 16 + 1);
            mbar_init(&s.sh->op_empty[i], 1);
        }
        mbar_init(&s.sh->acc_full, 1);
        mbar_init(&s.sh->acc_empty, 4);
        s.sh->dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 20) tc_alloc<1>(&s.sh->tmem_base, 512u);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    s.tmem = s.sh->tmem_base;
    sat_grid_wait();   // everything above is set-up of this block; no global memory has been touched
    if (warp < 16) nt_rows<STORED>(p, s, warp, lane);
    else if (warp < 20) nt_results(p, s, &map_c, warp - 16, lane);
    else if (warp == 20) nt_issue(p, s);
    else if (warp == 21 && lane == 0 && !STORED) nt_load_a(p, s, &map_a);
    else if (warp == 22) nt_load_w(p, s, &map_w, lane);
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 20) {
        tc_fence_after();
        tc_dealloc<1>(s.tmem, 512u);
    }
}

// ---- a few rows ---------------------------------------------------------------------------------------------------------------
// Up to NT_FEW rows of A: bound by the time to read W, if not by the launch.  Twice an element is a small integer, so a group's sum of products is
// exact in integers (four bytes a dp4a).  Every block has all rows of A as bytes in shared memory; `lpr` lanes share a row of W, a group each in
// turn.  One row, 512 x 512: 1.9 us, 9.0 with the tiles above.
#define NT_FEW 16
#define NT_FEW_WARPS 4
#define NT_FEW_SMEM (96 * 1024)
// Four codes (the low half of w) as bytes of twice their values
__device__ __forceinline__ uint32_t nt_bytes(uint32_t w, uint32_t &negative)
{
    const uint32_t size = __byte_perm(0x03020100u, 0x0C080604u, w & 0x7777u);
    uint32_t m;
    asm("prmt.b32 %0, %1, %1, %2;" : "=r"(m) : "r"(0x80808080u), "r"(w));   // a selector's top bit spreads the byte's sign: FF or 80
    negative = m & 0x01010101u;
    return size ^ (negative * 255u);   // (one less than it should be where negative)
}

template <int MT>
__global__ void __launch_bounds__(32 * NT_FEW_WARPS)
k_mx_nt_few(const float *__restrict__ A, int64_t lda, int32_t m, int32_t n, int32_t k, int32_t groups, int32_t lpr, MxView a, MxView w, const float *__restrict__ bias,
            float *__restrict__ C, int64_t ldc)
{
    extern __shared__ __align__(16) uint8_t few_smem[];
    uint8_t *vals = few_smem;                                    // [m][groups][32] bytes
    int16_t *exps = reinterpret_cast<int16_t *>(vals + m * groups * 32);   // [m][groups], 1000 for NaN
    sat_grid_wait();
    for (int32_t i = threadIdx.x >> 3; i < m * groups; i += 4 * NT_FEW_WARPS) {   // eight lanes to a group, four elements each
        const int32_t r = i / groups, g = i - r * groups, sub = threadIdx.x & 7, c = g * MX_GROUP + 4 * sub;
        const unsigned lanes = 0xFFu << (threadIdx.x & 24);
        uint32_t code, byte;
        if (A) {
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (c < k) v = __ldg(reinterpret_cast<const float4 *>(A + r * lda + c));
            if (c + 1 >= k) v.y = 0.f;
            if (c + 2 >= k) v.z = 0.f;
            if (c + 3 >= k) v.w = 0.f;
            uint32_t top = max(max(__float_as_uint(v.x) & 0x7FFFFFFFu, __float_as_uint(v.y) & 0x7FFFFFFFu), max(__float_as_uint(v.z) & 0x7FFFFFFFu, __float_as_uint(v.w) & 0x7FFFFFFFu));
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) top = max(top, __shfl_xor_sync(lanes, top, o));
            byte = mx_scale_byte<SAT_MX4>(top);
            const float f = mx_inverse(byte);
            code = byte == 255u ? 0u : mx_encode4<SAT_MX4>(v.x * f, v.y * f, v.z * f, v.w * f) & 0xFFFFu;
            if (a.codes && blockIdx.x == 0) {
                *reinterpret_cast<uint16_t *>(a.codes + r * a.ld_codes + c / 2) = (uint16_t)code;
                if (sub == 0) a.scales[r * a.ld_scales + g] = (uint8_t)byte;
            }
        } else {
            code = __ldg(reinterpret_cast<const uint16_t *>(a.codes + r * a.ld_codes + c / 2));
            byte = __ldg(a.scales + r * a.ld_scales + g);
        }
        uint32_t neg;
        const uint32_t b = nt_bytes(code, neg);
        *reinterpret_cast<uint32_t *>(vals + i * 32 + 4 * sub) = __vadd4(b, neg);
        if (sub == 0) exps[i] = byte == 255u ? 1000 : (int16_t)((int32_t)byte - 127);
    }
    __syncthreads();
    const int lane = threadIdx.x & 31, sub = lane & (lpr - 1);
    const int32_t rows = 32 / lpr, row = ((int32_t)blockIdx.x * NT_FEW_WARPS + (threadIdx.x >> 5)) * rows + lane / lpr;
    const bool there = row < n;
    float acc[MT];
#pragma unroll
    for (int r = 0; r < MT; ++r) acc[r] = 0.f;
    if (there) {
        for (int32_t g = sub; g < groups; g += lpr) {
            const uint4 c = __ldg(reinterpret_cast<const uint4 *>(w.codes + row * w.ld_codes) + g);
            const uint32_t byte = __ldg(w.scales + row * w.ld_scales + g), words[4] = {c.x, c.y, c.z, c.w};
            uint32_t b[8], neg[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) b[i] = nt_bytes(words[i / 2] >> (16 * (i & 1)), neg[i]);
            const int32_t we = byte == 255u ? 2000 : (int32_t)byte - 129;   // -127, and a quarter for the doubled values
#pragma unroll
            for (int r = 0; r < MT; ++r) {
                if (r >= m) break;
                const uint4 x0 = *reinterpret_cast<const uint4 *>(vals + (r * groups + g) * 32), x1 = *reinterpret_cast<const uint4 *>(vals + (r * groups + g) * 32 + 16);
                const uint32_t x[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
                int32_t sum = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum = __dp4a((int32_t)x[i], (int32_t)b[i], __dp4a((int32_t)x[i], (int32_t)neg[i], sum));
                // 2^e in two steps, neither of which leaves the range before the product does.  A sum is at most 32 x 144, so what lies below 2^-252 is
                // 0 in fp32; two groups of zeros, whose scales are the least, come to -256
                const int32_t e = we + exps[r * groups + g], f = max(e, -252), half = f >> 1;
                const float p = __int_as_float((half + 127) << 23), q = __int_as_float((f - half + 127) << 23);
                acc[r] += e > 500 ? __int_as_float(0x7FFFFFFF) : (float)sum * p * q;
            }
        }
    }
#pragma unroll
    for (int r = 0; r < MT; ++r) {
        if (r >= m) break;
        for (int o = lpr >> 1; o > 0; o >>= 1) acc[r] += __shfl_xor_sync(0xffffffffu, acc[r], o);
        if (there && sub == 0) C[r * ldc + row] = acc[r] + (bias ? __ldg(bias + row) : 0.f);
    }
}

// Whether the rows are few: the tiles take the same time for 1 to 64 rows, this kernel time in proportion to rows x groups.  Measured, this kernel
// against tiles: n = 256, k = 100 1.8 / 5.8 us with one row, 5.7 / 5.9 with 16, 7.8 / 5.9 with 24; 512 x 512 1.9 / 9.0 with one, 8.6 / 9.0 with 12,
// 11.0 / 9.0 with 16; 1024 x 1024 2.6 / 13.6 with one, 11.9 / 13.6 with 8, 17.0 / 13.6 with 12.  The bytes of A and their exponents have to fit.
static bool nt_few(int64_t m, int32_t groups) { return m <= NT_FEW && m * groups <= 120 + 5 * (int64_t)groups && m * groups * 34 <= NT_FEW_SMEM; }

static sat_status nt_launch_few(sat_ctx *ctx, int32_t m, const float *A, int32_t lda, const sat_mx_matrix *Aq, const sat_mx_matrix *W, const float *bias, float *C, int32_t ldc)
{
    const int32_t n = (int32_t)W->rows, k = W->d, groups = mx_groups(k);
    int32_t lpr = 1;
    while (lpr < groups && lpr < 32) lpr <<= 1;
    const unsigned blocks = (unsigned)cdiv64(n, NT_FEW_WARPS * (32 / lpr));
    const size_t smem = (size_t)m * groups * 34;
    static PerDeviceOnce attr;
    if (attr.need(ctx->device)) {
        SAT_CUDA(ctx, cudaFuncSetAttribute(k_mx_nt_few<1>, cudaFuncAttributeMaxDynamicSharedMemorySize, NT_FEW_SMEM));
        SAT_CUDA(ctx, cudaFuncSetAttribute(k_mx_nt_few<4>, cudaFuncAttributeMaxDynamicSharedMemorySize, NT_FEW_SMEM));
        SAT_CUDA(ctx, cudaFuncSetAttribute(k_mx_nt_few<NT_FEW>, cudaFuncAttributeMaxDynamicSharedMemorySize, NT_FEW_SMEM));
        attr.mark(ctx->device);
    }
    sat_pdl(ctx->stream, m == 1 ? k_mx_nt_few<1> : m <= 4 ? k_mx_nt_few<4> : k_mx_nt_few<NT_FEW>, blocks, 32 * NT_FEW_WARPS, smem)(
        A, (int64_t)lda, m, n, k, groups, lpr, Aq ? mx_view(Aq) : MxView{}, mx_view(W), bias, C, (int64_t)ldc);
    SAT_LAUNCHED(ctx);
    return SAT_OK;
}

template <bool STORED>
static sat_status nt_launch(sat_ctx *ctx, const CUtensorMap &map_a, const CUtensorMap &map_w, const CUtensorMap &map_c, const NtArgs &p)
{
    static PerDeviceOnce attr;
    if (attr.need(ctx->device)) {
        SAT_CUDA(ctx, cudaFuncSetAttribute(k_mx_nt<STORED>, cudaFuncAttributeMaxDynamicSharedMemorySize, NT_SMEM));
        attr.mark(ctx->device);
    }
    sat_pdl(ctx->stream, k_mx_nt<STORED>, (unsigned)std::min(p.tiles, ctx->sms), NT_THREADS, NT_SMEM)(map_a, map_w, map_c, p);
    SAT_LAUNCHED(ctx);
    return SAT_OK;
}

sat_status sat_mx_tc_nt(sat_ctx *ctx, int64_t m, const float *A, int32_t lda, const sat_mx_matrix *Aq, const sat_mx_matrix *W, const float *bias, float *C, int32_t ldc)
{
    if (nt_few(m, mx_groups(W->d))) return nt_launch_few(ctx, (int32_t)m, A, lda, Aq, W, bias, C, ldc);
    NtArgs p{};
    if (Aq) p.a = mx_view(Aq);
    p.w = mx_view(W);
    p.m = (int32_t)m;
    p.n = (int32_t)W->rows;
    p.k = W->d;
    p.groups = mx_groups(p.k);
    p.stages = (p.groups + 3) / 4;
    p.bn = mx_tile_columns(p.n);
    p.tiles_n = (int32_t)cdiv64(p.n, p.bn);
    if (cdiv64(m, 128) * p.tiles_n > INT32_MAX / 2) return sat_fail(ctx, SAT_EINVAL, "sat_mx_dense_nt: shape is too large");
    p.tiles = (int32_t)cdiv64(m, 128) * p.tiles_n;
    p.bias = bias;
    p.C = C;
    p.ldc = ldc;
    p.status = ctx->d_flag + 1;
    CUtensorMap map_a{}, map_w, map_c;
    if (A) SAT_TRY(sat_tensor_map(ctx, &map_a, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, A, p.k, m, (int64_t)lda * 4, 32, 128, CU_TENSOR_MAP_SWIZZLE_128B));
    SAT_TRY(sat_tensor_map(ctx, &map_w, CU_TENSOR_MAP_DATA_TYPE_UINT8, W->codes, mx_row_bytes(W), W->rows, W->ld_codes, NT_KB / 2, p.bn, CU_TENSOR_MAP_SWIZZLE_64B));
    SAT_TRY(sat_tensor_map(ctx, &map_c, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, C, p.n, m, (int64_t)ldc * 4, 32, 32, CU_TENSOR_MAP_SWIZZLE_128B));
    return A ? nt_launch<false>(ctx, map_a, map_w, map_c, p) : nt_launch<true>(ctx, map_a, map_w, map_c, p);
}

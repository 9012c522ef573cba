// Microscaled matrices: quantisation to and from groups of 32 elements with one power of two, and the contractions that read them.
//     group G of a row:  x ~ q 2^e,  e = least integer >= -127 with max |x| <= largest 2^e,  q = rne(x 2^-e) in e4m3 or e2m1
//   sat_mx_dense_nt   C = A^ W^^T + bias    both operands 4-bit
//   sat_mx_dense_nn   C = A W^              A fp32
//   sat_mx_dense_tn   C (+)= A^^T B         B fp32, split over the rows
#include "sat_mx.h"
#include "sat_ptx.h"

#include <algorithm>

static sat_status mx_check(sat_ctx *ctx, const sat_mx_matrix *q, const char *who)
{
    if (!q || (q->format != SAT_MX8 && q->format != SAT_MX4) || q->rows < 0 || q->rows > MX_MAX || q->d <= 0 || q->d > MX_MAX)
        return sat_fail(ctx, SAT_EINVAL, "%s: no microscaled matrix, or one of bad format or shape", who);
    if (q->rows > 0 && (!q->codes || !q->scales || !aligned16(q->codes) || ((uintptr_t)q->scales & 3)))
        return sat_fail(ctx, SAT_EINVAL, "%s: null or misaligned codes / scales", who);
    if (q->ld_codes < mx_row_bytes(q) || (q->ld_codes & 15) || q->ld_scales < mx_groups(q->d) || (q->ld_scales & 3))
        return sat_fail(ctx, SAT_EINVAL, "%s: bad row stride of codes or scales", who);
    return SAT_OK;
}

// =====================================================================================
// quantisation and back
// =====================================================================================
#define MX_UNROLL 4
// Eight lanes per group, four elements each.  One pass over the data; bound by memory.
template <int FMT>
__global__ void __launch_bounds__(256)
k_mx_quantise(const float *__restrict__ x, int64_t ld, int64_t total, int32_t groups, int32_t d, MxView q)
{
    sat_grid_wait();
    const int sub = threadIdx.x & 7;
    const int64_t step = (int64_t)gridDim.x * 32, first = (int64_t)blockIdx.x * 32 + (threadIdx.x >> 3);
    for (int64_t g0 = first - (threadIdx.x >> 3); g0 < total; g0 += MX_UNROLL * step) {   // (the same for the whole block: the lanes meet below)
        float4 v[MX_UNROLL];
        int64_t row[MX_UNROLL];
        int32_t col[MX_UNROLL];
#pragma unroll
        for (int u = 0; u < MX_UNROLL; ++u) {
            const int64_t g = g0 + (threadIdx.x >> 3) + u * step;
            v[u] = make_float4(0.f, 0.f, 0.f, 0.f);
            row[u] = -1;
            if (g < total) {
                row[u] = sat_div(g, groups);
                col[u] = (int32_t)(g - row[u] * groups) * MX_GROUP + 4 * sub;
                if (col[u] < d) v[u] = __ldg(reinterpret_cast<const float4 *>(x + row[u] * ld + col[u]));
                if (col[u] + 1 >= d) v[u].y = 0.f;   // what lies behind the row's end is not part of it
                if (col[u] + 2 >= d) v[u].z = 0.f;
                if (col[u] + 3 >= d) v[u].w = 0.f;
            }
        }
#pragma unroll
        for (int u = 0; u < MX_UNROLL; ++u) {
            uint32_t amax = max(max(__float_as_uint(v[u].x) & 0x7FFFFFFFu, __float_as_uint(v[u].y) & 0x7FFFFFFFu),
                                max(__float_as_uint(v[u].z) & 0x7FFFFFFFu, __float_as_uint(v[u].w) & 0x7FFFFFFFu));
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, o));
            if (row[u] < 0) continue;
            const uint32_t byte = mx_scale_byte<FMT>(amax);
            const float s = mx_inverse(byte);
            const uint32_t c = byte == 255u ? 0u : mx_encode4<FMT>(v[u].x * s, v[u].y * s, v[u].z * s, v[u].w * s);
            if (FMT == SAT_MX8) *reinterpret_cast<uint32_t *>(q.codes + row[u] * q.ld_codes + col[u]) = c;
            else *reinterpret_cast<uint16_t *>(q.codes + row[u] * q.ld_codes + col[u] / 2) = (uint16_t)c;
            if (sub == 0) q.scales[row[u] * q.ld_scales + (col[u] >> 5)] = (uint8_t)byte;
        }
    }
}

template <int FMT>
__global__ void __launch_bounds__(256)
k_mx_dequantise(MxView q, int64_t total, int32_t groups, int32_t d, float *__restrict__ x, int64_t ld)
{
    sat_grid_wait();
    const int sub = threadIdx.x & 7;
    const int64_t step = (int64_t)gridDim.x * 32;
    for (int64_t g0 = (int64_t)blockIdx.x * 32 + (threadIdx.x >> 3); g0 < total; g0 += MX_UNROLL * step) {
        uint32_t code[MX_UNROLL], byte[MX_UNROLL];
        int64_t row[MX_UNROLL];
        int32_t col[MX_UNROLL];
#pragma unroll
        for (int u = 0; u < MX_UNROLL; ++u) {
            const int64_t g = g0 + u * step;
            row[u] = -1;
            if (g < total) {
                row[u] = sat_div(g, groups);
                col[u] = (int32_t)(g - row[u] * groups) * MX_GROUP + 4 * sub;
                if (FMT == SAT_MX8) code[u] = __ldg(reinterpret_cast<const uint32_t *>(q.codes + row[u] * q.ld_codes + col[u]));
                else code[u] = __ldg(reinterpret_cast<const uint16_t *>(q.codes + row[u] * q.ld_codes + col[u] / 2));
                byte[u] = __ldg(q.scales + row[u] * q.ld_scales + (col[u] >> 5));
            }
        }
#pragma unroll
        for (int u = 0; u < MX_UNROLL; ++u) {
            if (row[u] < 0 || col[u] >= d) continue;
            const float s = mx_power(byte[u]);
            const float2 a = mx_unpack(mx_decode2<FMT>(code[u])), b = mx_unpack(mx_decode2<FMT>(code[u] >> (FMT == SAT_MX8 ? 16 : 8)));
            float *o = x + row[u] * ld + col[u];
            if (col[u] + 4 <= d) {
                *reinterpret_cast<float4 *>(o) = make_float4(a.x * s, a.y * s, b.x * s, b.y * s);
            } else {
                o[0] = a.x * s;
                if (col[u] + 1 < d) o[1] = a.y * s;
                if (col[u] + 2 < d) o[2] = b.x * s;
            }
        }
    }
}

// Matrices of some size: boxes of 128 rows by one group, a warpgroup to a box and a thread to a group, so that neither its maximum nor its scale is
// worked out more than once (the kernels above take nine times the instructions for an element).  fp32 rows go between memory and 128-byte
// rows of shared memory by TMA, three boxes per warpgroup in flight, and cross the banks swizzled.  612257 x 256 in 8 bits: 133 us, and 146 back (84 % of
// the copy rate together); 58241 x 602 in 4 bits 32 and 38.
#define MXB_SLOTS 3
#define MXB_BOX (128 * 32 * 4)
#define MXB_SMEM (1024 + 4 * MXB_SLOTS * MXB_BOX)
struct MxbShared {
    uint64_t full[4][MXB_SLOTS];
    int dead;
};
__device__ __forceinline__ void mxb_sync(int wg) { asm volatile("bar.sync %0, 128;" ::"r"(wg + 1) : "memory"); }

template <int FMT>
__global__ void __launch_bounds__(512, 1)
k_mx_quantise_boxes(const __grid_constant__ CUtensorMap map_x, int64_t boxes, int32_t groups, int64_t rows, int wide, MxView q, int *status)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    __shared__ MxbShared sh;
    const int wg = threadIdx.x >> 7, t = threadIdx.x & 127;
    if (threadIdx.x == 0) {
        for (int i = 0; i < 4 * MXB_SLOTS; ++i) mbar_init(&sh.full[i / MXB_SLOTS][i % MXB_SLOTS], 1);
        sh.dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    sat_grid_wait();
    const int64_t step = (int64_t)gridDim.x * 4;
    int64_t b = (int64_t)blockIdx.x * 4 + wg;
    uint8_t *mine = smem + wg * MXB_SLOTS * MXB_BOX;
    uint32_t issued = 0;
    auto load = [&](int slot, int64_t box) {
        if (t != 0 || box >= boxes || *(volatile int *)&sh.dead) return;
        ++issued;
        const int64_t tile = sat_div(box, groups);
        mbar_expect_tx(&sh.full[wg][slot], MXB_BOX);
        tma_load_2d(mine + slot * MXB_BOX, &map_x, &sh.full[wg][slot], (int32_t)(box - tile * groups) * MX_GROUP, (int32_t)tile * 128);
    };
    for (int i = 0; i < MXB_SLOTS; ++i) load(i, b + i * step);
    uint32_t slot = 0, ph = 0;
    for (; b < boxes; b += step) {
        (void)mbar_wait(&sh.full[wg][slot], ph, &sh.dead, status);   // (having given up, all finish on what is there)
        float4 v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const float4 *>(mine + slot * MXB_BOX + t * 128 + ((i ^ (t & 7)) << 4));
        fence_async_smem();   // these loads are done before the TMA writes there again (a barrier alone lets it overtake them)
        mxb_sync(wg);
        load((int)slot, b + MXB_SLOTS * step);
        if (++slot == MXB_SLOTS) slot = 0, ph ^= 1u;
        uint32_t c[FMT];
        const uint32_t byte = mx_quantise32<FMT>(v, c);
        const int64_t tile = sat_div(b, groups), r = tile * 128 + t;
        const int32_t g = (int32_t)(b - tile * groups);
        if (r < rows) {
            uint8_t *o = q.codes + r * q.ld_codes + g * (4 * FMT);
            if (FMT == SAT_MX8 && wide) {
                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(o), "r"(c[0]), "r"(c[1]), "r"(c[2]), "r"(c[3]), "r"(c[FMT - 4]), "r"(c[FMT - 3]),
                             "r"(c[FMT - 2]), "r"(c[FMT - 1])
                             : "memory");
            } else {
#pragma unroll
                for (int i = 0; i < FMT; i += 4) *reinterpret_cast<uint4 *>(o + 4 * i) = make_uint4(c[i], c[i + 1], c[i + 2], c[i + 3]);
            }
            q.scales[r * q.ld_scales + g] = (uint8_t)byte;
        }
    }
    if (t == 0 && *(volatile int *)&sh.dead) mbar_settle(sh.full[wg], MXB_SLOTS, issued);
}

template <int FMT>
__global__ void __launch_bounds__(512, 1)
k_mx_dequantise_boxes(const __grid_constant__ CUtensorMap map_x, int64_t boxes, int32_t groups, int64_t rows, int32_t d, MxView q, float *__restrict__ x, int64_t ld)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const int wg = threadIdx.x >> 7, t = threadIdx.x & 127;
    sat_grid_wait();
    const int64_t step = (int64_t)gridDim.x * 4;
    int64_t b = (int64_t)blockIdx.x * 4 + wg;
    uint8_t *mine = smem + wg * MXB_SLOTS * MXB_BOX;
    uint32_t next[FMT], next_byte = 0u;
    auto fetch = [&](int64_t box) {
        if (box >= boxes) return;
        const int64_t tile = sat_div(box, groups), r = tile * 128 + t;
        const int32_t g = (int32_t)(box - tile * groups);
        if (r >= rows) return;
        const uint8_t *o = q.codes + r * q.ld_codes + g * (4 * FMT);
#pragma unroll
        for (int i = 0; i < FMT; i += 4) {
            const uint4 w = __ldg(reinterpret_cast<const uint4 *>(o + 4 * i));
            next[i] = w.x, next[i + 1] = w.y, next[i + 2] = w.z, next[i + 3] = w.w;
        }
        next_byte = __ldg(q.scales + r * q.ld_scales + g);
    };
#pragma unroll
    for (int i = 0; i < FMT; ++i) next[i] = 0u;
    fetch(b);
    uint32_t slot = 0;
    for (; b < boxes; b += step) {
        uint32_t c[FMT];
#pragma unroll
        for (int i = 0; i < FMT; ++i) c[i] = next[i];
        const float s = mx_power(next_byte);
        fetch(b + step);
        uint8_t *box = mine + slot * MXB_BOX;
        if (t == 0) tma_store_wait_read<MXB_SLOTS - 1>();   // the box that was here has left
        mxb_sync(wg);
        // A bulk store writes whole 16 bytes: those of a row that are left are written from here
        const int64_t tile = sat_div(b, groups), r = tile * 128 + t;
        const int32_t col = (int32_t)(b - tile * groups) * MX_GROUP, left = r < rows ? d - (d & ~3) : 0, last = (d & ~3) - col;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t w = FMT == SAT_MX8 ? c[i % FMT] : c[(i / 2) % FMT] >> (16 * (i & 1));
            const float2 lo = mx_unpack(mx_decode2<FMT>(w)), hi = mx_unpack(mx_decode2<FMT>(w >> (FMT == SAT_MX8 ? 16 : 8)));
            const float4 v = make_float4(lo.x * s, lo.y * s, hi.x * s, hi.y * s);
            *reinterpret_cast<float4 *>(box + t * 128 + ((i ^ (t & 7)) << 4)) = v;
            if (4 * i == last) {
                float *o = x + r * ld + (d & ~3);
                if (left > 0) o[0] = v.x;
                if (left > 1) o[1] = v.y;
                if (left > 2) o[2] = v.z;
            }
        }
        if (last == 0) continue;
        fence_async_smem();
        mxb_sync(wg);
        if (t == 0) tma_store_2d(&map_x, box, col, (int32_t)tile * 128);
        if (++slot == MXB_SLOTS) slot = 0;
    }
    if (t == 0) tma_store_wait_all();
}

// From how many boxes on boxes are used, against threads that each take a group from memory.  Measured, threads against boxes, 256 columns:
// quantising 1000 rows (64 boxes) 2.2 / 2.4 us, 4000 rows (256) 3.6 / 2.5 us, 40000 rows (2504) 14.3 / 8.1 us;
// back to fp32 1000 rows 1.6 / 3.3 us, 9472 rows (592) 3.5 / 3.4 us, 20000 rows (1256) 5.7 / 6.5 us, 40000 rows in 4 bits 10.1 / 8.7 us.
#define MXB_LEAST_QUANTISE(ctx) ((int64_t)(ctx)->sms)
#define MXB_LEAST_DEQUANTISE(ctx) (16 * (int64_t)(ctx)->sms)

template <typename K, typename... A>
static sat_status mx_launch_boxes(sat_ctx *ctx, PerDeviceOnce &attr, K kernel, int64_t boxes, const A &...args)
{
    if (attr.need(ctx->device)) {
        SAT_CUDA(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, MXB_SMEM));
        attr.mark(ctx->device);
    }
    sat_pdl(ctx->stream, kernel, (unsigned)std::min<int64_t>(cdiv64(boxes, 4), ctx->sms), 512, MXB_SMEM)(args...);
    SAT_LAUNCHED(ctx);
    return SAT_OK;
}

sat_status sat_mx_quantise_rows(sat_ctx *ctx, const float *x, int32_t ld, const sat_mx_matrix *q)
{
    if (q->rows == 0) return SAT_OK;
    const int32_t groups = mx_groups(q->d);
    const int64_t total = q->rows * groups, blocks = std::min<int64_t>(cdiv64(total, 32), (int64_t)ctx->sms * 8), boxes = cdiv64(q->rows, 128) * groups;
    ProfScope prof(ctx, SATK_MX, (double)q->rows * (4.0 * q->d + mx_row_bytes(q) + groups), 0.0);
    if (boxes >= MXB_LEAST_QUANTISE(ctx)) {
        static PerDeviceOnce attr8, attr4;
        CUtensorMap map;
        SAT_TRY(sat_tensor_map(ctx, &map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, x, q->d, q->rows, (int64_t)ld * 4, MX_GROUP, 128, CU_TENSOR_MAP_SWIZZLE_128B));
        const int wide = !(((uintptr_t)q->codes | (uintptr_t)q->ld_codes) & 31);
        if (q->format == SAT_MX8) return mx_launch_boxes(ctx, attr8, k_mx_quantise_boxes<SAT_MX8>, boxes, map, boxes, groups, q->rows, wide, mx_view(q), ctx->d_flag + 1);
        return mx_launch_boxes(ctx, attr4, k_mx_quantise_boxes<SAT_MX4>, boxes, map, boxes, groups, q->rows, wide, mx_view(q), ctx->d_flag + 1);
    }
    sat_pdl(ctx->stream, q->format == SAT_MX8 ? k_mx_quantise<SAT_MX8> : k_mx_quantise<SAT_MX4>, (unsigned)blocks, 256, 0)(x, ld, total, groups, q->d, mx_view(q));
    SAT_LAUNCHED(ctx);
    return SAT_OK;
}

extern "C" sat_status sat_mx_quantise(sat_ctx *ctx, const float *x, int32_t ld, const sat_mx_matrix *q)
{
    CHECK_CTX(ctx);
    SAT_TRY(mx_check(ctx, q, "sat_mx_quantise"));
    if (!ok_ld(ld, q->d) || (q->rows > 0 && (!x || !aligned16(x)))) return sat_fail(ctx, SAT_EINVAL, "sat_mx_quantise: null / misaligned x or bad leading dimension");
    return sat_mx_quantise_rows(ctx, x, ld, q);
}

extern "C" sat_status sat_mx_dequantise(sat_ctx *ctx, const sat_mx_matrix *q, float *x, int32_t ld)
{
    CHECK_CTX(ctx);
    SAT_TRY(mx_check(ctx, q, "sat_mx_dequantise"));
    if (!ok_ld(ld, q->d) || (q->rows > 0 && (!x || !aligned16(x)))) return sat_fail(ctx, SAT_EINVAL, "sat_mx_dequantise: null / misaligned x or bad leading dimension");
    if (q->rows == 0) return SAT_OK;
    const int32_t groups = mx_groups(q->d);
    const int64_t total = q->rows * groups, blocks = std::min<int64_t>(cdiv64(total, 32), (int64_t)ctx->sms * 8), boxes = cdiv64(q->rows, 128) * groups;
    ProfScope prof(ctx, SATK_MX, (double)q->rows * (4.0 * q->d + mx_row_bytes(q) + groups), 0.0);
    if (boxes >= MXB_LEAST_DEQUANTISE(ctx)) {
        static PerDeviceOnce attr8, attr4;
        CUtensorMap map;
        SAT_TRY(sat_tensor_map(ctx, &map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, x, std::max(q->d & ~3, 4), q->rows, (int64_t)ld * 4, MX_GROUP, 128, CU_TENSOR_MAP_SWIZZLE_128B));
        if (q->format == SAT_MX8) return mx_launch_boxes(ctx, attr8, k_mx_dequantise_boxes<SAT_MX8>, boxes, map, boxes, groups, q->rows, q->d, mx_view(q), x, (int64_t)ld);
        return mx_launch_boxes(ctx, attr4, k_mx_dequantise_boxes<SAT_MX4>, boxes, map, boxes, groups, q->rows, q->d, mx_view(q), x, (int64_t)ld);
    }
    sat_pdl(ctx->stream, q->format == SAT_MX8 ? k_mx_dequantise<SAT_MX8> : k_mx_dequantise<SAT_MX4>, (unsigned)blocks, 256, 0)(mx_view(q), total, groups, q->d, x, ld);
    SAT_LAUNCHED(ctx);
    return SAT_OK;
}

// =====================================================================================
// contractions on CUDA cores: C[M x N] = sum_k a(i, k) b(k, j), tiles of 64 x 64, fp32 FMA
// =====================================================================================
enum { MX_NT = 0, MX_NN = 1, MX_TN = 2 };
struct MxSimple {
    MxView q1, q2;        // NT: A^, W^;  NN: -, W^;  TN: A^, -
    const float *x;       // NN: A;  TN: B
    int64_t ld_x;
    int64_t M, K, kps;    // kps: terms per block along z (TN)
    int32_t N;
    const float *bias;
    float *C, *cs;        // TN: partial sums [z][M x N] and [z][N]
    int64_t ldc;
};
template <int OP, int F1, int F2>
__global__ void __launch_bounds__(256)
k_mx_simple(MxSimple p)
{
    sat_grid_wait();
    __shared__ float As[16][68], Bs[16][68];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int64_t i0 = (int64_t)blockIdx.x * 64;
    const int32_t j0 = (int32_t)blockIdx.y * 64;
    const int64_t k0 = (int64_t)blockIdx.z * p.kps, k1 = k0 + p.kps < p.K ? k0 + p.kps : p.K;
    float acc[4][4] = {}, cs = 0.f;
    for (int64_t kb = k0; kb < k1; kb += 16) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int t = threadIdx.x + 256 * u;
            {
                const int kk = OP == MX_TN ? t >> 6 : t & 15, ii = OP == MX_TN ? t & 63 : t >> 4;   // along the rows in memory
                const int64_t k = kb + kk, i = i0 + ii;
                float a = 0.f;
                if (k < k1 && i < p.M) a = OP == MX_TN ? mx_element<F1>(p.q1, k, (int32_t)i) : OP == MX_NN ? __ldg(p.x + i * p.ld_x + k) : mx_element<F1>(p.q1, i, (int32_t)k);
                As[kk][ii] = a;
            }
            {
                const int kk = OP == MX_NT ? t & 15 : t >> 6, jj = OP == MX_NT ? t >> 4 : t & 63;
                const int64_t k = kb + kk;
                const int32_t j = j0 + jj;
                float b = 0.f;
                if (k < k1 && j < p.N) b = OP == MX_TN ? __ldg(p.x + k * p.ld_x + j) : OP == MX_NN ? mx_element<F2>(p.q2, k, j) : mx_element<F2>(p.q2, j, (int32_t)k);
                Bs[kk][jj] = b;
            }
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const float4 a = *reinterpret_cast<const float4 *>(&As[k][4 * ty]), b = *reinterpret_cast<const float4 *>(&Bs[k][4 * tx]);
            const float av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(av[i], bv[j], acc[i][j]);
        }
        if (OP == MX_TN && p.cs && blockIdx.x == 0 && threadIdx.x < 64)
            for (int k = 0; k < 16; ++k) cs += Bs[k][threadIdx.x];
        __syncthreads();
    }
    float *C = OP == MX_TN ? p.C + (int64_t)blockIdx.z * p.M * p.N : p.C;
    const int64_t ldc = OP == MX_TN ? p.N : p.ldc;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t r = i0 + 4 * ty + i;
            const int32_t c = j0 + 4 * tx + j;
            if (r < p.M && c < p.N) C[r * ldc + c] = acc[i][j] + (p.bias ? __ldg(p.bias + c) : 0.f);
        }
    if (OP == MX_TN && p.cs && blockIdx.x == 0 && threadIdx.x < 64 && j0 + (int32_t)threadIdx.x < p.N) p.cs[(int64_t)blockIdx.z * p.N + j0 + threadIdx.x] = cs;
}

// All contractions run on the tensor cores, however narrow and short, where the environment does not say otherwise.  Measured, k_mx_simple against them:
// A W^ of 1000 x 256 by 256 x 256 in 8 bits 38.6 / 8.5 us, of 1 x 40 by 40 x 256 6.6 / 4.8, of 83947 x 413 by 413 x 1 294 / 51; A^T B of 50758 x 17 by
// 50758 x 192 101 / 24, of 30 x 100 by 30 x 18 8.1 / 6.3; A^ W^T of 3000 x 64 by 8 16.8 / 4.7.  Where there is least to do k_mx_simple would save a little:
// A W^ of 2048 x 16 by 16 x 32 4.7 / 5.2 us, A^T B of 3 x 448 by 3 x 18 5.1 / 6.4.
static bool mx_tc() { return sat_use_tc(16, 16); }
static sat_status mx_grid(sat_ctx *ctx, int64_t M, int32_t N, int64_t splits, dim3 *grid)
{
    if (cdiv64(N, 64) > 65535 || splits > 65535 || cdiv64(M, 64) > INT32_MAX) return sat_fail(ctx, SAT_EINVAL, "microscaled contraction: shape is too large");
    *grid = dim3((unsigned)cdiv64(M, 64), (unsigned)cdiv64(N, 64), (unsigned)splits);
    return SAT_OK;
}

extern "C" sat_status sat_mx_dense_nt(sat_ctx *ctx, int64_t m, const float *A, int32_t lda, const sat_mx_matrix *Aq, const sat_mx_matrix *W,
                                      const float *bias, float *C, int32_t ldc)
{
    CHECK_CTX(ctx);
    SAT_TRY(mx_check(ctx, W, "sat_mx_dense_nt"));
    if (W->format != SAT_MX4 || (Aq && Aq->format != SAT_MX4)) return sat_fail(ctx, SAT_EINVAL, "sat_mx_dense_nt: operands are in 4 bits (SAT_MX4)");
    if (Aq) SAT_TRY(mx_check(ctx, Aq, "sat_mx_dense_nt"));
    if (m < 0 || m > MX_MAX || (Aq && (Aq->rows != m || Aq->d != W->d)) || W->rows == 0)
        return sat_fail(ctx, SAT_EINVAL, "sat_mx_dense_nt: shapes of the operands do not fit");
    const int32_t n = (int32_t)W->rows, k = W->d;
    if ((m > 0 && !A && !Aq) || (A && (!ok_ld(lda, k) || !aligned16(A))) || !ok_ld(ldc, n) || (m > 0 && (!C || !aligned16(C))))
        return sat_fail(ctx, SAT_EINVAL, "sat_mx_dense_nt: null / misaligned tensor or bad leading dimension");
    if (m == 0) return SAT_OK;
    ProfScope prof(ctx, SATK_MX, 4.0 * (double)m * (k + n), 2.0 * (double)m * n * k);
    if (mx_tc()) return sat_mx_tc_nt(ctx, m, A, lda, Aq, W, bias, C, ldc);
    sat_mx_matrix tmp;
    if (!Aq) {
        const int32_t groups = mx_groups(k), lds = (groups + 3) & ~3, ldq = groups * 16;
        SAT_TRY(sat_ensure(ctx, ctx->buf_mx, (size_t)m * (ldq + lds)));
        tmp = sat_mx_matrix{(uint8_t *)ctx->buf_mx.p, (uint8_t *)ctx->buf_mx.p + (size_t)m * ldq, m, k, ldq, lds, SAT_MX4};
        Aq = &tmp;
    }
    if (A) SAT_TRY(sat_mx_quantise_rows(ctx, A, lda, Aq));
    dim3 grid;
    SAT_TRY(mx_grid(ctx, m, n, 1, &grid));
    const MxSimple p{mx_view(Aq), mx_view(W), nullptr, 0, m, k, k, n, bias, C, nullptr, ldc};
    sat_pdl(ctx->stream, k_mx_simple<MX_NT, SAT_MX4, SAT_MX4>, grid, 256, 0)(p);
    SAT_LAUNCHED(ctx);
    return SAT_OK;
}

extern "C" sat_status sat_mx_dense_nn(sat_ctx *ctx, int64_t m, const float *A, int32_t lda, const sat_mx_matrix *W, float *C, int32_t ldc)
{
    CHECK_CTX(ctx);
    SAT_TRY(mx_check(ctx, W, "sat_mx_dense_nn"));
    const int32_t n = W->d, k = (int32_t)W->rows;
    if (m < 0 || m > MX_MAX || (k > 0 && !ok_ld(lda, k)) || !ok_ld(ldc, n) || (m > 0 && ((k > 0 && (!A || !aligned16(A))) || !C || !aligned16(C))))
        return sat_fail(ctx, SAT_EINVAL, "sat_mx_dense_nn: null / misaligned tensor or bad shape");
    if (m == 0) return SAT_OK;
    ProfScope prof(ctx, SATK_MX, 4.0 * (double)m * (k + n), 2.0 * (double)m * n * k);
    if (k > 0 && mx_tc()) return sat_mx_tc_nn(ctx, m, A, lda, W, C, ldc);
    dim3 grid;
    SAT_TRY(mx_grid(ctx, m, n, 1, &grid));
    const MxSimple p{MxView{}, mx_view(W), A, lda, m, k, k, n, nullptr, C, nullptr, ldc};
    sat_pdl(ctx->stream, W->format == SAT_MX8 ? k_mx_simple<MX_NN, SAT_MX8, SAT_MX8> : k_mx_simple<MX_NN, SAT_MX4, SAT_MX4>, grid, 256, 0)(p);
    SAT_LAUNCHED(ctx);
    return SAT_OK;
}

sat_status sat_mx_gradient(sat_ctx *ctx, const sat_mx_matrix *A, int32_t n, const float *B, int32_t ldb, float *C, float *colsum, int accumulate)
{
    const int32_t m = A->d;
    ProfScope prof(ctx, SATK_MX, (double)A->rows * (mx_row_bytes(A) + mx_groups(m) + 4.0 * n), 2.0 * (double)A->rows * m * n);
    if (A->rows > 0 && mx_tc()) return sat_mx_tc_tn(ctx, A, n, B, ldb, C, colsum, accumulate);
    const int64_t rows = A->rows > 0 ? A->rows : 1, tiles = cdiv64(m, 64) * cdiv64(n, 64);
    int64_t splits = std::max<int64_t>(cdiv64(rows, 4096), std::min<int64_t>(cdiv64(4 * ctx->sms, tiles), cdiv64(rows, 64)));
    if (splits > 1024) splits = 1024;
    const int64_t kps = cdiv64(cdiv64(rows, splits), 16) * 16;
    splits = cdiv64(rows, kps);
    SAT_TRY(sat_ensure(ctx, ctx->buf_splitk, (size_t)splits * ((size_t)m * n + n) * sizeof(float)));
    float *part = (float *)ctx->buf_splitk.p, *part_cs = colsum ? part + (size_t)splits * m * n : nullptr;
    dim3 grid;
    SAT_TRY(mx_grid(ctx, m, n, splits, &grid));
    const MxSimple p{mx_view(A), MxView{}, B, ldb, m, A->rows, kps, n, nullptr, part, part_cs, n};
    sat_pdl(ctx->stream, A->format == SAT_MX8 ? k_mx_simple<MX_TN, SAT_MX8, SAT_MX8> : k_mx_simple<MX_TN, SAT_MX4, SAT_MX4>, grid, 256, 0)(p);
    SAT_LAUNCHED(ctx);
    return sat_splitk_reduce(ctx, part, (int64_t)m * n, (int32_t)splits, accumulate, C, n, n, part_cs, n, colsum);
}

extern "C" sat_status sat_mx_dense_tn(sat_ctx *ctx, const sat_mx_matrix *A, int32_t n, const float *B, int32_t ldb, float *C, float *colsum, int accumulate)
{
    CHECK_CTX(ctx);
    SAT_TRY(mx_check(ctx, A, "sat_mx_dense_tn"));
    if (n <= 0 || !C || !ok_ld(ldb, n) || (A->rows > 0 && (!B || !aligned16(B))) || (accumulate != 0 && accumulate != 1))
        return sat_fail(ctx, SAT_EINVAL, "sat_mx_dense_tn: null / misaligned tensor or bad shape");
    return sat_mx_gradient(ctx, A, n, B, ldb, C, colsum, accumulate);
}

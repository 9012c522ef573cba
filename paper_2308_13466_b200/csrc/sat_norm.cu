// Layer norm by rows, forward and backward:
//     mu = sum x / d,  s = (sum (x - mu)^2 / d + eps)^(-1/2),  xh = (x - mu) s,  y = xh gamma + beta
//     u = g gamma,  g_x = s (u - sum u / d - xh sum (u xh) / d),  g_gamma = sum over rows g xh,  g_beta = sum over rows g
#include "sat_rows.h"

#include <algorithm>

#define NORM_MAX 16384   // width: a row lies in the registers of one block

// TPR threads hold a row in registers, CH times 16 bytes each.
#define NORM_THREADS(TPR) ((TPR) > 32 ? (TPR) : 256)   // of a block

template <typename T, int TPR, int CH>
__global__ void __launch_bounds__(NORM_THREADS(TPR))
k_norm_fwd(int64_t rows, int32_t d, const T *x, int64_t ld_x, const float *__restrict__ gamma, const float *__restrict__ beta, float eps, T *y,
           int64_t ld_y, float *__restrict__ mean, float *__restrict__ rstd)
{
    sat_grid_wait();
    constexpr int V = RowVec<T>::V, NT = NORM_THREADS(TPR), RPB = NT / TPR;
    __shared__ float2 red[2][32];
    int turn = 0;
    const int t = threadIdx.x % TPR;
    const float inv_d = 1.f / (float)d;
    for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < rows; r0 += (int64_t)gridDim.x * RPB) {
        const int64_t r = r0 + threadIdx.x / TPR;
        const bool ok = r < rows;
        float v[CH][V];
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            row_load(x + (ok ? r : 0) * ld_x, ok ? (j * TPR + t) * V : d, d, v[j]);
#pragma unroll
            for (int i = 0; i < V; ++i) s += v[j][i];
        }
        const float m0 = row_sum2<TPR>(s, 0.f, red, turn).x * inv_d;
        // what the rounding of the mean left is taken off with the squares
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int j = 0; j < CH; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                v[j][i] = (j * TPR + t) * V + i < d ? v[j][i] - m0 : 0.f;
                a += v[j][i];
                b = fmaf(v[j][i], v[j][i], b);
            }
        const float2 ab = row_sum2<TPR>(a, b, red, turn);
        const float m1 = ab.x * inv_d, var = fmaxf(ab.y * inv_d - m1 * m1, 0.f), sd = 1.f / sqrtf(var + eps);
        if (!ok) continue;
        if (t == 0) {
            if (mean) mean[r] = m0 + m1;
            if (rstd) rstd[r] = sd;
        }
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int32_t col = (j * TPR + t) * V;
            if (col >= d) continue;
            float ga[V], be[V];
            param_load<V>(gamma, col, d, 1.f, ga);
            param_load<V>(beta, col, d, 0.f, be);
#pragma unroll
            for (int i = 0; i < V; ++i) v[j][i] = fmaf((v[j][i] - m1) * sd, ga[i], be[i]);
            row_store(y + r * ld_y, col, d, v[j]);
        }
    }
}

// The sums over the rows: a thread adds up its columns over the block's rows in registers, the block leaves one row of partial sums
// [g_gamma | g_beta], k_norm_sums adds these up in a fixed order.
template <typename T, int TPR, int CH>
__global__ void __launch_bounds__(NORM_THREADS(TPR))
k_norm_bwd(int64_t rows, int32_t d, const T *x, int64_t ld_x, const T *g, int64_t ld_g, const float *__restrict__ gamma,
           const float *__restrict__ mean, const float *__restrict__ rstd, T *gx, int64_t ld_gx, float *__restrict__ part, int32_t ld_part)
{
    sat_grid_wait();
    constexpr int V = RowVec<T>::V, NT = NORM_THREADS(TPR), RPB = NT / TPR;
    __shared__ float2 red[2][32];
    int turn = 0;
    const int t = threadIdx.x % TPR;
    const float inv_d = 1.f / (float)d;
    float ag[CH][V] = {}, ab[CH][V] = {};
    for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < rows; r0 += (int64_t)gridDim.x * RPB) {
        const int64_t r = r0 + threadIdx.x / TPR;
        const bool ok = r < rows;
        float xh[CH][V], u[CH][V];
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int32_t col = ok ? (j * TPR + t) * V : d;
            row_load(x + (ok ? r : 0) * ld_x, col, d, xh[j]);
            row_load(g + (ok ? r : 0) * ld_g, col, d, u[j]);
        }
        const float m = ok ? __ldg(mean + r) : 0.f, sd = ok ? __ldg(rstd + r) : 0.f;
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int32_t col = (j * TPR + t) * V;
            float ga[V];
            param_load<V>(gamma, col, d, 1.f, ga);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                xh[j][i] = ok && col + i < d ? (xh[j][i] - m) * sd : 0.f;
                ag[j][i] = fmaf(u[j][i], xh[j][i], ag[j][i]);
                ab[j][i] += u[j][i];
                u[j][i] *= ga[i];
                s1 += u[j][i];
                s2 = fmaf(u[j][i], xh[j][i], s2);
            }
        }
        if (!gx) continue;   // (the same for all threads)
        const float2 s = row_sum2<TPR>(s1, s2, red, turn);
        const float c1 = s.x * inv_d, c2 = s.y * inv_d;
        if (!ok) continue;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int32_t col = (j * TPR + t) * V;
            if (col >= d) continue;
#pragma unroll
            for (int i = 0; i < V; ++i) u[j][i] = sd * (u[j][i] - fmaf(xh[j][i], c2, c1));
            row_store(gx + r * ld_gx, col, d, u[j]);
        }
    }
    if (!part) return;
    float *out = part + (int64_t)blockIdx.x * 2 * ld_part;
    if constexpr (RPB == 1) {
#pragma unroll
        for (int j = 0; j < CH; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int32_t col = (j * TPR + t) * V + i;
                if (col < d) out[col] = ag[j][i], out[ld_part + col] = ab[j][i];
            }
    } else {
        __shared__ float sum[2][TPR * V];
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            for (int w = 0; w < RPB; ++w) {   // one group of rows after the other
                __syncthreads();
                if (threadIdx.x / TPR == w) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        sum[0][t * V + i] = w ? sum[0][t * V + i] + ag[j][i] : ag[j][i];
                        sum[1][t * V + i] = w ? sum[1][t * V + i] + ab[j][i] : ab[j][i];
                    }
                }
            }
            __syncthreads();
            for (int c = threadIdx.x; c < 2 * TPR * V; c += NT) {
                const int which = c / (TPR * V), i = c % (TPR * V), col = j * TPR * V + i;
                if (col < d) out[which * ld_part + col] = sum[which][i];
            }
        }
    }
}

// out[c] (+)= sum over b of part[b][c]: 32 columns a block, eight threads a column
__global__ void __launch_bounds__(256)
k_norm_sums(const float *__restrict__ part, int32_t blocks, int32_t d, int32_t ld_part, int accumulate, float *__restrict__ g_gamma, float *__restrict__ g_beta)
{
    sat_grid_wait();
    __shared__ float red[8][32];
    const int32_t col = (int32_t)blockIdx.x * 32 + (threadIdx.x & 31);
    const int w = threadIdx.x >> 5;
    float *out = blockIdx.y ? g_beta : g_gamma;
    if (!out) return;
    float s = 0.f;
    if (col < d)
        for (int32_t b = w; b < blocks; b += 8) s += __ldcg(part + ((int64_t)b * 2 + blockIdx.y) * ld_part + col);
    red[w][threadIdx.x & 31] = s;
    __syncthreads();
    if (w == 0 && col < d) {
        for (int i = 1; i < 8; ++i) s += red[i][threadIdx.x];
        out[col] = accumulate ? out[col] + s : s;
    }
}

template <typename T>
struct NormArgs {
    sat_ctx *ctx;
    int64_t rows;
    int32_t d;
    const T *x, *g;
    int64_t ld_x, ld_g, ld_y;
    const float *gamma, *beta;
    float eps;
    T *y;                 // or g_x
    float *mean, *rstd;
    float *part;          // backward: partial sums of `blocks` blocks
    int32_t ld_part, blocks;
};
template <typename T, int TPR, int CH>
static void norm_go(const NormArgs<T> &a, bool back)
{
    constexpr int NT = NORM_THREADS(TPR), RPB = NT / TPR;
    if (back) {
        sat_pdl(a.ctx->stream, k_norm_bwd<T, TPR, CH>, (unsigned)a.blocks, NT, 0)(a.rows, a.d, a.x, a.ld_x, a.g, a.ld_g, a.gamma, a.mean, a.rstd, a.y, a.ld_y, a.part,
                                                                                   a.ld_part);
    } else {
        const int64_t blocks = std::min<int64_t>(cdiv64(a.rows, RPB), (int64_t)a.ctx->sms * (2048 / NT));
        sat_pdl(a.ctx->stream, k_norm_fwd<T, TPR, CH>, (unsigned)blocks, NT, 0)(a.rows, a.d, a.x, a.ld_x, a.gamma, a.beta, a.eps, a.y, a.ld_y, a.mean, a.rstd);
    }
}
// threads of a row: as few as hold it with up to eight (a block: four) pieces of 16 bytes each, so that sums cross few lanes
static int norm_tpr(int32_t pieces) { return pieces <= 8 ? 8 : pieces <= 16 ? 16 : pieces <= 256 ? 32 : pieces <= 512 ? 128 : pieces <= 1024 ? 256 : pieces <= 2048 ? 512 : 1024; }
template <typename T>
static void norm_launch(const NormArgs<T> &a, bool back)
{
    const int32_t pieces = (a.d + RowVec<T>::V - 1) / RowVec<T>::V;
    const int tpr = norm_tpr(pieces), ch = (pieces + tpr - 1) / tpr;
    switch (tpr) {
    case 8: return norm_go<T, 8, 1>(a, back);
    case 16: return norm_go<T, 16, 1>(a, back);
    case 32:
        if (ch == 1) return norm_go<T, 32, 1>(a, back);
        if (ch == 2) return norm_go<T, 32, 2>(a, back);
        if (ch == 3) return norm_go<T, 32, 3>(a, back);
        if (ch == 4) return norm_go<T, 32, 4>(a, back);
        if (ch <= 6) return norm_go<T, 32, 6>(a, back);
        return norm_go<T, 32, 8>(a, back);
    case 128: return ch <= 3 ? norm_go<T, 128, 3>(a, back) : norm_go<T, 128, 4>(a, back);
    case 256: return ch <= 3 ? norm_go<T, 256, 3>(a, back) : norm_go<T, 256, 4>(a, back);
    case 512: return ch <= 3 ? norm_go<T, 512, 3>(a, back) : norm_go<T, 512, 4>(a, back);
    default: return ch <= 3 ? norm_go<T, 1024, 3>(a, back) : norm_go<T, 1024, 4>(a, back);
    }
}

static sat_status norm_check(sat_ctx *ctx, const char *who, int64_t rows, int32_t d, int type)
{
    if (!ok_type(type)) return sat_fail(ctx, SAT_EINVAL, "%s: unknown element type", who);
    if (rows < 0 || rows >= INT32_MAX || d <= 0 || d > NORM_MAX) return sat_fail(ctx, SAT_EINVAL, "%s: rows must be in [0, 2^31 - 1), the width in [1, %d]", who, NORM_MAX);
    return SAT_OK;
}
static bool norm_param_ok(const float *p) { return !p || aligned16(p); }

template <typename T>
static void norm_fwd_as(sat_ctx *ctx, int64_t rows, int32_t d, const void *x, int32_t ld_x, const float *gamma, const float *beta, float eps, void *y, int32_t ld_y,
                        float *mean, float *rstd)
{
    NormArgs<T> a = {};
    a.ctx = ctx, a.rows = rows, a.d = d, a.x = (const T *)x, a.ld_x = ld_x, a.gamma = gamma, a.beta = beta, a.eps = eps, a.y = (T *)y, a.ld_y = ld_y;
    a.mean = mean, a.rstd = rstd;
    norm_launch(a, false);
}

extern "C" sat_status sat_layernorm_fwd(sat_ctx *ctx, int64_t rows, int32_t d, int type, const void *x, int32_t ld_x, const float *gamma, const float *beta,
                                        float eps, void *y, int32_t ld_y, float *mean, float *rstd)
{
    CHECK_CTX(ctx);
    SAT_TRY(norm_check(ctx, "sat_layernorm_fwd", rows, d, type));
    if (!(eps >= 0.f) || !ok_ld_of(type, ld_x, d) || !ok_ld_of(type, ld_y, d) || !norm_param_ok(gamma) || !norm_param_ok(beta) ||
        (rows > 0 && (!x || !y || !aligned16(x) || !aligned16(y))))
        return sat_fail(ctx, SAT_EINVAL, "sat_layernorm_fwd: null / misaligned tensor, bad leading dimension or negative eps");
    if (rows == 0) return SAT_OK;
    ProfScope prof(ctx, SATK_NORM, 2.0 * type_bytes(type) * (double)rows * d, 8.0 * (double)rows * d);
    if (type == SAT_F32) norm_fwd_as<float>(ctx, rows, d, x, ld_x, gamma, beta, eps, y, ld_y, mean, rstd);
    else if (type == SAT_BF16) norm_fwd_as<__nv_bfloat16>(ctx, rows, d, x, ld_x, gamma, beta, eps, y, ld_y, mean, rstd);
    else norm_fwd_as<__half>(ctx, rows, d, x, ld_x, gamma, beta, eps, y, ld_y, mean, rstd);
    SAT_LAUNCHED(ctx);
    return SAT_OK;
}

template <typename T>
static void norm_bwd_as(sat_ctx *ctx, int64_t rows, int32_t d, const void *x, int32_t ld_x, const void *g, int32_t ld_g, const float *gamma, const float *mean,
                        const float *rstd, void *g_x, int32_t ld_gx, float *part, int32_t ld_part, int32_t blocks)
{
    NormArgs<T> a = {};
    a.ctx = ctx, a.rows = rows, a.d = d, a.x = (const T *)x, a.ld_x = ld_x, a.g = (const T *)g, a.ld_g = ld_g, a.gamma = gamma, a.y = (T *)g_x, a.ld_y = ld_gx;
    a.mean = const_cast<float *>(mean), a.rstd = const_cast<float *>(rstd), a.part = part, a.ld_part = ld_part, a.blocks = blocks;
    norm_launch(a, true);
}

extern "C" sat_status sat_layernorm_bwd(sat_ctx *ctx, int64_t rows, int32_t d, int type, const void *x, int32_t ld_x, const void *g, int32_t ld_g,
                                        const float *gamma, const float *mean, const float *rstd, void *g_x, int32_t ld_gx, float *g_gamma, float *g_beta,
                                        int accumulate)
{
    CHECK_CTX(ctx);
    SAT_TRY(norm_check(ctx, "sat_layernorm_bwd", rows, d, type));
    if (!ok_ld_of(type, ld_x, d) || !ok_ld_of(type, ld_g, d) || (g_x && !ok_ld_of(type, ld_gx, d)) || !norm_param_ok(gamma) || (g_x && !aligned16(g_x)) ||
        (rows > 0 && (!x || !g || !mean || !rstd || !aligned16(x) || !aligned16(g))))
        return sat_fail(ctx, SAT_EINVAL, "sat_layernorm_bwd: null / misaligned tensor or bad leading dimension");
    if (accumulate != 0 && accumulate != 1) return sat_fail(ctx, SAT_EINVAL, "sat_layernorm_bwd: accumulate is 0 or 1");
    const bool params = g_gamma || g_beta;
    if (!g_x && !params) return sat_fail(ctx, SAT_EINVAL, "sat_layernorm_bwd: no result is asked for");
    if (rows == 0) {
        if (!accumulate && g_gamma) SAT_CUDA(ctx, cudaMemsetAsync(g_gamma, 0, (size_t)d * sizeof(float), ctx->stream));
        if (!accumulate && g_beta) SAT_CUDA(ctx, cudaMemsetAsync(g_beta, 0, (size_t)d * sizeof(float), ctx->stream));
        return SAT_OK;
    }
    const int32_t pieces = (d + 16 / type_bytes(type) - 1) / (16 / type_bytes(type));
    const int tpr = norm_tpr(pieces), nt = tpr > 32 ? tpr : 256;
    const int32_t blocks = (int32_t)std::min<int64_t>(cdiv64(rows, nt / tpr), (int64_t)ctx->sms * std::max(1, 1024 / nt));
    const int32_t ld_part = round_up4(d);
    float *part = nullptr;
    if (params) {
        SAT_TRY(sat_ensure(ctx, ctx->buf_norm, (size_t)blocks * 2 * ld_part * sizeof(float)));
        part = (float *)ctx->buf_norm.p;
    }
    ProfScope prof(ctx, SATK_NORM, (g_x ? 3.0 : 2.0) * type_bytes(type) * (double)rows * d, 14.0 * (double)rows * d);
    if (type == SAT_F32) norm_bwd_as<float>(ctx, rows, d, x, ld_x, g, ld_g, gamma, mean, rstd, g_x, ld_gx, part, ld_part, blocks);
    else if (type == SAT_BF16) norm_bwd_as<__nv_bfloat16>(ctx, rows, d, x, ld_x, g, ld_g, gamma, mean, rstd, g_x, ld_gx, part, ld_part, blocks);
    else norm_bwd_as<__half>(ctx, rows, d, x, ld_x, g, ld_g, gamma, mean, rstd, g_x, ld_gx, part, ld_part, blocks);
    SAT_LAUNCHED(ctx);
    if (params) {
        sat_pdl(ctx->stream, k_norm_sums, dim3((unsigned)cdiv64(d, 32), 2), 256, 0)(part, blocks, d, ld_part, accumulate, g_gamma, g_beta);
        SAT_LAUNCHED(ctx);
    }
    return SAT_OK;
}

// Distillation from a teacher's top logits, the loss and its gradient in one pass:
//     p = softmax(t / T) over the k entries (id, t) of a row,   q = softmax(z / T),   q1 = softmax(z)
//     loss = (1 - h) T^2 sum_j p_j (log p_j - log q_{id_j}) + h (-log q1_y)
//     g_c = w [ (1 - h) T (q_c - sum_{j: id_j = c} p_j) + h (q1_c - [c = y]) ]
#include "sat_loss.h"
#include "sat_rows.h"

#include <algorithm>

#define DISTILL_MAX_K 256
#define LOG2E 1.4426950408889634f

struct Distill {
    int64_t rows;
    int32_t C, k;
    int64_t ld_z, ld_g;
    const int32_t *ids;
    const float *logits;
    float T, hard;
    const int32_t *labels;
    const float *row_weight;
    float weight;
    float *row_loss;
    double *block_partial;
    int *ticket;
    double *loss_sum;
    int *status;
};

// an entry of the teacher's row; -1 where there is none: no id, or a logit of -inf, which has no weight
__device__ __forceinline__ int32_t distill_entry(const Distill &p, int64_t row, int32_t j, float &t)
{
    const int32_t id = __ldg(p.ids + row * p.k + j);
    t = __ldg(p.logits + row * p.k + j);
    if (id >= p.C) {
        atomicOr(p.status, 8);
        return -1;
    }
    return id < 0 || t == -INFINITY ? -1 : id;
}
__device__ __forceinline__ int32_t distill_label(const Distill &p, int64_t row)
{
    const int32_t y = p.hard > 0.f ? __ldg(p.labels + row) : -1;
    if (y >= p.C) {
        atomicOr(p.status, 8);
        return -1;
    }
    return y < 0 ? -1 : y;
}

// Up to 1,024 classes: TPR lanes hold a row in registers.  The teacher's probabilities meet their columns in shared memory, which is all zeros between rows.
template <typename T, int TPR, int CH, bool HARD>
__global__ void __launch_bounds__(256)
k_distill_rows(Distill p, const T *__restrict__ z, T *__restrict__ g)
{
    sat_grid_wait();
    constexpr int V = RowVec<T>::V, RPW = 32 / TPR;
    extern __shared__ float4 distill_smem[];
    const int lane = threadIdx.x & 31, t = lane % TPR;
    const unsigned mates = TPR == 32 ? 0xffffffffu : ((1u << (TPR & 31)) - 1u) << (lane - t);
    float *sp = reinterpret_cast<float *>(distill_smem) + (threadIdx.x / TPR) * (TPR * CH * V);
    for (int i = t; i < TPR * CH * V; i += TPR) sp[i] = 0.f;
    __syncwarp();
    float2 (*none)[32] = nullptr;
    int turn = 0;
    const float cT = LOG2E / p.T, inv_T = 1.f / p.T;
    double acc = 0.0;
    for (int64_t rw = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 5; rw * RPW < p.rows; rw += (int64_t)gridDim.x * 8) {
        const int64_t r = rw * RPW + lane / TPR;
        const bool ok = r < p.rows;
        const int64_t row = ok ? r : p.rows - 1;
        const T *zr = z + row * p.ld_z;
        const float w = p.weight * (p.row_weight ? __ldg(p.row_weight + row) : 1.f);
        const int32_t y = HARD ? distill_label(p, row) : -1;
        const float zy = y >= 0 ? RowVec<T>::from(zr[y]) : 0.f;   // (before g is written, which may be z)
        float v[CH][V], e1[HARD ? CH : 1][V];
        float m = -INFINITY;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int32_t col = (j * TPR + t) * V;
            row_load(zr, col, p.C, v[j]);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (col + i >= p.C) v[j][i] = -INFINITY;
                m = fmaxf(m, v[j][i]);
            }
        }
        float tm = -INFINITY;
        bool some = false;
        for (int32_t j0 = 0; j0 < p.k; j0 += TPR) {
            float tj = 0.f;
            const int32_t id = j0 + t < p.k ? distill_entry(p, row, j0 + t, tj) : -1;
            if (id >= 0) tm = fmaxf(tm, tj);
            some |= (__ballot_sync(0xffffffffu, id >= 0) & mates) != 0;
        }
#pragma unroll
        for (int o = TPR / 2; o > 0; o >>= 1) {
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            tm = fmaxf(tm, __shfl_xor_sync(0xffffffffu, tm, o));
        }
        float s = 0.f, s1 = 0.f;
#pragma unroll
        for (int j = 0; j < CH; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const bool in = (j * TPR + t) * V + i < p.C;
                const float x = v[j][i] - m;
                v[j][i] = in ? ex2_fast(x * cT) : 0.f;
                s += v[j][i];
                if (HARD) {
                    e1[j][i] = in ? ex2_fast(x * LOG2E) : 0.f;
                    s1 += e1[j][i];
                }
            }
        float st = 0.f, num = 0.f;
        for (int32_t j0 = 0; j0 < p.k; j0 += TPR) {
            float tj = 0.f;
            const int32_t id = j0 + t < p.k ? distill_entry(p, row, j0 + t, tj) : -1;
            float e = 0.f;
            if (id >= 0) {
                e = ex2_fast((tj - tm) * cT);
                st += e;
                if (!(e <= 0.f)) num = fmaf(e, (tj - tm) - (RowVec<T>::from(zr[id]) - m), num);
            }
            // the same class more than once: its first lane adds up, in order
            const unsigned same = __match_any_sync(0xffffffffu, id) & mates;
            float sum = e;
            if (__any_sync(0xffffffffu, id >= 0 && same != (1u << lane))) {
                sum = 0.f;
                for (int i = 0; i < 32; ++i) {
                    const float other = __shfl_sync(0xffffffffu, e, i);
                    if ((same >> i) & 1u) sum += other;
                }
            }
            if (id >= 0 && (same & ((1u << lane) - 1u)) == 0) sp[id] += sum;
            __syncwarp();
        }
        const float2 sums = row_sum2<TPR>(s, s1, none, turn), ts = row_sum2<TPR>(st, num, none, turn);
        s = sums.x, s1 = sums.y;
        if (ok) {
            const bool soft_on = some && p.hard < 1.f, hard_on = HARD && y >= 0;
            const float a = soft_on ? w * (1.f - p.hard) * p.T : 0.f, b = hard_on ? w * p.hard : 0.f;
            const float aq = soft_on ? a / s : 0.f, ap = soft_on ? a / ts.x : 0.f, bq = hard_on ? b / s1 : 0.f;
            T *gr = g + r * p.ld_g;
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const int32_t col = (j * TPR + t) * V;
                if (col >= p.C) continue;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float x = soft_on ? aq * v[j][i] - ap * sp[col + i] : 0.f;
                    if (HARD && hard_on) x += bq * e1[j][i] - (col + i == y ? b : 0.f);
                    v[j][i] = w == 0.f ? 0.f : x;
                }
                if (g) row_store(gr, col, p.C, v[j]);
            }
            if (t == 0) {
                float loss = 0.f;
                if (w != 0.f) {
                    if (soft_on) loss = (1.f - p.hard) * p.T * p.T * (ts.y / ts.x * inv_T + (logf(s) - logf(ts.x)));
                    if (hard_on) loss += p.hard * (logf(s1) - (zy - m));
                }
                if (p.row_loss) p.row_loss[r] = loss;
                acc += (double)w * (double)loss;
            }
        }
        __syncwarp();
        for (int32_t j = t; j < p.k; j += TPR) {
            const int32_t id = __ldg(p.ids + row * p.k + j);
            if (id >= 0 && id < p.C) sp[id] = 0.f;
        }
        __syncwarp();
    }
    if (p.loss_sum) loss_finish(acc, p.block_partial, p.ticket, p.loss_sum, 0);
}

// Any number of classes: a block per row, two passes over it.
#define DISTILL_NT 512
template <typename T, bool HARD>
__global__ void __launch_bounds__(DISTILL_NT)
k_distill_wide(Distill p, const T *__restrict__ z, T *__restrict__ g)
{
    sat_grid_wait();
    constexpr int V = RowVec<T>::V, NT = DISTILL_NT;
    __shared__ int32_t sid[DISTILL_MAX_K + 1];
    __shared__ float se[DISTILL_MAX_K], smax[2][NT / 32], szy;
    __shared__ float2 red[2][32];
    int turn = 0;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const float cT = LOG2E / p.T, inv_T = 1.f / p.T;
    double acc = 0.0;
    for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
        const T *zr = z + r * p.ld_z;
        const float w = p.weight * (p.row_weight ? __ldg(p.row_weight + r) : 1.f);
        const int32_t y = HARD ? distill_label(p, r) : -1;
        float tj = 0.f;
        const int32_t id = tid < p.k ? distill_entry(p, r, tid, tj) : -1;
        const int32_t mine = tid == p.k ? y : id;                        // the thread behind the entries has the label
        const float zc = mine >= 0 ? RowVec<T>::from(zr[mine]) : 0.f;    // (before g is written, which may be z)
        // running maximum and sums
        float m = -INFINITY, s = 0.f, s1 = 0.f;
        for (int32_t col = tid * V; col < p.C; col += NT * V) {
            float v[V];
            row_load(zr, col, p.C, v);
            float top = m;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (col + i >= p.C) v[i] = -INFINITY;
                top = fmaxf(top, v[i]);
            }
            const float from = top == -INFINITY ? 0.f : top;
            if (top > m) {
                s *= ex2_fast((m - from) * cT);
                if (HARD) s1 *= ex2_fast((m - from) * LOG2E);
                m = top;
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                s += ex2_fast((v[i] - from) * cT);
                if (HARD) s1 += ex2_fast((v[i] - from) * LOG2E);
            }
        }
        float M = m, tm = id >= 0 ? tj : -INFINITY;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
            tm = fmaxf(tm, __shfl_xor_sync(0xffffffffu, tm, o));
        }
        if (lane == 0) smax[0][warp] = M, smax[1][warp] = tm;
        const bool some = __syncthreads_or(id >= 0);
        M = smax[0][lane % (NT / 32)], tm = smax[1][lane % (NT / 32)];
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) {
            M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
            tm = fmaxf(tm, __shfl_xor_sync(0xffffffffu, tm, o));
        }
        if (m != -INFINITY) {
            s *= ex2_fast((m - M) * cT);
            if (HARD) s1 *= ex2_fast((m - M) * LOG2E);
        }
        float st = 0.f, num = 0.f;
        if (id >= 0) {
            st = ex2_fast((tj - tm) * cT);
            if (!(st <= 0.f)) num = st * ((tj - tm) - (zc - M));
        }
        if (tid < p.k) sid[tid] = id, se[tid] = st;
        if (tid == p.k) sid[tid] = y, szy = zc;
        const float2 sums = row_sum2<NT>(s, s1, red, turn), ts = row_sum2<NT>(st, num, red, turn);
        s = sums.x, s1 = sums.y;
        const bool soft_on = some && p.hard < 1.f, hard_on = HARD && y >= 0;
        if (tid == 0) {
            float loss = 0.f;
            if (w != 0.f) {
                if (soft_on) loss = (1.f - p.hard) * p.T * p.T * (ts.y / ts.x * inv_T + (logf(s) - logf(ts.x)));
                if (hard_on) loss += p.hard * (logf(s1) - (szy - M));
            }
            if (p.row_loss) p.row_loss[r] = loss;
            acc += (double)w * (double)loss;
        }
        if (g) {
            const float a = soft_on ? w * (1.f - p.hard) * p.T : 0.f, b = hard_on ? w * p.hard : 0.f;
            const float aq = soft_on ? a / s : 0.f, ap = soft_on ? a / ts.x : 0.f, bq = hard_on ? b / s1 : 0.f;
            T *gr = g + r * p.ld_g;
            auto grad = [&](float zv) {
                const float x = zv - M;
                float o = soft_on ? aq * ex2_fast(x * cT) : 0.f;
                if (HARD && hard_on) o += bq * ex2_fast(x * LOG2E);
                return w == 0.f ? 0.f : o;
            };
            for (int32_t col = tid * V; col < p.C; col += NT * V) {
                float v[V];
                row_load(zr, col, p.C, v);
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] = grad(v[i]);
                row_store(gr, col, p.C, v);
            }
            __syncthreads();
            // the columns of the teacher's entries and of the label once more; several of one class come to the same number
            if (mine >= 0 && w != 0.f) {
                float e = 0.f;
                for (int j = 0; j < p.k; ++j)
                    if (sid[j] == mine) e += se[j];
                float x = grad(zc);
                if (soft_on) x -= ap * e;
                if (hard_on && mine == y) x -= b;
                gr[mine] = RowVec<T>::to(x);
            }
        }
        __syncthreads();   // (sid, se, smax are the next row's)
    }
    if (p.loss_sum) loss_finish<NT>(acc, p.block_partial, p.ticket, p.loss_sum, 0);
}

template <typename T, bool HARD>
static void distill_launch(sat_ctx *ctx, const Distill &p, const void *z, void *g)
{
    constexpr int V = RowVec<T>::V;
    const int32_t pieces = (p.C + V - 1) / V;
    if (pieces > 32 * (32 / V)) {
        const unsigned blocks = (unsigned)std::min<int64_t>(p.rows, (int64_t)ctx->sms * 4);
        sat_pdl(ctx->stream, k_distill_wide<T, HARD>, blocks, DISTILL_NT, 0)(p, (const T *)z, (T *)g);
        return;
    }
    auto go = [&](auto kernel, int tpr, int ch) {
        const unsigned blocks = (unsigned)std::min<int64_t>(cdiv64(p.rows, 256 / tpr), LOSS_MAX_BLOCKS(ctx));
        sat_pdl(ctx->stream, kernel, blocks, 256, (size_t)256 * ch * 16 * V / 4)(p, (const T *)z, (T *)g);
    };
    if (pieces <= 8) go(k_distill_rows<T, 8, 1, HARD>, 8, 1);
    else if (pieces <= 16) go(k_distill_rows<T, 16, 1, HARD>, 16, 1);
    else if (pieces <= 32) go(k_distill_rows<T, 32, 1, HARD>, 32, 1);
    else if (pieces <= 64) go(k_distill_rows<T, 32, 2, HARD>, 32, 2);
    else if (pieces <= 128) go(k_distill_rows<T, 32, 4, HARD>, 32, 4);
    else go(k_distill_rows<T, 32, 32 / V, HARD>, 32, 32 / V);
}

extern "C" sat_status sat_distill_grad(sat_ctx *ctx, int64_t rows, int32_t n_classes, int type, const void *z, int32_t ld_z, int32_t k, const int32_t *top_ids,
                                       const float *top_logits, float temperature, float hard, const int32_t *labels, const float *row_weight, float weight,
                                       double *loss_sum, float *row_loss, void *g, int32_t ld_g)
{
    CHECK_CTX(ctx);
    if (!ok_type(type)) return sat_fail(ctx, SAT_EINVAL, "sat_distill_grad: unknown element type");
    if (rows < 0 || rows >= INT32_MAX || n_classes <= 0 || n_classes >= INT32_MAX - 8192) return sat_fail(ctx, SAT_EINVAL, "sat_distill_grad: bad number of rows or classes");
    if (k < 0 || k > DISTILL_MAX_K) return sat_fail(ctx, SAT_EINVAL, "sat_distill_grad: k must be in [0, %d]", DISTILL_MAX_K);
    if (!(temperature >= 1e-3f && temperature <= 1e3f) || !(hard >= 0.f && hard <= 1.f)) return sat_fail(ctx, SAT_EINVAL, "sat_distill_grad: temperature must be in [0.001, 1000], hard in [0, 1]");
    if (!ok_ld_of(type, ld_z, n_classes) || (g && !ok_ld_of(type, ld_g, n_classes)) || (g && !aligned16(g)) ||
        (rows > 0 && (!z || !aligned16(z) || (k > 0 && (!top_ids || !top_logits)) || (hard > 0.f && !labels))))
        return sat_fail(ctx, SAT_EINVAL, "sat_distill_grad: null / misaligned tensor or bad leading dimension");
    if (!g && !loss_sum && !row_loss) return sat_fail(ctx, SAT_EINVAL, "sat_distill_grad: no result is asked for");
    if (rows == 0) return SAT_OK;
    SAT_TRY(sat_ensure(ctx, ctx->buf_distill, (size_t)LOSS_MAX_BLOCKS(ctx) * sizeof(double)));
    Distill p = {rows, n_classes, k, ld_z, ld_g, top_ids, top_logits, temperature, hard, labels, row_weight, weight, row_loss, (double *)ctx->buf_distill.p,
                 ctx->d_flag + 2, loss_sum, ctx->d_flag + 1};
    ProfScope prof(ctx, SATK_LOSS, (g ? 2.0 : 1.0) * type_bytes(type) * (double)rows * n_classes, 0.0);
    if (hard > 0.f) {
        if (type == SAT_F32) distill_launch<float, true>(ctx, p, z, g);
        else if (type == SAT_BF16) distill_launch<__nv_bfloat16, true>(ctx, p, z, g);
        else distill_launch<__half, true>(ctx, p, z, g);
    } else {
        if (type == SAT_F32) distill_launch<float, false>(ctx, p, z, g);
        else if (type == SAT_BF16) distill_launch<__nv_bfloat16, false>(ctx, p, z, g);
        else distill_launch<__half, false>(ctx, p, z, g);
    }
    SAT_LAUNCHED(ctx);
    return SAT_OK;
}

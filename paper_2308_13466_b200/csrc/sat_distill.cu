// Distillation from a teacher's top logits, the loss and its gradient in one pass:
//     p = softmax(t / T) over the k entries (id, t) of a row,   q = softmax(z / T),   q1 = softmax(z)
//     loss = (1 - h) T^2 sum_j p_j (log p_j - log q_{id_j}) + h (-log q1_y)
//     g_c = w [ (1 - h) T (q_c - sum_{j: id_j = c} p_j) + h (q1_c - [c = y]) ]
#include "sat_loss.h"
#include "sat_ptx.h"
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

// A student that all but agrees with its teacher, at a high temperature.  KL = sum p d + log(s / st), d_j = (t_j - max t) / T - (z_j - max z) / T, is then a difference of numbers that are
// larger by far, and T^2 brings what their rounding left back to size.  With u = d - sum p d the same is
//     KL = log(1 + sum p (e^-u - 1 + u) + e^(sum p d) rest / st),     rest: the exponentials of the classes that the teacher does not name,
// where nothing is negative and nothing cancels; e^-u - 1 + u has its series where u is small, and `rest` is added up by itself.  (A class that is named twice would be
// in the sum twice: such rows keep what they have.)  Worked out behind the gradient, where little else is in registers, and called (612257 x 47 with labels, four lanes a row and two entries a
// lane: 76 us, inlined 82, ahead of the gradient 81, called there 96, not at all 70.5).  With the fewer shapes that there are of it 84 us, and 244 for 111 of 1000000 x 16 whose rows all take it; so temperatures of up
// to DISTILL_NEAR_FROM do without: the other form's error, about 2^-21 in KL, is 2^-17 in the loss there.
// sp has z - max z on entry and is left all zeros, as it is between rows.  `near` is the same for the lanes of a row; all lanes of the warp call.
#define DISTILL_NEAR_FROM 4.f
#define DISTILL_NEAR 0.125f   // of KL; beside more than that 2^-21 is small
template <int TPR>
__device__ __noinline__ float distill_near(const int32_t *ids, const float *logits, int32_t C, int32_t k, float cT, float inv_T, float *sp, int32_t stride, bool near, float kl)
{
    constexpr float TAKEN = -1e30f;   // what a class that the teacher names has in sp afterwards, times the lane's number; as far down logits add nothing to `rest`
    const int t = threadIdx.x % TPR;
    auto entry = [&](int32_t e, int32_t &id) {   // its logit; -inf: none
        id = near && e < k ? __ldg(ids + e) : -1;
        return (uint32_t)id < (uint32_t)C ? __ldg(logits + e) : -INFINITY;
    };
    float tm = -INFINITY, st = 0.f, mean = 0.f, sum = 0.f, rest = 0.f;
    int32_t id;
    for (int32_t e0 = 0; e0 < k; e0 += TPR) tm = fmaxf(tm, entry(e0 + t, id));
#pragma unroll
    for (int o = TPR / 2; o > 0; o >>= 1) tm = fmaxf(tm, __shfl_xor_sync(0xffffffffu, tm, o));
    for (int32_t e0 = 0; e0 < k; e0 += TPR) {
        const float gap = entry(e0 + t, id) - tm, w = ex2_fast(gap * cT);
        if (w > 0.f) st += w, mean = fmaf(w, gap - sp[id], mean);
    }
#pragma unroll
    for (int o = TPR / 2; o > 0; o >>= 1) {
        st += __shfl_xor_sync(0xffffffffu, st, o);
        mean += __shfl_xor_sync(0xffffffffu, mean, o);
    }
    mean /= st;
    int twice = 0;
    for (int32_t e0 = 0; e0 < k; e0 += TPR) {
        const float gap = entry(e0 + t, id) - tm, w = ex2_fast(gap * cT), x = w > 0.f ? sp[id] : 0.f;
        __syncwarp();
        if (w > 0.f) sp[id] = TAKEN * (float)(t + 1);
        __syncwarp();
        if (!(w > 0.f)) continue;
        if (x <= TAKEN || sp[id] != TAKEN * (float)(t + 1)) twice = 1;
        const float u = (gap - x - mean) * inv_T;
        if (fabsf(u) < 0.5f) {   // (the next term is 2^-24 of the first at most)
            const float f = fmaf(u, fmaf(u, fmaf(u, fmaf(u, fmaf(u, fmaf(u, 1.f / 40320.f, -1.f / 5040.f), 1.f / 720.f), -1.f / 120.f), 1.f / 24.f), -1.f / 6.f), 0.5f);
            sum = fmaf(w, u * u * f, sum);
        } else {   // (in two factors: a small weight may stand beside a large exponential)
            const float half = expf(-0.5f * u);
            sum += w * half * half + w * (u - 1.f);
        }
    }
    __syncwarp();
    for (int32_t c = t; near && c < C; c += TPR)
        if (sp[c] > TAKEN) rest += ex2_fast(sp[c] * cT);
    __syncwarp();
    for (int32_t c = t; c < stride; c += TPR) sp[c] = 0.f;
    __syncwarp();
#pragma unroll
    for (int o = TPR / 2; o > 0; o >>= 1) {
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
        rest += __shfl_xor_sync(0xffffffffu, rest, o);
        twice |= __shfl_xor_sync(0xffffffffu, twice, o);
    }
    return near && !twice ? log1pf((sum + expf(mean * inv_T) * rest) / st) : kl;
}

// Up to 1,024 classes: TPR lanes hold a row in registers, CH times 16 bytes each, and up to NE of the teacher's entries each.  The teacher's probabilities and
// the label meet their columns in shared memory (`sp`), which is all zeros between rows.  Few lanes a row, since what a row costs whatever its width (two sums
// and maxima across its lanes, logarithms, quotients) is paid once a warp for its 32 / TPR rows.  Bound by instruction issue: 612257 x 47 fp32 with labels 71 us (16 lanes a row and
// __match_any for repeated classes: 295).
template <int TPR, int CH, int V>
__host__ __device__ constexpr int distill_stride()   // floats of a row's `sp`: rows of a warp that are read together lie in other banks
{
    return TPR * CH * V + ((TPR * CH * V) % 32 == 0 && TPR < 8 ? 4 * TPR : 0);
}
template <typename T, int TPR, int CH, int NE, bool HARD, bool NEAR>
__global__ void __launch_bounds__(256, CH * RowVec<T>::V > 16 ? 2 : NE > 4 ? 3 : 4)
k_distill_rows(Distill p, const T *z, T *g)
{
    sat_grid_wait();
    constexpr int V = RowVec<T>::V, H = V / 2, RPW = 32 / TPR, STRIDE = distill_stride<TPR, CH, V>();
    extern __shared__ float4 distill_smem[];
    __shared__ float2 kept[NEAR ? 256 / TPR : 1];   // KL and the label's term of a row that distill_near takes
    const int lane = threadIdx.x & 31, t = lane % TPR;
    const unsigned mates = TPR == 32 ? 0xffffffffu : ((1u << (TPR & 31)) - 1u) << (lane - t);
    float *sp = reinterpret_cast<float *>(distill_smem) + (threadIdx.x / TPR) * STRIDE;
    for (int i = t; i < STRIDE; i += TPR) sp[i] = 0.f;
    __syncwarp();
    const float cT = LOG2E / p.T, inv_T = 1.f / p.T, soft = 1.f - p.hard;
    const uint64_t cT_2 = f2_pack(cT, cT), c1_2 = f2_pack(LOG2E, LOG2E);
    double acc = 0.0;
    for (int64_t rw = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 5; rw * RPW < p.rows; rw += (int64_t)gridDim.x * 8) {
        const int64_t r = rw * RPW + lane / TPR;
        const bool ok = r < p.rows;
        const int64_t row = ok ? r : p.rows - 1;
        const T *zr = z + row * p.ld_z;
        uint4 raw[CH];
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            raw[j] = make_uint4(0u, 0u, 0u, 0u);
            if (j * TPR * V < p.C) raw[j] = row_load_raw(zr, (j * TPR + t) * V, p.C);
        }
        // entries that are none: id -1, logit -inf
        const int32_t *ids = p.ids + row * p.k + t;
        const float *logits = p.logits + row * p.k + t;
        int32_t id[NE];
        float te[NE], ze[NE];
        bool outside = false;
#pragma unroll
        for (int e = 0; e < NE; ++e) {
            id[e] = -1;
            te[e] = -INFINITY;
            if (e * TPR + t < p.k) id[e] = __ldg(ids + e * TPR), te[e] = __ldg(logits + e * TPR);
        }
        const float w = p.weight * (p.row_weight ? __ldg(p.row_weight + row) : 1.f);
        int32_t y = HARD ? __ldg(p.labels + row) : -1;
        if (HARD && y >= p.C) y = -1, outside = true;
        const float zy = y >= 0 ? RowVec<T>::from(zr[y]) : 0.f;   // (this and ze before g is written, which may be z)
        unsigned any = 0;
#pragma unroll
        for (int e = 0; e < NE; ++e) {
            if (e * TPR >= p.k) break;
            outside |= id[e] >= p.C;
            if ((uint32_t)id[e] >= (uint32_t)p.C || te[e] == -INFINITY) id[e] = -1, te[e] = -INFINITY;
            any |= __ballot_sync(0xffffffffu, id[e] >= 0);
        }
        const bool some = (any & mates) != 0;
        if (outside) atomicOr(p.status, 8);
        uint64_t x[CH][H];   // z - max, by twos
        float m = -INFINITY, tm = -INFINITY;
#pragma unroll
        for (int e = 0; e < NE; ++e) {
            ze[e] = id[e] >= 0 ? RowVec<T>::from(zr[id[e]]) : 0.f;
            tm = fmaxf(tm, te[e]);
        }
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int32_t col = (j * TPR + t) * V;
            float v[V];
            RowVec<T>::unpack(raw[j], v);
            if (col + V > p.C) {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (col + i >= p.C) v[i] = -INFINITY;
            }
#pragma unroll
            for (int i = 0; i < V; ++i) m = fmaxf(m, v[i]);
#pragma unroll
            for (int i = 0; i < H; ++i) x[j][i] = f2_pack(v[2 * i], v[2 * i + 1]);
        }
#pragma unroll
        for (int o = TPR / 2; o > 0; o >>= 1) {
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            tm = fmaxf(tm, __shfl_xor_sync(0xffffffffu, tm, o));
        }
        float st = 0.f, num = 0.f;
        uint64_t s_2 = 0, s1_2 = 0;
        const uint64_t less_m = f2_pack(-m, -m);
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            if (j * TPR * V >= p.C) break;
#pragma unroll
            for (int i = 0; i < H; ++i) {
                x[j][i] = f2_add(x[j][i], less_m);
                s_2 = f2_add(s_2, f2_ex2(f2_mul(x[j][i], cT_2)));
                if (HARD) s1_2 = f2_add(s1_2, f2_ex2(f2_mul(x[j][i], c1_2)));
            }
        }
        float s = f2_unpack(s_2).x + f2_unpack(s_2).y, s1 = f2_unpack(s1_2).x + f2_unpack(s1_2).y;
#pragma unroll
        for (int e = 0; e < NE; ++e) {
            if (id[e] < 0) {
                te[e] = 0.f;
                continue;
            }
            const float gap = te[e] - tm;
            te[e] = ex2_fast(gap * cT);
            st += te[e];
            if (!(te[e] <= 0.f)) num = fmaf(te[e], gap - (ze[e] - m), num);
        }
#pragma unroll
        for (int o = TPR / 2; o > 0; o >>= 1) {
            s += __shfl_xor_sync(0xffffffffu, s, o);
            st += __shfl_xor_sync(0xffffffffu, st, o);
            num += __shfl_xor_sync(0xffffffffu, num, o);
            if (HARD) s1 += __shfl_xor_sync(0xffffffffu, s1, o);
        }
        const bool soft_on = some && soft > 0.f, hard_on = HARD && y >= 0, dead = w == 0.f || !(soft_on || hard_on);
        bool near = false, nears = false;   // nears: one of the warp's rows
        auto put = [&](float kl, float label) {
            const float loss = (1.f - p.hard) * p.T * p.T * kl + label;
            if (p.row_loss) p.row_loss[r] = loss;
            if (p.loss_sum) acc += (double)(p.weight * (p.row_weight ? __ldg(p.row_weight + r) : 1.f)) * (double)loss;
        };
        if ((p.row_loss || p.loss_sum) && (NEAR || (ok && t == 0))) {
            const float kl = soft_on && !dead ? num * rcp_fast(st) * inv_T + logf(s * rcp_fast(st)) : 0.f, label = hard_on && !dead ? p.hard * (logf(s1) - (zy - m)) : 0.f;
            if (NEAR) {
                near = ok && soft_on && !dead && kl < DISTILL_NEAR;
                nears = __any_sync(0xffffffffu, near);
                if (t == 0 && near) kept[threadIdx.x / TPR] = make_float2(kl, label);
            }
            if (t == 0 && ok && !near) put(kl, label);
        }
        if (!g) {   // (the same for all threads)
            if (!NEAR || !nears) continue;
#pragma unroll
            for (int j = 0; j < CH; ++j)
#pragma unroll
                for (int i = 0; i < H; ++i)
                    if ((j * TPR + t) * V < p.C) *reinterpret_cast<float2 *>(sp + (j * TPR + t) * V + 2 * i) = f2_unpack(x[j][i]);
        } else {
            const float a = soft_on ? w * soft * p.T : 0.f, b = hard_on ? w * p.hard : 0.f;
            const float aq = a * rcp_fast(s), ap = soft_on ? a * rcp_fast(st) : 0.f, bq = HARD ? b * rcp_fast(s1) : 0.f;
            const uint64_t aq_2 = f2_pack(aq, aq), bq_2 = f2_pack(bq, bq);
            // a class that is named more than once: whose tag is found says that others are there, and then one adds after the other
#pragma unroll
            for (int e = 0; e < NE; ++e) {
                if (e * TPR >= p.k) break;
                const bool mine = id[e] >= 0 && soft_on;
                const float val = ap * te[e], old = mine ? sp[id[e]] : 0.f;
                __syncwarp();
                if (mine) sp[id[e]] = __int_as_float(t);
                __syncwarp();
                const bool twice = __any_sync(0xffffffffu, mine && __float_as_int(sp[mine ? id[e] : 0]) != t);
                __syncwarp();
                if (mine) sp[id[e]] = twice ? old : old + val;
                __syncwarp();
                if (twice)
                    for (int i = 0; i < TPR; ++i) {
                        if (mine && t == i) sp[id[e]] += val;
                        __syncwarp();
                    }
            }
            if (HARD) {
                if (hard_on && t == 0) sp[y] += b;
                __syncwarp();
            }
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const int32_t col = (j * TPR + t) * V;
                if (col >= p.C) break;
                float o[V];
#pragma unroll
                for (int i = 0; i < V; i += 4) {
                    float4 *at = reinterpret_cast<float4 *>(sp + col + i);
                    const float4 q = *at;
                    const float2 x0 = f2_unpack(x[j][i / 2]), x1 = f2_unpack(x[j][i / 2 + 1]);
                    *at = NEAR && nears ? make_float4(x0.x, x0.y, x1.x, x1.y) : make_float4(0.f, 0.f, 0.f, 0.f);
                    uint64_t out[2] = {f2_pack(-q.x, -q.y), f2_pack(-q.z, -q.w)};
#pragma unroll
                    for (int h = 0; h < 2; ++h) {   // (exponentials once more: kept, they would take the registers of half of the warps)
                        const uint64_t xx = x[j][i / 2 + h];
                        if (HARD) out[h] = f2_fma(bq_2, f2_ex2(f2_mul(xx, c1_2)), out[h]);
                        out[h] = f2_fma(aq_2, f2_ex2(f2_mul(xx, cT_2)), out[h]);
                        const float2 f = f2_unpack(out[h]);
                        o[i + 2 * h] = dead ? 0.f : f.x, o[i + 2 * h + 1] = dead ? 0.f : f.y;
                    }
                }
                if (ok) row_store(g + r * p.ld_g, col, p.C, o);
            }
        }
        if (NEAR && nears) {
            __syncwarp();
            const float2 had = kept[threadIdx.x / TPR];
            const float kl = distill_near<TPR>(p.ids + r * p.k, p.logits + r * p.k, p.C, p.k, cT, 1.f / p.T, sp, STRIDE, near, had.x);
            if (t == 0 && near) put(kl, had.y);
        }
        __syncwarp();
    }
    if (p.loss_sum) loss_finish(acc, p.block_partial, p.ticket, p.loss_sum, 0);
}

// More classes: a block per row.  Every thread takes the maximum of what it has and sums relative to that, which are joined across the block, so that a row costs
// one barrier before its gradient is written and one behind.  What then differs at the teacher's entries and the label is written over it, a thread each.
struct DistillSum {
    float m, s, s1;   // largest logit, sums relative to it
};
__device__ __forceinline__ float warp_max(float x)
{
    float m;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(x));
    return m;
}
// over the lanes of a warp, the same in all of them (sums relative to -inf are zero)
template <bool HARD>
__device__ __forceinline__ DistillSum distill_join_lanes(DistillSum v, float cT)
{
    const float m = warp_max(v.m), from = m == -INFINITY ? 0.f : m;
    v.s *= ex2_fast((v.m - from) * cT);
    if (HARD) v.s1 *= ex2_fast((v.m - from) * LOG2E);
    v.m = m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        v.s += __shfl_xor_sync(0xffffffffu, v.s, o);
        if (HARD) v.s1 += __shfl_xor_sync(0xffffffffu, v.s1, o);
    }
    return v;
}
// Exponents of 2^((z - m) c): z c - o in one operation, o being m c rounded.  What that rounding leaves is the same for all z: a sum and a quotient are
// multiplied by 2^left.  That keeps the numbers' accuracy while m c is small: below 2^21 half a step of o is 2^-4 at most, far beyond `left` is as large as any
// exponent, and 2^left no number or none.  So a thread's reference does not lie below -2 DISTILL_FITS T: what it has so deep down (logits of -inf, finite masks, or no columns at
// all) adds up to zero, as it should beside a row's largest logit that is not.  A row whose largest logit lies beyond DISTILL_FITS T to either side takes the difference first (`exact`).
#define DISTILL_FITS 7e5f   // times log2(e): just below 2^20
struct DistillScale {
    float c, o, left;
    __device__ __forceinline__ DistillScale(float m, float c_, bool exact = false) : c(c_)
    {
        o = exact ? m : m * c_;
        left = exact ? 0.f : fmaf(m, -c_, o);
    }
};
// a thread's, at temperature T (1 for the label's term)
__device__ __forceinline__ DistillScale distill_scale(float m, float T, float c) { return DistillScale(fmaxf(m, -2.f * DISTILL_FITS * T), c); }
// 16 bytes of logits: their exponentials, by twos
template <typename T, bool EXACT>
__device__ __forceinline__ void distill_exp(const uint4 &raw, const DistillScale &sc, uint64_t (&e)[RowVec<T>::V / 2])
{
    constexpr int V = RowVec<T>::V;
    float v[V];
    RowVec<T>::unpack(raw, v);
    const uint64_t c = f2_pack(sc.c, sc.c), o = f2_pack(-sc.o, -sc.o);
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        const uint64_t x = f2_pack(v[2 * i], v[2 * i + 1]);
        e[i] = f2_ex2(EXACT ? f2_mul(f2_add(x, o), c) : f2_fma(x, c, o));
    }
}
// adds up the exponentials of 16 bytes of logits
template <typename T, bool HARD, bool EXACT>
__device__ __forceinline__ void distill_add(const uint4 &raw, const DistillScale &cs, const DistillScale &hs, uint64_t &s, uint64_t &s1)
{
    constexpr int H = RowVec<T>::V / 2;
    uint64_t e[H];
    distill_exp<T, EXACT>(raw, cs, e);
#pragma unroll
    for (int i = 0; i < H; ++i) s = f2_add(s, e[i]);
    if (!HARD) return;
    distill_exp<T, EXACT>(raw, hs, e);
#pragma unroll
    for (int i = 0; i < H; ++i) s1 = f2_add(s1, e[i]);
}

// What a row takes beside its logits, a thread per entry of the teacher's
struct DistillEntry {
    int32_t id, y;   // -1: none
    float t, w;
};
template <bool HARD>
__device__ __forceinline__ DistillEntry distill_entry(const Distill &p, int64_t r, int tid)
{
    DistillEntry e = {-1, -1, -INFINITY, 0.f};
    if (r >= p.rows) return e;
    e.w = p.weight * (p.row_weight ? __ldg(p.row_weight + r) : 1.f);
    if (HARD) e.y = __ldg(p.labels + r);
    if (tid < p.k) e.id = __ldg(p.ids + r * p.k + tid), e.t = __ldg(p.logits + r * p.k + tid);
    return e;
}
__device__ __forceinline__ void distill_known(const Distill &p, DistillEntry &e)
{
    if (e.id >= p.C || e.y >= p.C) atomicOr(p.status, 8);
    if (e.y >= p.C) e.y = -1;
    if ((uint32_t)e.id >= (uint32_t)p.C || e.t == -INFINITY) e.id = -1, e.t = -INFINITY;
}

// The part of a block of NT threads that does not depend on where its logits are.  By turns, so that a row's writes do not meet the reads of the row before it.
template <int NT>
struct DistillShared {
    static constexpr int K = NT < DISTILL_MAX_K ? NT : DISTILL_MAX_K, KW = K / 32, W = NT / 32;   // entries: a thread each
    int32_t id[K];
    float e[K], top[KW];
    unsigned any[KW];
    float2 part[KW];
    DistillSum sum[W];
    uint32_t table[256];   // a bit of each entry's class
    int twice;             // two entries had the same bit: they may be of one class
    __device__ __forceinline__ void clear()
    {
        for (int i = threadIdx.x; i < 256; i += NT) table[i] = 0;
        if (threadIdx.x == 0) twice = 0;
    }
};
#define DISTILL_TELLS(NT) ((NT) - 32)   // the thread that works out a row's loss: of the last warp, which has no entries unless there are many (the first: 1.3 % of 8192 x 50001 bf16)
template <int NT>
__device__ __forceinline__ void distill_sync() { asm volatile("bar.sync 1, %0;" ::"n"(NT) : "memory"); }

template <typename T, int NT, bool HARD>
struct DistillRow {
    DistillEntry en;
    float zc, zy;              // logits at the entry and the label, read before g is written, which may be z
    DistillSum sum;
    bool soft_on, hard_on, dead, exact, y_among = false;   // y_among: (first thread) an entry may be of the label's class
    float a, b, aq, bq;

    // from the sums of the threads (before the block's first barrier) to the factors of the gradient
    __device__ __forceinline__ void join(const Distill &p, DistillShared<NT> &sh, DistillShared<NT> &other, const T *zr, DistillSum mine, float cT)
    {
        constexpr int KW = DistillShared<NT>::KW, W = DistillShared<NT>::W;
        const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
        sum = distill_join_lanes<HARD>(mine, cT);
        if (lane == 0) sh.sum[warp] = sum;
        if (warp < KW) {
            const float top = warp_max(en.t);
            const unsigned any = __ballot_sync(0xffffffffu, en.id >= 0);
            if (lane == 0) sh.top[warp] = top, sh.any[warp] = any;
            if (tid < p.k) sh.id[tid] = en.id;
            if (en.id >= 0) {
                const uint32_t bit = 1u << (en.id & 31);
                if (atomicOr(sh.table + ((en.id >> 5) & 255), bit) & bit) sh.twice = 1;
            }
        }
        distill_sync<NT>();
        if (tid == 0) {
            other.twice = 0;   // (the row before this one is done with it)
            y_among = HARD && en.y >= 0 && ((sh.table[(en.y >> 5) & 255] >> (en.y & 31)) & 1u);
        }
        sum = distill_join_lanes<HARD>(lane < W ? sh.sum[lane] : DistillSum{-INFINITY, 0.f, 0.f}, cT);
        exact = !(fabsf(sum.m) <= DISTILL_FITS * (HARD ? fminf(p.T, 1.f) : p.T));
        if (exact) {   // (the same for the whole block) the sums once more
            const DistillScale cs(sum.m, cT, true), hs(sum.m, LOG2E, true);
            uint64_t s = 0, s1 = 0;
            for (int64_t col = (int64_t)tid * RowVec<T>::V; col < p.C; col += NT * RowVec<T>::V) {
                uint4 raw = row_load_raw(zr, (int32_t)col, p.C);
                if (col + RowVec<T>::V > p.C) raw = RowVec<T>::cut(raw, (int32_t)(p.C - col));
                distill_add<T, HARD, true>(raw, cs, hs, s, s1);
            }
            mine = {sum.m, f2_unpack(s).x + f2_unpack(s).y, f2_unpack(s1).x + f2_unpack(s1).y};
            mine = distill_join_lanes<HARD>(mine, cT);
            distill_sync<NT>();
            if (lane == 0) sh.sum[warp] = mine;
            distill_sync<NT>();
            sum = distill_join_lanes<HARD>(lane < W ? sh.sum[lane] : DistillSum{-INFINITY, 0.f, 0.f}, cT);
        }
        const bool some = __any_sync(0xffffffffu, sh.any[lane % KW] != 0);
        const float soft = 1.f - p.hard;
        soft_on = some && soft > 0.f, hard_on = HARD && en.y >= 0, dead = en.w == 0.f || !(soft_on || hard_on);
        a = soft_on ? en.w * soft * p.T : 0.f, b = hard_on ? en.w * p.hard : 0.f;
        aq = a * rcp_fast(sum.s), bq = HARD ? b * rcp_fast(sum.s1) : 0.f;
        if (warp < KW) {
            const float tm = warp_max(sh.top[lane % KW]);
            float2 s = make_float2(0.f, 0.f);   // weight of this thread's entry, and its part of the loss
            if (en.id >= 0) {
                const float gap = en.t - tm;
                s.x = ex2_fast(gap * cT);
                if (!(s.x <= 0.f)) s.y = s.x * (gap - (zc - sum.m));
            }
            if (tid < p.k) sh.e[tid] = s.x;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                s.x += __shfl_xor_sync(0xffffffffu, s.x, o);
                s.y += __shfl_xor_sync(0xffffffffu, s.y, o);
            }
            if (lane == 0) sh.part[warp] = s;
        }
    }
    // 16 bytes of the gradient without the teacher's part and the label's
    template <bool EXACT>
    __device__ __forceinline__ void grad(const uint4 &raw, const DistillScale &cs, const DistillScale &hs, float af, float bf, float (&o)[RowVec<T>::V]) const
    {
        constexpr int H = RowVec<T>::V / 2;
        uint64_t e[H], e1[H];
        distill_exp<T, EXACT>(raw, cs, e);
        if (HARD) distill_exp<T, EXACT>(raw, hs, e1);
#pragma unroll
        for (int i = 0; i < H; ++i) {
            uint64_t x = f2_mul(f2_pack(af, af), e[i]);
            if (HARD) x = f2_fma(f2_pack(bf, bf), e1[i], x);
            o[2 * i] = f2_unpack(x).x, o[2 * i + 1] = f2_unpack(x).y;
        }
    }
    // all of it for the rows that take another way: no gradient at all, or differences first
    __device__ __forceinline__ void other_rows(const Distill &p, const T *zr, T *gr, float cT) const
    {
        constexpr int V = RowVec<T>::V;
        const DistillScale cs(sum.m, cT, true), hs(sum.m, LOG2E, true);
        for (int64_t col = (int64_t)threadIdx.x * V; col < p.C; col += NT * V) {
            float o[V] = {};
            if (!dead) grad<true>(row_load_raw(zr, (int32_t)col, p.C), cs, hs, aq, bq, o);
            row_store(gr, (int32_t)col, p.C, o);
        }
    }
    // behind the block's second barrier: the columns of the entries and the label, and the loss
    __device__ __forceinline__ void finish(const Distill &p, DistillShared<NT> &sh, int64_t r, float cT, T *gr, double &acc) const
    {
        const int tid = threadIdx.x;
        const bool tells = tid == DISTILL_TELLS(NT);
        if (!tells && (tid >= DistillShared<NT>::K || (tid != 0 && en.id < 0))) return;
        if (en.id >= 0) sh.table[(en.id >> 5) & 255] = 0;
        float2 ts = make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < DistillShared<NT>::KW; ++i) ts.x += sh.part[i].x, ts.y += sh.part[i].y;
        const float ap = soft_on ? a * rcp_fast(ts.x) : 0.f;
        // several entries of one class, and the label's, come to the same number
        auto column = [&](int32_t c, float e, bool search, float zv) {
            if (!gr || dead) return;
            if (search) {
                e = 0.f;
                for (int j = 0; j < p.k; ++j)
                    if (sh.id[j] == c) e += sh.e[j];
            }
            const float x = zv - sum.m;
            float o = aq * ex2_fast(x * cT) - ap * e;
            if (HARD) o += bq * ex2_fast(x * LOG2E) - (c == en.y ? b : 0.f);
            gr[c] = RowVec<T>::to(o);
        };
        if (en.id >= 0) column(en.id, sh.e[tid], sh.twice != 0, zc);
        if (HARD && tid == 0 && en.y >= 0) column(en.y, 0.f, y_among, zy);
        if (!tells) return;
        float loss = 0.f;
        if (!dead) {
            if (soft_on) loss = (1.f - p.hard) * p.T * p.T * (ts.y * rcp_fast(ts.x) / p.T + (logf(sum.s) - logf(ts.x)));
            if (hard_on) loss += p.hard * (logf(sum.s1) - (zy - sum.m));
        }
        if (p.row_loss) p.row_loss[r] = loss;
        if (p.loss_sum) acc += (double)en.w * (double)loss;
    }
};

// Rows of up to CH pieces of 16 bytes a thread: they stay in registers as they lie in memory.  Where few blocks share an SM (STAGED) the next row comes into
// shared memory meanwhile (cp.async.bulk).  The sums, their join and the gradient take turns: 8192 x 50001 bf16 374 us (4.4 TB/s; not staged 389), of which the exponentials are
// 182; 16384 x 4000 bf16 62 us (4.3 TB/s), 32768 x 2000 fp32 100 (5.3).
template <typename T, int NT, int CH, bool HARD, bool STAGED>
__global__ void __launch_bounds__(NT, 1024 / NT)
k_distill_wide(Distill p, const T *z, T *g)
{
    constexpr int V = RowVec<T>::V;
    extern __shared__ uint4 stage[];   // [CH NT]
    __shared__ DistillShared<NT> sh[2];
    __shared__ uint64_t full;
    __shared__ int dead;
    const int tid = threadIdx.x;
    sh[0].clear();
    sh[1].clear();
    if (STAGED && tid == 0) {
        mbar_init(&full, 1);
        dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    distill_sync<NT>();
    sat_grid_wait();
    const uint32_t bytes = (uint32_t)((p.C + V - 1) / V) * 16;
    uint32_t issued = 0;
    const float cT = LOG2E / p.T;
    double acc = 0.0;
    int turn = 0;
    uint4 raw[CH];
    DistillEntry next;
    auto load = [&](int64_t r) {
        if (STAGED) {
            if (tid == 0 && r < p.rows && !*(volatile int *)&dead) {
                ++issued;
                mbar_expect_tx(&full, bytes);
                asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(stage)), "l"(z + r * p.ld_z),
                             "r"(bytes), "r"(smem_u32(&full))
                             : "memory");
            }
            return;
        }
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int32_t col = (j * NT + tid) * V;
            raw[j] = r < p.rows && col < p.C ? row_load_raw(z + r * p.ld_z, col, p.C) : RowVec<T>::lowest();
        }
    };
    load(blockIdx.x);
    next = distill_entry<HARD>(p, blockIdx.x, tid);
    uint32_t phase = 0;
    for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x, turn ^= 1) {
        const T *zr = z + r * p.ld_z;
        DistillRow<T, NT, HARD> row;
        row.en = next;
        distill_known(p, row.en);
        row.zc = row.en.id >= 0 ? RowVec<T>::from(zr[row.en.id]) : 0.f;
        row.zy = row.en.y >= 0 ? RowVec<T>::from(zr[row.en.y]) : 0.f;
        if (STAGED) {
            (void)mbar_wait(&full, phase, &dead, p.status);   // (having given up, all finish on what is there)
            phase ^= 1u;
#pragma unroll
            for (int j = 0; j < CH; ++j) raw[j] = (j * NT + tid) * V < p.C ? stage[j * NT + tid] : RowVec<T>::lowest();
            fence_async_smem();   // these loads are done before the next row lands
            distill_sync<NT>();
            load(r + gridDim.x);
        }
        DistillSum sum = {-INFINITY, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int32_t col = (j * NT + tid) * V;
            if ((j * NT + (tid & ~31)) * V >= p.C) break;   // (nothing for the whole warp)
            if (col < p.C && col + V > p.C) raw[j] = RowVec<T>::cut(raw[j], p.C - col);
            sum.m = fmaxf(sum.m, RowVec<T>::largest(raw[j]));
        }
        {
            const DistillScale cs = distill_scale(sum.m, p.T, cT), hs = distill_scale(sum.m, 1.f, LOG2E);
            uint64_t s_2 = 0, s1_2 = 0;
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                if ((j * NT + (tid & ~31)) * V >= p.C) break;
                distill_add<T, HARD, false>(raw[j], cs, hs, s_2, s1_2);
            }
            sum.s = (f2_unpack(s_2).x + f2_unpack(s_2).y) * ex2_fast(cs.left);
            sum.s1 = HARD ? (f2_unpack(s1_2).x + f2_unpack(s1_2).y) * ex2_fast(hs.left) : 0.f;
        }
        row.join(p, sh[turn], sh[turn ^ 1], zr, sum, cT);
        next = distill_entry<HARD>(p, r + gridDim.x, tid);
        T *gr = g ? g + r * p.ld_g : nullptr;
        if (g && (row.dead || row.exact)) {
            row.other_rows(p, zr, gr, cT);
        } else if (g) {
            const DistillScale cs(row.sum.m, cT), hs(row.sum.m, LOG2E);
            const float af = row.aq * ex2_fast(cs.left), bf = HARD ? row.bq * ex2_fast(hs.left) : 0.f;
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const int32_t col = (j * NT + tid) * V;
                if (col >= p.C) break;
                float o[V];
                row.template grad<false>(raw[j], cs, hs, af, bf, o);
                row_store(gr, col, p.C, o);
            }
        }
        if (!STAGED) load(r + gridDim.x);   // (while the rest of this row is done)
        distill_sync<NT>();
        row.finish(p, sh[turn], r, cT, gr, acc);
    }
    if (STAGED && tid == 0 && *(volatile int *)&dead) mbar_settle(&full, 1, issued);
    if (p.loss_sum) loss_finish_first<DISTILL_TELLS(NT)>(acc, p.block_partial, p.ticket, p.loss_sum);
}

// Longer rows, which no ring holds, come through shared memory in chunks of a piece a thread, with as many slots as two blocks an SM have room for; one warp asks for them
// (cp.async.bulk).  Where a gradient is asked for they come twice, the second time from the L2 for the most part.
// 2048 x 131072 fp32: 530 us (4.1 TB/s).
#define DISTILL_LONG_NT 512
#define DISTILL_SLOTS 13
template <typename T, bool HARD>
__global__ void __launch_bounds__(DISTILL_LONG_NT + 32, 2)
k_distill_long(Distill p, const T *z, T *g)
{
    constexpr int V = RowVec<T>::V, NT = DISTILL_LONG_NT, CHUNK = NT;   // pieces
    extern __shared__ uint4 ring[];   // [slots][CHUNK]
    __shared__ DistillShared<NT> sh[2];
    __shared__ uint64_t full[DISTILL_SLOTS], empty[DISTILL_SLOTS];
    __shared__ int dead;
    const int tid = threadIdx.x, lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < DISTILL_SLOTS; ++i) mbar_init(full + i, 1), mbar_init(empty + i, NT / 32);
        dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid < NT) sh[0].clear(), sh[1].clear();
    __syncthreads();
    sat_grid_wait();
    const int32_t pieces = (p.C + V - 1) / V, chunks = (pieces + CHUNK - 1) / CHUNK;
    double acc = 0.0;
    if (tid >= NT) {
        if (lane == 0) {
            uint32_t slot = 0, turn = 0, issued = 0;
            for (int64_t r = blockIdx.x; r < p.rows && !*(volatile int *)&dead; r += gridDim.x)
                for (int32_t i = 0; i < (g ? 2 * chunks : chunks); ++i) {
                    const int32_t c = i < chunks ? i : i - chunks, here = pieces - c * CHUNK < CHUNK ? pieces - c * CHUNK : CHUNK;
                    if (turn > 0 && !mbar_wait<64>(empty + slot, (turn - 1) & 1u, &dead, p.status)) break;
                    mbar_expect_tx(full + slot, (uint32_t)here * 16);
                    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(ring + slot * CHUNK)),
                                 "l"(z + r * p.ld_z + (int64_t)c * CHUNK * V), "r"((uint32_t)here * 16), "r"(smem_u32(full + slot))
                                 : "memory");
                    ++issued;
                    if (++slot == DISTILL_SLOTS) slot = 0, ++turn;
                }
            if (*(volatile int *)&dead) mbar_settle(full, DISTILL_SLOTS, issued);
        }
    } else {
        const float cT = LOG2E / p.T;
        int which = 0;
        uint32_t slot = 0, phase = 0;
        DistillEntry next = distill_entry<HARD>(p, blockIdx.x, tid);
        auto release = [&](uint32_t s) {
            fence_async_smem();   // these loads are done before the next ones from memory land
            __syncwarp();
            if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(empty + s)) : "memory");
        };
        for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x, which ^= 1) {
            const T *zr = z + r * p.ld_z;
            DistillRow<T, NT, HARD> row;
            row.en = next;
            distill_known(p, row.en);
            row.zc = row.en.id >= 0 ? RowVec<T>::from(zr[row.en.id]) : 0.f;
            row.zy = row.en.y >= 0 ? RowVec<T>::from(zr[row.en.y]) : 0.f;
            // sums relative to the largest logit so far
            float m = -INFINITY;
            DistillScale cs = distill_scale(m, p.T, cT), hs = distill_scale(m, 1.f, LOG2E);
            uint64_t s_2 = 0, s1_2 = 0;
            auto step = [&](uint32_t &s, uint32_t &ph) {
                if (++s == DISTILL_SLOTS) s = 0, ph ^= 1u;
            };
            for (int32_t c = 0; c < chunks; c += 2) {   // two chunks at a time
                uint4 raw[2];
                float top = m;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int32_t piece = (c + u) * CHUNK + tid;
                    raw[u] = RowVec<T>::lowest();
                    if (c + u >= chunks) break;
                    (void)mbar_wait(full + slot, phase, &dead, p.status);   // (having given up, all finish on what is there)
                    if (piece < pieces) raw[u] = ring[slot * CHUNK + tid];
                    if (piece == pieces - 1 && p.C % V) raw[u] = RowVec<T>::cut(raw[u], p.C % V);
                    release(slot);
                    step(slot, phase);
                }
                top = fmaxf(top, fmaxf(RowVec<T>::largest(raw[0]), RowVec<T>::largest(raw[1])));
                if (top > m) {   // (rare after the first chunks)
                    const DistillScale ns = distill_scale(top, p.T, cT), ks = distill_scale(top, 1.f, LOG2E);
                    const float f = ex2_fast(cs.o - ns.o);
                    s_2 = f2_mul(s_2, f2_pack(f, f));
                    if (HARD) {
                        const float f1 = ex2_fast(hs.o - ks.o);
                        s1_2 = f2_mul(s1_2, f2_pack(f1, f1));
                    }
                    cs = ns, hs = ks, m = top;
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) distill_add<T, HARD, false>(raw[u], cs, hs, s_2, s1_2);
            }
            DistillSum sum = {m, (f2_unpack(s_2).x + f2_unpack(s_2).y) * ex2_fast(cs.left), 0.f};
            if (HARD) sum.s1 = (f2_unpack(s1_2).x + f2_unpack(s1_2).y) * ex2_fast(hs.left);
            row.join(p, sh[which], sh[which ^ 1], zr, sum, cT);
            next = distill_entry<HARD>(p, r + gridDim.x, tid);
            T *gr = g ? g + r * p.ld_g : nullptr;
            if (g) {
                const DistillScale gs(row.sum.m, cT), gh(row.sum.m, LOG2E);
                const float af = row.aq * ex2_fast(gs.left), bf = HARD ? row.bq * ex2_fast(gh.left) : 0.f;
                const bool other = row.dead || row.exact;   // (its chunks are taken off all the same)
                if (other) row.other_rows(p, zr, gr, cT);
                for (int32_t c = 0; c < chunks; c += 2) {
                    uint4 raw[2];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        raw[u] = make_uint4(0u, 0u, 0u, 0u);
                        if (c + u >= chunks) break;
                        (void)mbar_wait(full + slot, phase, &dead, p.status);
                        if ((c + u) * CHUNK + tid < pieces) raw[u] = ring[slot * CHUNK + tid];
                        release(slot);
                        step(slot, phase);
                    }
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int32_t piece = (c + u) * CHUNK + tid;
                        if (piece >= pieces || other) break;
                        float o[V];
                        row.template grad<false>(raw[u], gs, gh, af, bf, o);
                        row_store(gr, piece * V, p.C, o);
                    }
                }
            }
            distill_sync<NT>();
            row.finish(p, sh[which], r, cT, gr, acc);
        }
    }
    __syncwarp();
    __syncthreads();
    if (p.loss_sum) loss_finish_first<DISTILL_TELLS(NT)>(acc, p.block_partial, p.ticket, p.loss_sum);
}

template <typename T, int TPR, int CH, int NE, bool HARD, bool NEAR = false>
static void distill_rows_go(sat_ctx *ctx, const Distill &p, const T *z, T *g)
{
    const int resident = CH * RowVec<T>::V > 16 ? 2 : NE > 4 ? 3 : 4;   // blocks of an SM: all of them at work from the beginning to the end
    const unsigned blocks = (unsigned)std::min<int64_t>(cdiv64(p.rows, 256 / TPR), (int64_t)ctx->sms * resident);
    sat_pdl(ctx->stream, k_distill_rows<T, TPR, CH, NE, HARD, NEAR>, blocks, 256, (256 / TPR) * distill_stride<TPR, CH, RowVec<T>::V>() * sizeof(float))(p, z, g);
}
template <typename T, int NT, int CH, bool HARD, bool STAGED>
static sat_status distill_wide_go(sat_ctx *ctx, const Distill &p, const T *z, T *g)
{
    static PerDeviceOnce set;
    constexpr int stage = STAGED ? NT * CH * 16 : 0;
    if (STAGED && set.need(ctx->device)) {
        SAT_CUDA(ctx, cudaFuncSetAttribute(k_distill_wide<T, NT, CH, HARD, STAGED>, cudaFuncAttributeMaxDynamicSharedMemorySize, stage));
        set.mark(ctx->device);
    }
    sat_pdl(ctx->stream, k_distill_wide<T, NT, CH, HARD, STAGED>, (unsigned)std::min<int64_t>(p.rows, ctx->sms * (1024 / NT)), NT, stage)(p, z, g);
    return SAT_OK;
}
template <typename T, bool HARD>
static sat_status distill_launch(sat_ctx *ctx, const Distill &p, const T *z, T *g)
{
    constexpr int V = RowVec<T>::V, CH = 16 / V;   // 16 elements a lane
    const int32_t pieces = (p.C + V - 1) / V;
    if (pieces > 32 * 2 * CH) {
        // a block whose registers hold the row in four pieces a thread, or in eight, staged; or the ring, which holds less than the last of these
        if (pieces <= 128 * 4 && p.k <= 128) return distill_wide_go<T, 128, 4, HARD, false>(ctx, p, z, g);
        if (pieces <= 256 * 4) return distill_wide_go<T, 256, 4, HARD, false>(ctx, p, z, g);
        if (pieces <= 512 * 4) return distill_wide_go<T, 512, 4, HARD, false>(ctx, p, z, g);
        if (pieces <= 512 * 8) return distill_wide_go<T, 512, 8, HARD, false>(ctx, p, z, g);
        if (pieces <= 1024 * 8) return distill_wide_go<T, 1024, 8, HARD, true>(ctx, p, z, g);
        static PerDeviceOnce set;
        constexpr int smem = DISTILL_SLOTS * DISTILL_LONG_NT * 16;
        if (set.need(ctx->device)) {
            SAT_CUDA(ctx, cudaFuncSetAttribute(k_distill_long<T, HARD>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
            set.mark(ctx->device);
        }
        sat_pdl(ctx->stream, k_distill_long<T, HARD>, (unsigned)std::min<int64_t>(p.rows, ctx->sms * 2), DISTILL_LONG_NT + 32, smem)(p, z, g);
        return SAT_OK;
    }
    if (p.T > DISTILL_NEAR_FROM) {   // (fewer shapes of this one; the same with and without losses, so that a gradient is the same bits)
        if (pieces > 32 * CH) distill_rows_go<T, 32, 2 * CH, 8, HARD, true>(ctx, p, z, g);
        else if (pieces > 16 * CH || p.k > 64) distill_rows_go<T, 32, CH, 8, HARD, true>(ctx, p, z, g);
        else if (pieces > 4 * CH || p.k > 16) distill_rows_go<T, 16, CH, 4, HARD, true>(ctx, p, z, g);
        else distill_rows_go<T, 4, CH, 4, HARD, true>(ctx, p, z, g);
        return SAT_OK;
    }
    // the fewest lanes that hold the row and, with four entries each, the teacher's (two, where that is enough: more warps fit)
    auto rows = [&](auto two, auto four, int tpr) {
        if (p.k <= 2 * tpr) two(ctx, p, z, g);
        else four(ctx, p, z, g);
        return SAT_OK;
    };
    if (pieces > 32 * CH) return rows(distill_rows_go<T, 32, 2 * CH, 8, HARD>, distill_rows_go<T, 32, 2 * CH, 8, HARD>, 32);
    if (p.k > 128) return rows(distill_rows_go<T, 32, CH, 8, HARD>, distill_rows_go<T, 32, CH, 8, HARD>, 32);
    if (pieces > 16 * CH || p.k > 64) return rows(distill_rows_go<T, 32, CH, 2, HARD>, distill_rows_go<T, 32, CH, 4, HARD>, 32);
    if (pieces > 8 * CH || p.k > 32) return rows(distill_rows_go<T, 16, CH, 2, HARD>, distill_rows_go<T, 16, CH, 4, HARD>, 16);
    if (pieces > 4 * CH || p.k > 16) return rows(distill_rows_go<T, 8, CH, 2, HARD>, distill_rows_go<T, 8, CH, 4, HARD>, 8);
    if (pieces > 2 * CH || p.k > 8) return rows(distill_rows_go<T, 4, CH, 2, HARD>, distill_rows_go<T, 4, CH, 4, HARD>, 4);
    return rows(distill_rows_go<T, 2, CH, 2, HARD>, distill_rows_go<T, 2, CH, 4, HARD>, 2);
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
    SAT_TRY(sat_ensure(ctx, ctx->buf_distill, (size_t)ctx->sms * 8 * sizeof(double)));   // of the blocks of a launch
    Distill p = {rows, n_classes, k, ld_z, ld_g, top_ids, top_logits, temperature, hard, labels, row_weight, weight, row_loss, (double *)ctx->buf_distill.p,
                 ctx->d_flag + 2, loss_sum, ctx->d_flag + 1};
    ProfScope prof(ctx, SATK_LOSS, (g ? 2.0 : 1.0) * type_bytes(type) * (double)rows * n_classes, 0.0);
    if (hard > 0.f) {
        if (type == SAT_F32) SAT_TRY((distill_launch<float, true>(ctx, p, (const float *)z, (float *)g)));
        else if (type == SAT_BF16) SAT_TRY((distill_launch<__nv_bfloat16, true>(ctx, p, (const __nv_bfloat16 *)z, (__nv_bfloat16 *)g)));
        else SAT_TRY((distill_launch<__half, true>(ctx, p, (const __half *)z, (__half *)g)));
    } else {
        if (type == SAT_F32) SAT_TRY((distill_launch<float, false>(ctx, p, (const float *)z, (float *)g)));
        else if (type == SAT_BF16) SAT_TRY((distill_launch<__nv_bfloat16, false>(ctx, p, (const __nv_bfloat16 *)z, (__nv_bfloat16 *)g)));
        else SAT_TRY((distill_launch<__half, false>(ctx, p, (const __half *)z, (__half *)g)));
    }
    SAT_LAUNCHED(ctx);
    return SAT_OK;
}

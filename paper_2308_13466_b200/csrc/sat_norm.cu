// Layer norm by rows, forward and backward:
//     mu = sum x / d,  s = (sum (x - mu)^2 / d + eps)^(-1/2),  xh = (x - mu) s,  y = xh gamma + beta
//     u = g gamma,  g_x = s (u - sum u / d - xh sum (u xh) / d),  g_gamma = sum over rows g xh,  g_beta = sum over rows g
#include "sat_ptx.h"
#include "sat_rows.h"

#include <algorithm>

#define NORM_MAX 16384   // width: a row lies in the registers of one block

// The work on 16 bytes of a row, by pairs.
// Forward: x -> x - m0 (zeros behind the row's end), with its sum and that of its squares
template <int V>
__device__ __forceinline__ void norm_centre(uint64_t (&v)[V / 2], float m0, int32_t col, int32_t d, uint64_t &a, uint64_t &b)
{
    const uint64_t less = f2_all(-m0);
#pragma unroll
    for (int i = 0; i < V / 2; ++i) v[i] = f2_add(v[i], less);
    if (col + V > d) {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) v[i] = f2_pack(col + 2 * i < d ? f2_unpack(v[i]).x : 0.f, col + 2 * i + 1 < d ? f2_unpack(v[i]).y : 0.f);
    }
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        a = f2_add(a, v[i]);
        b = f2_fma(v[i], v[i], b);
    }
}
// (what rounding leaves of a constant row may be below zero; a row that is no number keeps that)
__device__ __forceinline__ float norm_variance(float v) { return v < 0.f ? 0.f : v; }
// ... -> y = (x - m0 - m1) s gamma + beta
template <typename T>
__device__ __forceinline__ void norm_finish(T *y, int32_t col, int32_t d, const uint64_t (&v)[RowVec<T>::V / 2], float m1, float sd, const uint64_t (&gamma)[RowVec<T>::V / 2],
                                            const uint64_t (&beta)[RowVec<T>::V / 2])
{
    constexpr int V = RowVec<T>::V;
    const uint64_t less = f2_all(-m1), s = f2_all(sd);
    uint64_t o[V / 2];
#pragma unroll
    for (int i = 0; i < V / 2; ++i) o[i] = f2_fma(f2_mul(f2_add(v[i], less), s), gamma[i], beta[i]);
    float out[V];
    pair_floats<V>(o, out);
    row_store(y, col, d, out);
}
// Backward: x -> xh, g -> u (both zero behind the row's end, or times zero), with sum u, sum u xh and the columns' sums
template <int V>
__device__ __forceinline__ void norm_back(uint64_t (&x)[V / 2], uint64_t (&g)[V / 2], float m, float sd, const uint64_t (&gamma)[V / 2], uint64_t &s1, uint64_t &s2,
                                          uint64_t (&ag)[V / 2], uint64_t (&ab)[V / 2])
{
    const uint64_t less = f2_all(-m), s = f2_all(sd);
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        x[i] = f2_mul(f2_add(x[i], less), s);
        ag[i] = f2_fma(g[i], x[i], ag[i]);
        ab[i] = f2_add(ab[i], g[i]);
        g[i] = f2_mul(g[i], gamma[i]);
        s1 = f2_add(s1, g[i]);
        s2 = f2_fma(g[i], x[i], s2);
    }
}
// ... -> g_x = s (u - c1 - xh c2)
template <typename T>
__device__ __forceinline__ void norm_back_finish(T *gx, int32_t col, int32_t d, const uint64_t (&xh)[RowVec<T>::V / 2], const uint64_t (&u)[RowVec<T>::V / 2], float sd, float c1, float c2)
{
    constexpr int V = RowVec<T>::V;
    const uint64_t s = f2_all(sd), k1 = f2_all(-c1), k2 = f2_all(-c2);
    uint64_t o[V / 2];
#pragma unroll
    for (int i = 0; i < V / 2; ++i) o[i] = f2_mul(f2_add(u[i], f2_fma(xh[i], k2, k1)), s);
    float out[V];
    pair_floats<V>(o, out);
    row_store(gx, col, d, out);
}

// =====================================================================================
// rows of up to 512 elements: TPR lanes hold one in registers, CH times 16 bytes each.  Bound by memory: 612257 x 256 fp32 forward 198 to 214 us (91 to 98 % of the copy rate, from one GPU to
// another; without the next row on its way 245), backward 287 to 295 (the copy rate).  Rows of 9 to 16 pieces of 16 bytes leave half of the lanes' room empty (610000 x 50 fp32: 40 and 43 % of the copy rate), rows of 16 bits
// lie on twice the lanes that they need with 16 elements each (400000 x 256 bf16: 60 and 67 %).
// =====================================================================================

// (the next row is asked for before this one is worked on)
template <typename T, int TPR, int CH>
__global__ void __launch_bounds__(256)
k_norm_fwd(int64_t rows, int32_t d, const T *x, int64_t ld_x, const float *__restrict__ gamma, const float *__restrict__ beta, float eps, T *y,
           int64_t ld_y, float *__restrict__ mean, float *__restrict__ rstd)
{
    sat_grid_wait();
    constexpr int V = RowVec<T>::V, H = V / 2, NT = 256, RPB = NT / TPR;
    float2 (*none)[32] = nullptr;
    int turn = 0;
    const int t = threadIdx.x % TPR;
    const float inv_d = 1.f / (float)d;
    const int64_t step = (int64_t)gridDim.x * RPB;
    int64_t r = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    uint4 raw[CH];
    auto fetch = [&](int64_t row) {
#pragma unroll
        for (int j = 0; j < CH; ++j) raw[j] = row_load_raw(x + row * ld_x, row < rows ? (j * TPR + t) * V : d, d);
    };
    fetch(r);
    // (rows that share a warp go on together: its lanes meet in the sums)
    for (int64_t first = r - (threadIdx.x & 31) / TPR; first < rows; first += step, r += step) {
        uint64_t v[CH][H], s = 0;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            pair_unpack<T>(raw[j], (j * TPR + t) * V, d, v[j]);
#pragma unroll
            for (int i = 0; i < H; ++i) s = f2_add(s, v[j][i]);
        }
        fetch(r + step);
        const float m0 = row_sum<TPR>(f2_sum(s), none, turn) * inv_d;
        // what the rounding of the mean left is taken off with the squares
        uint64_t a = 0, b = 0;
#pragma unroll
        for (int j = 0; j < CH; ++j) norm_centre<V>(v[j], m0, (j * TPR + t) * V, d, a, b);
        const float2 ab = row_sum2<TPR>(f2_sum(a), f2_sum(b), none, turn);
        const float m1 = ab.x * inv_d, var = norm_variance(ab.y * inv_d - m1 * m1), sd = 1.f / sqrtf(var + eps);
        if (r >= rows) continue;
        if (t == 0) {
            if (mean) mean[r] = m0 + m1;
            if (rstd) rstd[r] = sd;
        }
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int32_t col = (j * TPR + t) * V;
            if (col >= d) continue;
            uint64_t ga[H], be[H];
            pair_param<V>(gamma, col, d, 1.f, ga);
            pair_param<V>(beta, col, d, 0.f, be);
            norm_finish<T>(y + r * ld_y, col, d, v[j], m1, sd, ga, be);
        }
    }
}

// Sums of few blocks: the block that ends last adds them up itself, which saves a launch.  A thread takes four columns of [g_gamma | g_beta] and every side-th block; `red` has room for a float4 a thread.
struct NormLast {
    int *ticket;           // null: k_norm_sums follows
    int accumulate;
    float *g_gamma, *g_beta;
};
template <int NT>
__device__ __forceinline__ void norm_last(const NormLast &l, const float *part, int32_t d, int32_t ld_part, float4 *red)
{
    __shared__ int last;
    const int tid = threadIdx.x, blocks = (int)gridDim.x;
    __threadfence();
    __syncthreads();
    if (tid == 0) last = atomicAdd(l.ticket, 1) == blocks - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    const int quads = ld_part / 2, side = quads < NT ? NT / quads : 1, mine = quads < NT ? tid / quads : 0;
    for (int q0 = quads < NT ? tid % quads : tid; q0 < (quads < NT ? quads : (quads + NT - 1) / NT * NT); q0 += NT) {
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        if (mine < side && q0 < quads)
#pragma unroll 8
            for (int b = mine; b < blocks; b += side) {
                const float4 v = __ldcg(reinterpret_cast<const float4 *>(part + (int64_t)b * 2 * ld_part) + q0);
                s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
            }
        if (side > 1) {
            red[tid] = s;
            __syncthreads();
            for (int i = 1; mine == 0 && i < side; ++i) {
                const float4 v = red[tid + i * quads];
                s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
            }
        }
        if (mine != 0 || q0 >= quads) continue;
        const int32_t col = 4 * q0 % ld_part;
        float *out = 4 * q0 < ld_part ? l.g_gamma : l.g_beta;
        const float f[4] = {s.x, s.y, s.z, s.w};
        if (out)
            for (int i = 0; i < 4; ++i)
                if (col + i < d) out[col + i] = l.accumulate ? out[col + i] + f[i] : f[i];
    }
    if (tid == 0) *l.ticket = 0;   // the next launch on this stream starts from zero again
}

// The sums over the rows: a thread adds up its columns over its rows in registers, the block leaves one row of partial sums [g_gamma | g_beta], k_norm_sums
// adds these up in a fixed order.
template <typename T, int TPR, int CH>
__global__ void __launch_bounds__(256, CH * RowVec<T>::V > 8 ? 2 : 3)
k_norm_bwd(int64_t rows, int32_t d, const T *x, int64_t ld_x, const T *g, int64_t ld_g, const float *__restrict__ gamma,
           const float *__restrict__ mean, const float *__restrict__ rstd, T *gx, int64_t ld_gx, float *part, int32_t ld_part, NormLast last)
{
    sat_grid_wait();
    constexpr int V = RowVec<T>::V, H = V / 2, NT = 256, RPB = NT / TPR;
    float2 (*none)[32] = nullptr;
    int turn = 0;
    const int t = threadIdx.x % TPR;
    const float inv_d = 1.f / (float)d;
    uint64_t ag2[CH][H] = {}, ab2[CH][H] = {};
    const int64_t step = (int64_t)gridDim.x * RPB;
    int64_t r = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    for (int64_t first = r - (threadIdx.x & 31) / TPR; first < rows; first += step, r += step) {
        const bool ok = r < rows;
        uint4 xr[CH], gr[CH];
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int32_t col = ok ? (j * TPR + t) * V : d;
            xr[j] = row_load_raw(x + r * ld_x, col, d);
            gr[j] = row_load_raw(g + r * ld_g, col, d);
        }
        const float m = ok ? __ldg(mean + r) : 0.f, sd0 = ok ? __ldg(rstd + r) : 0.f;
        uint64_t xh[CH][H], u[CH][H], s1 = 0, s2 = 0;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int32_t col = (j * TPR + t) * V;
            pair_unpack<T>(xr[j], col, d, xh[j]);
            pair_unpack<T>(gr[j], col, d, u[j]);
            uint64_t ga[H];
            pair_param<V>(gamma, col, d, 1.f, ga);
            norm_back<V>(xh[j], u[j], m, sd0, ga, s1, s2, ag2[j], ab2[j]);
        }
        if (!gx) continue;   // (the same for all threads)
        const float2 s = row_sum2<TPR>(f2_sum(s1), f2_sum(s2), none, turn);
        if (!ok) continue;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int32_t col = (j * TPR + t) * V;
            if (col < d) norm_back_finish<T>(gx + r * ld_gx, col, d, xh[j], u[j], sd0, s.x * inv_d, s.y * inv_d);
        }
    }
    if (!part) return;
    float *out = part + (int64_t)blockIdx.x * 2 * ld_part;
    __shared__ float sum[2][TPR * V];
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        float ag[V], ab[V];
        pair_floats<V>(ag2[j], ag);
        pair_floats<V>(ab2[j], ab);
        for (int w = 0; w < RPB; ++w) {   // one group of rows after the other
            __syncthreads();
            if (threadIdx.x / TPR == w) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    sum[0][t * V + i] = w ? sum[0][t * V + i] + ag[i] : ag[i];
                    sum[1][t * V + i] = w ? sum[1][t * V + i] + ab[i] : ab[i];
                }
            }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * TPR * V; c += NT) {
            const int which = c / (TPR * V), i = c % (TPR * V), col = j * TPR * V + i;
            if (col < ld_part) out[which * ld_part + col] = sum[which][i];   // (zeros behind the last column)
        }
    }
    if (last.ticket) {
        __shared__ float4 red[NT];
        norm_last<NT>(last, part, d, ld_part, red);
    }
}

// =====================================================================================
// wider rows: a block holds one in registers, CH times 16 bytes a thread; the next ones are on their way into a ring in shared memory (cp.async.bulk), so that what an SM
// has asked for does not depend on its registers.  A slot is asked for again behind the barrier of the row's sums, when all threads have taken their part of it.
// 16384 x 4096 bf16 backward 85 us (73 % of the copy rate; with 8 elements a thread and rows asked for into registers 108): instructions, and a barrier a row; forward 79 (53 %): two barriers a row, and two blocks an SM to
// fill their waits.
// =====================================================================================
#define NORM_SLOTS 8
// gamma and beta in shared memory, or else from the L1, which has the rest of the SM.  Measured, kept against not: gradients of 50000 x 2048 bf16 125 / 225 us, of 16384 x
// 4096 bf16 85 / 100, of 16000 x 8192 fp32 248 / 266, of 100000 x 1024 fp32 (where they take a slot's room) 227 / 218; 100000 x 1024 fp32 forward 131 / 166.
#define NORM_KEPT(NT, V, BACK) ((NT) >= 256 || (V) == 8 || !(BACK))
#define NORM_RING_BLOCKS(NT) ((NT) >= 512 ? 1 : 640 / (NT))   // of an SM
template <typename T>
struct NormRing {
    int64_t rows;
    int32_t d, slots;
    const T *x, *g;        // backward: both
    int64_t ld_x, ld_g, ld_y;
    const float *gamma, *beta;
    float eps;
    T *y;                  // or g_x
    float *mean, *rstd;    // forward: written, backward: read
    float *part;
    int32_t ld_part;
    NormLast last;
    int *status;
};
template <typename T, int NT, int CH, bool BACK>
__global__ void __launch_bounds__(NT, NORM_RING_BLOCKS(NT))
k_norm_ring(NormRing<T> p)
{
    constexpr int V = RowVec<T>::V, H = V / 2;
    constexpr bool KEPT = NORM_KEPT(NT, RowVec<T>::V, BACK);
    extern __shared__ uint4 norm_smem[];
    __shared__ uint64_t full[NORM_SLOTS];
    __shared__ int dead;
    __shared__ float2 red[2][32];
    const int tid = threadIdx.x;
    const int32_t pieces = (p.d + V - 1) / V, stage = (BACK ? 2 : 1) * pieces;   // of 16 bytes
    if (tid == 0) {
        for (int i = 0; i < NORM_SLOTS; ++i) mbar_init(full + i, 1);
        dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    sat_grid_wait();
    // gamma and beta of rows that leave no room for them in the L1: four elements of a piece, then the next four of all pieces
    uint4 *gamma_s = norm_smem + p.slots * stage, *beta_s = gamma_s + pieces * (V / 4);
    for (int32_t i = tid; KEPT && i < pieces; i += NT) {
        float f[V];
        param_load<V>(p.gamma, i * V, p.d, 1.f, f);
#pragma unroll
        for (int h = 0; h < V / 4; ++h) gamma_s[h * pieces + i] = make_uint4(__float_as_uint(f[4 * h]), __float_as_uint(f[4 * h + 1]), __float_as_uint(f[4 * h + 2]), __float_as_uint(f[4 * h + 3]));
        if (BACK) continue;
        param_load<V>(p.beta, i * V, p.d, 0.f, f);
#pragma unroll
        for (int h = 0; h < V / 4; ++h) beta_s[h * pieces + i] = make_uint4(__float_as_uint(f[4 * h]), __float_as_uint(f[4 * h + 1]), __float_as_uint(f[4 * h + 2]), __float_as_uint(f[4 * h + 3]));
    }
    auto params = [&](const uint4 *of, const float *at, float other, int32_t piece, uint64_t (&f)[H]) {
        if (!KEPT) return pair_param<V>(at, piece * V, p.d, other, f);
#pragma unroll
        for (int h = 0; h < V / 4; ++h) {
            const uint4 v = of[h * pieces + piece];
            f[2 * h] = f2_pack(__uint_as_float(v.x), __uint_as_float(v.y)), f[2 * h + 1] = f2_pack(__uint_as_float(v.z), __uint_as_float(v.w));
        }
    };
    __syncthreads();
    uint32_t issued = 0;
    auto ask = [&](int64_t r, uint32_t slot) {   // first thread
        if (r >= p.rows || *(volatile int *)&dead) return;
        ++issued;
        mbar_expect_tx(full + slot, (uint32_t)stage * 16);
        auto copy = [&](const T *from, uint4 *to) {
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(to)), "l"(from), "r"((uint32_t)pieces * 16),
                         "r"(smem_u32(full + slot))
                         : "memory");
        };
        copy(p.x + r * p.ld_x, norm_smem + slot * stage);
        if (BACK) copy(p.g + r * p.ld_g, norm_smem + slot * stage + pieces);
    };
    if (tid == 0)
        for (int i = 0; i < p.slots; ++i) ask(blockIdx.x + (int64_t)i * gridDim.x, i);
    int turn = 0;
    uint32_t slot = 0, phase = 0;
    const float inv_d = 1.f / (float)p.d;
    uint64_t ag[BACK ? CH : 1][H] = {}, ab[BACK ? CH : 1][H] = {};
    float m_next = 0.f, sd_next = 0.f;
    auto statistics = [&](int64_t r) {
        if (BACK && r < p.rows) m_next = __ldg(p.mean + r), sd_next = __ldg(p.rstd + r);
    };
    statistics(blockIdx.x);
    for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
        (void)mbar_wait(full + slot, phase, &dead, p.status);   // (having given up, all finish on what is there)
        const uint4 *from = norm_smem + slot * stage;
        uint64_t v[CH][H], u[BACK ? CH : 1][H];
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int32_t at = j * NT + tid;
            if (at < pieces) {
                pair_unpack<T>(from[at], at * V, p.d, v[j]);
                if (BACK) pair_unpack<T>(from[pieces + at], at * V, p.d, u[j % (BACK ? CH : 1)]);
            } else {
#pragma unroll
                for (int i = 0; i < H; ++i) v[j][i] = u[j % (BACK ? CH : 1)][i] = 0;
            }
        }
        fence_async_smem();   // these loads are done before a later row lands there
        T *yr = p.y + r * p.ld_y;
        const int64_t later = r + (int64_t)p.slots * gridDim.x;
        if constexpr (BACK) {
            const float m = m_next, sd = sd_next;
            statistics(r + gridDim.x);
            uint64_t s1 = 0, s2 = 0;
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                if (j * NT + tid >= pieces) break;
                uint64_t ga[H];
                params(gamma_s, p.gamma, 1.f, j * NT + tid, ga);
                norm_back<V>(v[j], u[j], m, sd, ga, s1, s2, ag[j], ab[j]);
            }
            const float2 s = row_sum2<NT>(f2_sum(s1), f2_sum(s2), red, turn);
            if (tid == 0) ask(later, slot);
            if (p.y) {
#pragma unroll
                for (int j = 0; j < CH; ++j) {
                    const int32_t col = (j * NT + tid) * V;
                    if (col < p.d) norm_back_finish<T>(yr, col, p.d, v[j], u[j], sd, s.x * inv_d, s.y * inv_d);
                }
            }
        } else {
            uint64_t s = 0;
#pragma unroll
            for (int j = 0; j < CH; ++j)
#pragma unroll
                for (int i = 0; i < H; ++i) s = f2_add(s, v[j][i]);
            const float m0 = row_sum<NT>(f2_sum(s), red, turn) * inv_d;
            if (tid == 0) ask(later, slot);
            uint64_t a = 0, b = 0;   // (as in k_norm_fwd)
#pragma unroll
            for (int j = 0; j < CH; ++j) norm_centre<V>(v[j], m0, (j * NT + tid) * V, p.d, a, b);
            const float2 t = row_sum2<NT>(f2_sum(a), f2_sum(b), red, turn);
            const float m1 = t.x * inv_d, var = norm_variance(t.y * inv_d - m1 * m1), sd = 1.f / sqrtf(var + p.eps);
            if (tid == 0) {
                if (p.mean) p.mean[r] = m0 + m1;
                if (p.rstd) p.rstd[r] = sd;
            }
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const int32_t col = (j * NT + tid) * V;
                if (col >= p.d) break;
                uint64_t ga[H], be[H];
                params(gamma_s, p.gamma, 1.f, j * NT + tid, ga);
                params(beta_s, p.beta, 0.f, j * NT + tid, be);
                norm_finish<T>(yr, col, p.d, v[j], m1, sd, ga, be);
            }
        }
        if (++slot == (uint32_t)p.slots) slot = 0, phase ^= 1u;
    }
    if (tid == 0 && *(volatile int *)&dead) mbar_settle(full, (uint32_t)p.slots, issued);
    if constexpr (BACK) {
        if (!p.part) return;
        float *out = p.part + (int64_t)blockIdx.x * 2 * p.ld_part;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int32_t col = (j * NT + tid) * V;
            float sum[V];
            pair_floats<V>(ag[j], sum);
            row_store_f32<V>(out, col, p.d, sum);
            pair_floats<V>(ab[j], sum);
            row_store_f32<V>(out + p.ld_part, col, p.d, sum);
        }
        if (p.last.ticket) norm_last<NT>(p.last, p.part, p.d, p.ld_part, nullptr);   // (rows of more than 512: a thread has four columns or more)
    }
}

// out[c] (+)= sum over b of part[b][c]: eight columns (a sector of memory) a block, 32 threads a column
__global__ void __launch_bounds__(256)
k_norm_sums(const float *__restrict__ part, int32_t blocks, int32_t d, int32_t ld_part, int accumulate, float *__restrict__ g_gamma, float *__restrict__ g_beta)
{
    sat_grid_wait();
    __shared__ float red[32][9];
    const int c = threadIdx.x & 7, w = threadIdx.x >> 3;
    const int32_t col = (int32_t)blockIdx.x * 8 + c;
    float *out = blockIdx.y ? g_beta : g_gamma;
    if (!out) return;
    float s = 0.f;
    for (int32_t b0 = w; col < d && b0 < blocks; b0 += 32 * 64) {   // (64 at a time: as with a block's rows)
        const int32_t b1 = b0 + 32 * 64 < blocks ? b0 + 32 * 64 : blocks;
        float some = 0.f;
#pragma unroll 8
        for (int32_t b = b0; b < b1; b += 32) some += __ldcg(part + ((int64_t)b * 2 + blockIdx.y) * ld_part + col);
        s += some;
    }
    red[w][c] = s;
    __syncthreads();
    const int lane = threadIdx.x & 31, mine = threadIdx.x >> 5;   // a warp per column
    s = red[lane][mine];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    const int32_t to = (int32_t)blockIdx.x * 8 + mine;
    if (lane == 0 && to < d) out[to] = accumulate ? out[to] + s : s;
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
    float *g_gamma, *g_beta;
    int accumulate;
};
// Blocks of a backward pass: `resident` of them, or as many times that as leave a thread no more than NORM_CHAIN rows.  A thread's sums are additions one after the other, in which many small
// terms would be lost beside a large sum; partial sums of blocks meet in shorter chains.  (Up to 7 million narrow rows nothing changes.)
#define NORM_CHAIN 512
static int32_t norm_blocks(int64_t rows, int32_t rows_of_block, int32_t resident)   // rows_of_block: side by side
{
    return resident * (int32_t)std::max<int64_t>(1, cdiv64(rows, (int64_t)resident * rows_of_block * NORM_CHAIN));
}
// room for a row of partial sums of every block
template <typename T>
static sat_status norm_parts(const NormArgs<T> &a, int32_t blocks, int32_t ld_part, float **part)
{
    *part = nullptr;
    if (!a.g_gamma && !a.g_beta) return SAT_OK;
    SAT_TRY(sat_ensure(a.ctx, a.ctx->buf_norm, (size_t)blocks * 2 * ld_part * sizeof(float)));
    *part = (float *)a.ctx->buf_norm.p;
    return SAT_OK;
}
// Up to 32 KB of partial sums are added up by the last of the blocks.  Measured, with it against a launch of their own: 100 x 100 (4 blocks) 9.7 / 12.7 us, 60 x 500 (4) 10.2 /
// 11.8; 6000 x 50 (188 blocks, 84 KB) 14.7 / 12.7, 60000 x 30 (444) 18.9 / 12.8.
template <typename T>
static NormLast norm_last_of(const NormArgs<T> &a, int32_t blocks, int32_t ld_part, const float *part)
{
    const bool few = part && (int64_t)blocks * 2 * ld_part <= 8192;
    return NormLast{few ? a.ctx->d_flag + 2 : nullptr, a.accumulate, a.g_gamma, a.g_beta};
}
template <typename T>
static sat_status norm_sums(const NormArgs<T> &a, int32_t blocks, int32_t ld_part, const float *part)
{
    if (!part || norm_last_of(a, blocks, ld_part, part).ticket) return SAT_OK;
    sat_pdl(a.ctx->stream, k_norm_sums, dim3((unsigned)cdiv64(a.d, 8), 2), 256, 0)(part, blocks, a.d, ld_part, a.accumulate, a.g_gamma, a.g_beta);
    SAT_LAUNCHED(a.ctx);
    return SAT_OK;
}
template <typename T, int TPR, int CH>
static sat_status norm_rows_go(const NormArgs<T> &a, bool back)
{
    constexpr int RPB = 256 / TPR;
    sat_ctx *ctx = a.ctx;
    if (!back) {
        const int64_t blocks = std::min<int64_t>(cdiv64(a.rows, RPB), (int64_t)ctx->sms * 8);
        sat_pdl(ctx->stream, k_norm_fwd<T, TPR, CH>, (unsigned)blocks, 256, 0)(a.rows, a.d, a.x, a.ld_x, a.gamma, a.beta, a.eps, a.y, a.ld_y, a.mean, a.rstd);
        SAT_LAUNCHED(ctx);
        return SAT_OK;
    }
    // every block is a row of partial sums: as many as the SMs hold, and two rows a thread at least
    const int32_t blocks = (int32_t)std::min<int64_t>(cdiv64(a.rows, 2 * RPB), norm_blocks(a.rows, RPB, ctx->sms * (CH * RowVec<T>::V > 8 ? 2 : 3))), ld_part = (a.d + 7) & ~7;
    float *part;
    SAT_TRY(norm_parts(a, blocks, ld_part, &part));
    sat_pdl(ctx->stream, k_norm_bwd<T, TPR, CH>, (unsigned)blocks, 256, 0)(a.rows, a.d, a.x, a.ld_x, a.g, a.ld_g, a.gamma, (const float *)a.mean, (const float *)a.rstd, a.y, a.ld_y,
                                                                           part, ld_part, norm_last_of(a, blocks, ld_part, part));
    SAT_LAUNCHED(ctx);
    return norm_sums(a, blocks, ld_part, part);
}
template <typename T, int NT, int CH, bool BACK>
static sat_status norm_ring_go(const NormArgs<T> &a)
{
    static PerDeviceOnce set;
    sat_ctx *ctx = a.ctx;
    constexpr int room = (NORM_KEPT(NT, RowVec<T>::V, BACK) ? 208 : 128) * 1024 / NORM_RING_BLOCKS(NT);   // of a block; the rest is L1
    if (set.need(ctx->device)) {
        SAT_CUDA(ctx, cudaFuncSetAttribute(k_norm_ring<T, NT, CH, BACK>, cudaFuncAttributeMaxDynamicSharedMemorySize, room));
        set.mark(ctx->device);
    }
    const int32_t pieces = (a.d + RowVec<T>::V - 1) / RowVec<T>::V, stage = (BACK ? 2 : 1) * pieces * 16, params = NORM_KEPT(NT, RowVec<T>::V, BACK) ? (BACK ? 1 : 2) * pieces * RowVec<T>::V * 4 : 0;
    const int32_t slots = std::min(NORM_SLOTS, (room - params) / stage);   // one at least: 16,384 fp32 elements take 192 KB
    const int32_t resident = ctx->sms * NORM_RING_BLOCKS(NT), blocks = (int32_t)std::min<int64_t>(a.rows, BACK ? norm_blocks(a.rows, 1, resident) : resident), ld_part = (a.d + 7) & ~7;
    float *part = nullptr;
    if (BACK) SAT_TRY(norm_parts(a, blocks, ld_part, &part));
    const NormRing<T> p = {a.rows, a.d, slots, a.x, a.g, a.ld_x, a.ld_g, a.ld_y, a.gamma, a.beta, a.eps, a.y, a.mean, a.rstd, part, ld_part, norm_last_of(a, blocks, ld_part, part), ctx->d_flag + 1};
    sat_pdl(ctx->stream, k_norm_ring<T, NT, CH, BACK>, (unsigned)blocks, NT, (size_t)slots * stage + params)(p);
    SAT_LAUNCHED(ctx);
    return BACK ? norm_sums(a, blocks, ld_part, part) : SAT_OK;
}
template <typename T>
static sat_status norm_launch(const NormArgs<T> &a, bool back)
{
    constexpr int CH = 8 / RowVec<T>::V;   // pieces of a thread with 8 elements
    const int32_t pieces = (a.d + RowVec<T>::V - 1) / RowVec<T>::V;
    if (pieces <= 8) return norm_rows_go<T, 8, 1>(a, back);
    if (pieces <= 16 * CH) return norm_rows_go<T, 16, CH>(a, back);
    if (pieces <= 32 * CH) return norm_rows_go<T, 32, CH>(a, back);
    if (pieces <= 64 * CH) return norm_rows_go<T, 32, 2 * CH>(a, back);
    // (16 elements a thread: what a row costs a warp whatever it holds, its part of the sums above all, is then a fifth of the instructions)
    if (pieces <= 128 * CH) return back ? norm_ring_go<T, 64, 2 * CH, true>(a) : norm_ring_go<T, 64, 2 * CH, false>(a);
    if (pieces <= 256 * CH) return back ? norm_ring_go<T, 128, 2 * CH, true>(a) : norm_ring_go<T, 128, 2 * CH, false>(a);
    if (pieces <= 512 * CH) return back ? norm_ring_go<T, 256, 2 * CH, true>(a) : norm_ring_go<T, 256, 2 * CH, false>(a);
    if (pieces <= 1024 * CH) return back ? norm_ring_go<T, 512, 2 * CH, true>(a) : norm_ring_go<T, 512, 2 * CH, false>(a);
    return back ? norm_ring_go<T, 1024, 2 * CH, true>(a) : norm_ring_go<T, 1024, 2 * CH, false>(a);
}

static sat_status norm_check(sat_ctx *ctx, const char *who, int64_t rows, int32_t d, int type)
{
    if (!ok_type(type)) return sat_fail(ctx, SAT_EINVAL, "%s: unknown element type", who);
    if (rows < 0 || rows >= INT32_MAX || d <= 0 || d > NORM_MAX) return sat_fail(ctx, SAT_EINVAL, "%s: rows must be in [0, 2^31 - 1), the width in [1, %d]", who, NORM_MAX);
    return SAT_OK;
}
static bool norm_param_ok(const float *p) { return !p || aligned16(p); }

template <typename T>
static sat_status norm_as(sat_ctx *ctx, bool back, int64_t rows, int32_t d, const void *x, int32_t ld_x, const void *g, int32_t ld_g, const float *gamma, const float *beta,
                          float eps, void *y, int32_t ld_y, float *mean, float *rstd, float *g_gamma, float *g_beta, int accumulate)
{
    const NormArgs<T> a = {ctx, rows, d, (const T *)x, (const T *)g, ld_x, ld_g, ld_y, gamma, beta, eps, (T *)y, mean, rstd, g_gamma, g_beta, accumulate};
    return norm_launch(a, back);
}
#define NORM_AS(...)                                         \
    (type == SAT_F32    ? norm_as<float>(__VA_ARGS__)         \
     : type == SAT_BF16 ? norm_as<__nv_bfloat16>(__VA_ARGS__) \
                        : norm_as<__half>(__VA_ARGS__))

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
    return NORM_AS(ctx, false, rows, d, x, ld_x, nullptr, 0, gamma, beta, eps, y, ld_y, mean, rstd, nullptr, nullptr, 0);
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
    if (!g_x && !g_gamma && !g_beta) return sat_fail(ctx, SAT_EINVAL, "sat_layernorm_bwd: no result is asked for");
    if (rows == 0) {
        if (!accumulate && g_gamma) SAT_CUDA(ctx, cudaMemsetAsync(g_gamma, 0, (size_t)d * sizeof(float), ctx->stream));
        if (!accumulate && g_beta) SAT_CUDA(ctx, cudaMemsetAsync(g_beta, 0, (size_t)d * sizeof(float), ctx->stream));
        return SAT_OK;
    }
    ProfScope prof(ctx, SATK_NORM, (g_x ? 3.0 : 2.0) * type_bytes(type) * (double)rows * d, 14.0 * (double)rows * d);
    return NORM_AS(ctx, true, rows, d, x, ld_x, g, ld_g, gamma, nullptr, 0.f, g_x, ld_gx, const_cast<float *>(mean), const_cast<float *>(rstd), g_gamma, g_beta, accumulate);
}

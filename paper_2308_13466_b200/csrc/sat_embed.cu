// Embedding lookup with scaling, and its gradient by sorted tokens:
//     out[i] = scale table[t_i]            g_table[v] (+)= scale sum of g[i] over the i with t_i = v, in a fixed order: ascending i within a run of positions, then the runs
// The tokens are sorted once (sat_token_sort: keys of 32 bits, by digits, stable), the gradient then walks them in that order.
#include "sat_rows.h"

#include <algorithm>

// =====================================================================================
// lookup: a thread per 16 bytes of a row, bound by memory (32768 x 2048 bf16 of 32000 words: 48 us, 5.5 TB/s)
// =====================================================================================
#define EMB_UNROLL 4
template <typename T>
__global__ void __launch_bounds__(256)
k_embed(int64_t n, const int32_t *__restrict__ tokens, int32_t vocabulary, int32_t padding, const T *__restrict__ table, int64_t ld_table, int32_t d, float scale,
        T *__restrict__ out, int64_t ld_out, int *status)
{
    sat_grid_wait();
    constexpr int V = RowVec<T>::V;
    const int32_t pieces = (d + V - 1) / V;
    const int64_t total = n * pieces, step = (int64_t)gridDim.x * 256;
    for (int64_t i0 = (int64_t)blockIdx.x * 256 + threadIdx.x; i0 < total; i0 += EMB_UNROLL * step) {
        uint4 v[EMB_UNROLL];
        int64_t row[EMB_UNROLL];
        int32_t col[EMB_UNROLL];
#pragma unroll
        for (int u = 0; u < EMB_UNROLL; ++u) {
            const int64_t i = i0 + u * step;
            row[u] = -1;
            v[u] = make_uint4(0u, 0u, 0u, 0u);
            if (i >= total) continue;
            row[u] = sat_div(i, pieces);
            const int32_t p = (int32_t)(i - row[u] * pieces), t = __ldg(tokens + row[u]);
            col[u] = p * V;
            if (t == padding) continue;
            if ((uint32_t)t >= (uint32_t)vocabulary) {   // no such row: zeros, and the status word says so
                if (p == 0) atomicOr(status, 8);
                continue;
            }
            v[u] = row_load_raw(table + (int64_t)t * ld_table, col[u], d);
        }
#pragma unroll
        for (int u = 0; u < EMB_UNROLL; ++u) {
            if (row[u] < 0) continue;
            float f[V];
            RowVec<T>::unpack(v[u], f);
#pragma unroll
            for (int k = 0; k < V; ++k) f[k] *= scale;
            row_store(out + row[u] * ld_out, col[u], d, f);
        }
    }
}

static bool embed_vocabulary_ok(int32_t vocabulary) { return vocabulary > 0 && vocabulary < INT32_MAX; }

extern "C" sat_status sat_embed_fwd(sat_ctx *ctx, int64_t n, const int32_t *tokens, int32_t vocabulary, int32_t padding, int32_t d, int type, const void *table,
                                    int32_t ld_table, float scale, void *out, int32_t ld_out)
{
    CHECK_CTX(ctx);
    if (!ok_type(type)) return sat_fail(ctx, SAT_EINVAL, "sat_embed_fwd: unknown element type");
    if (n < 0 || n >= INT32_MAX || d <= 0 || d >= INT32_MAX - 16 || !embed_vocabulary_ok(vocabulary)) return sat_fail(ctx, SAT_EINVAL, "sat_embed_fwd: bad number of tokens, vocabulary or width");
    if (!ok_ld_of(type, ld_table, d) || !ok_ld_of(type, ld_out, d) || (n > 0 && (!tokens || !table || !out || !aligned16(table) || !aligned16(out))))
        return sat_fail(ctx, SAT_EINVAL, "sat_embed_fwd: null / misaligned tensor or bad leading dimension");
    if (n == 0) return SAT_OK;
    const int32_t v = 16 / type_bytes(type);
    const int64_t total = n * ((d + v - 1) / v);
    const unsigned blocks = (unsigned)std::min<int64_t>(cdiv64(total, 256), (int64_t)ctx->sms * 64);
    ProfScope prof(ctx, SATK_EMBED, 2.0 * type_bytes(type) * (double)n * d + 4.0 * n, 0.0);
#define ARGS(T) n, tokens, vocabulary, padding, (const T *)table, (int64_t)ld_table, d, scale, (T *)out, (int64_t)ld_out, ctx->d_flag + 1
    if (type == SAT_F32) sat_pdl(ctx->stream, k_embed<float>, blocks, 256, 0)(ARGS(float));
    else if (type == SAT_BF16) sat_pdl(ctx->stream, k_embed<__nv_bfloat16>, blocks, 256, 0)(ARGS(__nv_bfloat16));
    else sat_pdl(ctx->stream, k_embed<__half>, blocks, 256, 0)(ARGS(__half));
#undef ARGS
    SAT_LAUNCHED(ctx);
    return SAT_OK;
}

// =====================================================================================
// order of the tokens: digits of up to 11 bits from the lowest up, each pass stable
//   k_tok_count   how often every digit occurs in each tile of keys
//   k_tok_prefix  running sums over the tiles, digit by digit
//   k_tok_place   every key to its place
// Keys that pad or lie outside the vocabulary take the place of the token `vocabulary`, behind all others.
// =====================================================================================
#define TOK_TILE 2048
#define TOK_WARPS 8
#define TOK_ROUNDS (TOK_TILE / (TOK_WARPS * 32))
#define TOK_BITS 11

struct TokPass {
    const int32_t *tokens;      // first pass: the caller's tokens
    const int2 *pairs;          // later ones: {key, position} as the pass before left them
    int32_t *keys_out, *vals_out;   // last pass
    int2 *pairs_out;                // the others
    int64_t n;
    int32_t vocabulary, padding;
    int shift, bits, first;
    int32_t tiles;
    int32_t *count;             // [digits][tiles]; k_tok_prefix: running sums
    int32_t *total;             // [digits]
    int *status;
};

// {key, position} of entry i
__device__ __forceinline__ int2 tok_pair(const TokPass &p, int64_t i)
{
    if (!p.first) return __ldg(p.pairs + i);
    const int32_t t = __ldg(p.tokens + i);
    return make_int2(t == p.padding || (uint32_t)t >= (uint32_t)p.vocabulary ? p.vocabulary : t, (int32_t)i);
}

// lanes of the warp with the same digit (of `bits` bits; all lanes call)
__device__ __forceinline__ unsigned tok_same(int digit, int bits)
{
    unsigned same = 0xffffffffu;
    for (int b = 0; b <= bits; ++b) {   // one bit more: lanes without a key have it
        const bool one = (digit >> b) & 1;
        const unsigned with = __ballot_sync(0xffffffffu, one);
        same &= one ? with : ~with;
    }
    return same;
}

__global__ void __launch_bounds__(TOK_WARPS * 32)
k_tok_count(TokPass p)
{
    sat_grid_wait();
    extern __shared__ int32_t tok_smem[];
    const int digits = 1 << p.bits;
    for (int i = threadIdx.x; i < digits; i += TOK_WARPS * 32) tok_smem[i] = 0;
    __syncthreads();
    int32_t key[TOK_ROUNDS];
    bool outside = false;
#pragma unroll
    for (int r = 0; r < TOK_ROUNDS; ++r) {
        const int64_t i = (int64_t)blockIdx.x * TOK_TILE + r * (TOK_WARPS * 32) + threadIdx.x;
        key[r] = -1;
        if (i >= p.n) continue;
        if (p.first) {
            const int32_t t = __ldg(p.tokens + i);
            const bool none = (uint32_t)t >= (uint32_t)p.vocabulary;
            outside |= none && t != p.padding;
            key[r] = none || t == p.padding ? p.vocabulary : t;
        } else {
            key[r] = __ldg(p.pairs + i).x;
        }
    }
    if (outside) atomicOr(p.status, 8);
#pragma unroll
    for (int r = 0; r < TOK_ROUNDS; ++r)
        if (key[r] >= 0) atomicAdd(tok_smem + ((key[r] >> p.shift) & (digits - 1)), 1);
    __syncthreads();
    for (int i = threadIdx.x; i < digits; i += TOK_WARPS * 32) p.count[(int64_t)i * p.tiles + blockIdx.x] = tok_smem[i];
}

__global__ void __launch_bounds__(256)
k_tok_prefix(TokPass p)   // a warp per digit
{
    sat_grid_wait();
    const int lane = threadIdx.x & 31, digit = (int)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (digit >= 1 << p.bits) return;
    int32_t *c = p.count + (int64_t)digit * p.tiles;
    int32_t run = 0;
    for (int32_t b = 0; b < p.tiles; b += 32) {
        const int32_t v = b + lane < p.tiles ? c[b + lane] : 0;
        int32_t s = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t w = __shfl_up_sync(0xffffffffu, s, o);
            if (lane >= o) s += w;
        }
        if (b + lane < p.tiles) c[b + lane] = run + s - v;
        run += __shfl_sync(0xffffffffu, s, 31);
    }
    if (lane == 0) p.total[digit] = run;
}

__global__ void __launch_bounds__(TOK_WARPS * 32)
k_tok_place(TokPass p)
{
    sat_grid_wait();
    extern __shared__ int32_t tok_smem[];   // [digits] first place of the digit, [warps][digits] counts as 16-bit numbers
    __shared__ int32_t wsum[TOK_WARPS];
    const int digits = 1 << p.bits, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint16_t *mine = reinterpret_cast<uint16_t *>(tok_smem + digits) + warp * digits;
    for (int i = lane; i < digits; i += 32) mine[i] = 0;
    __syncwarp();
    // the digits that this thread has to place: how many keys have each, and how many of them lie in tiles before this one
    constexpr int PER = (1 << TOK_BITS) / (TOK_WARPS * 32);
    const int per = digits / (TOK_WARPS * 32) > 0 ? digits / (TOK_WARPS * 32) : 1, d0 = threadIdx.x * per;
    int32_t total[PER], ahead[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const bool there = i < per && d0 + i < digits;
        total[i] = there ? __ldcg(p.total + d0 + i) : 0;
        ahead[i] = there ? __ldcg(p.count + (int64_t)(d0 + i) * p.tiles + blockIdx.x) : 0;
    }
    // within the warp: keys of the same digit before this one, in this round and the rounds before
    int32_t key[TOK_ROUNDS], val[TOK_ROUNDS];
    uint16_t rank[TOK_ROUNDS];
    const int64_t base = (int64_t)blockIdx.x * TOK_TILE + warp * (TOK_ROUNDS * 32);
#pragma unroll
    for (int r = 0; r < TOK_ROUNDS; ++r) {
        const int64_t i = base + r * 32 + lane;
        const int2 pair = i < p.n ? tok_pair(p, i) : make_int2(-1, 0);
        key[r] = pair.x, val[r] = pair.y;
    }
#pragma unroll
    for (int r = 0; r < TOK_ROUNDS; ++r) {
        const int digit = key[r] < 0 ? digits : (key[r] >> p.shift) & (digits - 1);
        const unsigned same = tok_same(digit, p.bits);
        const int before = __popc(same & ((1u << lane) - 1));
        const int had = key[r] < 0 ? 0 : mine[digit];
        __syncwarp();
        if (key[r] >= 0 && before == 0) mine[digit] = (uint16_t)(had + __popc(same));
        __syncwarp();
        rank[r] = (uint16_t)(had + before);
    }
    // first place of every digit: of all keys with lower digits, then of the tiles before this one
    int32_t run = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) run += total[i];
    int32_t s = run;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int32_t w = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += w;
    }
    if (lane == 31) wsum[warp] = s;
    __syncthreads();
    s -= run;
    for (int w = 0; w < warp; ++w) s += wsum[w];
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (i < per && d0 + i < digits) {
            tok_smem[d0 + i] = s + ahead[i];
            s += total[i];
        }
    // counts of the warps before
    const uint16_t *all = reinterpret_cast<const uint16_t *>(tok_smem + digits);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < TOK_ROUNDS; ++r) {
        if (key[r] < 0) continue;
        const int digit = (key[r] >> p.shift) & (digits - 1);
        int32_t at = tok_smem[digit] + rank[r];
        for (int w = 0; w < warp; ++w) at += all[w * digits + digit];
        if ((uint32_t)at >= (uint32_t)p.n) continue;   // (only if somebody has changed the tokens meanwhile)
        if (p.pairs_out) {
            p.pairs_out[at] = make_int2(key[r], val[r]);
        } else {
            p.keys_out[at] = key[r];
            p.vals_out[at] = val[r];
        }
    }
}

// A batch of up to TOK_SMALL: one launch, a block or a cluster of up to eight, does all of it.  Keys and positions lie in the blocks' registers and change places
// through (distributed) shared memory, a pass over a digit of up to eight bits at a time; every block has the digit counts of all of them.  Order and gradient of
// 6000 positions of a vocabulary of 100000, 16 columns: 33.6 us, with the passes below 39.9; of 32000 48.2 and 49.1.
#define TOK_ROUNDS_MAX 4
#define TOK_CLUSTER 8
#define TOK_SMALL (TOK_CLUSTER * TOK_ROUNDS_MAX * 1024)
struct TokSmem {
    uint16_t cnt[256 * 32];                      // [digit][warp]
    int32_t total[TOK_CLUSTER][256];             // keys with a digit, by block
    int32_t base[256];                           // the digit's first place for keys of this block, less what lies before it in the block
    int2 pairs[TOK_ROUNDS_MAX * 1024];           // {key, position}
    int32_t wsum[32];
};
__device__ __forceinline__ uint32_t tok_remote(const void *p, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ void tok_cluster_sync() { asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// exclusive sums over the block of what its 1024 threads have
__device__ __forceinline__ int tok_scan(int v, int32_t *wsum)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int run = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int w = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += w;
    }
    if (lane == 31) wsum[warp] = run;
    __syncthreads();
    int ahead = lane < warp ? wsum[lane] : 0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ahead += __shfl_xor_sync(0xffffffffu, ahead, o);
    __syncthreads();
    return run + ahead - v;
}

__global__ void __launch_bounds__(1024)
k_tok_small(TokPass p, int all_bits, int rounds, int blocks)
{
    extern __shared__ uint4 tok_raw[];
    TokSmem &sh = *reinterpret_cast<TokSmem *>(tok_raw);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = (int)p.n, per = rounds * 1024;   // keys of a block
    uint32_t rank = 0;
    if (blocks > 1) {
        asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
        tok_cluster_sync();   // (all blocks of the cluster are there before one writes into another's memory)
    }
    sat_grid_wait();
    const int base = warp * rounds * 32, first = (int)rank * per;   // a warp's keys are side by side
    int32_t key[TOK_ROUNDS_MAX];
    uint16_t val[TOK_ROUNDS_MAX], at[TOK_ROUNDS_MAX];
    bool outside = false;
#pragma unroll
    for (int r = 0; r < TOK_ROUNDS_MAX; ++r) {
        const int i = first + base + r * 32 + lane;
        key[r] = -1;
        val[r] = (uint16_t)i;
        if (r < rounds && i < n) {
            const int32_t t = __ldg(p.tokens + i);
            const bool none = (uint32_t)t >= (uint32_t)p.vocabulary;
            outside |= none && t != p.padding;
            key[r] = none || t == p.padding ? p.vocabulary : t;
        }
    }
    if (outside) atomicOr(p.status, 8);
    const int passes = (all_bits + 7) / 8;
    for (int k = 0, shift = 0; k < passes; ++k) {
        const int bits = (all_bits - shift + passes - k - 1) / (passes - k), digits = 1 << bits;
        for (int i = threadIdx.x; i < 32 * digits; i += 1024) sh.cnt[i] = 0;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < TOK_ROUNDS_MAX; ++r) {
            if (r >= rounds) break;
            const int digit = key[r] < 0 ? digits : (key[r] >> shift) & (digits - 1);
            const unsigned same = tok_same(digit, bits);
            const int before = __popc(same & ((1u << lane) - 1));
            const int had = key[r] < 0 ? 0 : sh.cnt[digit * 32 + warp];
            __syncwarp();
            if (key[r] >= 0 && before == 0) sh.cnt[digit * 32 + warp] = (uint16_t)(had + __popc(same));
            __syncwarp();
            at[r] = (uint16_t)(had + before);
        }
        __syncthreads();
        // running sums over [digit][warp], eight counts a thread
        int sum = 0;
        uint16_t mine[8];
        const int i0 = threadIdx.x * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            mine[i] = i0 < 32 * digits ? sh.cnt[i0 + i] : 0;
            sum += mine[i];
        }
        int run = tok_scan(sum, sh.wsum);
        // four threads have a digit: its first place in the block, and how many keys have it
        const int start = __shfl_sync(0xffffffffu, run, lane & ~3), end = __shfl_sync(0xffffffffu, run + sum, lane | 3);
        if (i0 < 32 * digits) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sh.cnt[i0 + i] = (uint16_t)run;
                run += mine[i];
            }
        }
        const int d = threadIdx.x >> 2;
        if (blocks > 1) {
            if ((threadIdx.x & 3) == 0 && d < digits)
                for (int b = 0; b < blocks; ++b) asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(tok_remote(&sh.total[rank][d], b)), "r"(end - start) : "memory");
            tok_cluster_sync();
            int all = 0, before = 0;
            if ((threadIdx.x & 3) == 0 && d < digits)
                for (int b = 0; b < blocks; ++b) {
                    const int t = sh.total[b][d];
                    all += t;
                    if (b < (int)rank) before += t;
                }
            const int place = tok_scan(all, sh.wsum);
            if ((threadIdx.x & 3) == 0 && d < digits) sh.base[d] = place + before - start;
        } else if ((threadIdx.x & 3) == 0 && d < digits) {
            sh.base[d] = 0;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < TOK_ROUNDS_MAX; ++r) {
            if (key[r] < 0) continue;
            const int digit = (key[r] >> shift) & (digits - 1), to = sh.base[digit] + sh.cnt[digit * 32 + warp] + at[r];
            if (k == passes - 1) {
                p.keys_out[to] = key[r];
                p.vals_out[to] = val[r];
            } else if (blocks == 1) {
                sh.pairs[to] = make_int2(key[r], val[r]);
            } else {
                const uint32_t b = (uint32_t)to / (uint32_t)per, i = (uint32_t)to - b * per;
                asm volatile("st.shared::cluster.v2.s32 [%0], {%1, %2};" ::"r"(tok_remote(&sh.pairs[i], b)), "r"(key[r]), "r"((int)val[r]) : "memory");
            }
        }
        if (k == passes - 1) break;
        if (blocks > 1) tok_cluster_sync();
        else __syncthreads();
        shift += bits;
#pragma unroll
        for (int r = 0; r < TOK_ROUNDS_MAX; ++r) {
            const int i = base + r * 32 + lane;
            if (r < rounds && first + i < n) key[r] = sh.pairs[i].x, val[r] = (uint16_t)sh.pairs[i].y;
        }
    }
    if (blocks > 1) tok_cluster_sync();   // (nobody's memory goes while it may be written to)
}

static sat_status order_check(sat_ctx *ctx, const sat_token_order *o, const char *who)
{
    if (!o || o->n < 0 || o->n >= INT32_MAX || !embed_vocabulary_ok(o->vocabulary)) return sat_fail(ctx, SAT_EINVAL, "%s: no order of tokens, or one of bad size", who);
    if (o->n > 0 && (!o->tokens || !o->index)) return sat_fail(ctx, SAT_EINVAL, "%s: null array in the order of tokens", who);
    return SAT_OK;
}

extern "C" sat_status sat_token_sort(sat_ctx *ctx, const int32_t *tokens, int32_t padding, const sat_token_order *order)
{
    CHECK_CTX(ctx);
    SAT_TRY(order_check(ctx, order, "sat_token_sort"));
    const int64_t n = order->n;
    if (n > 0 && (!tokens || tokens == order->tokens || tokens == order->index)) return sat_fail(ctx, SAT_EINVAL, "sat_token_sort: null tokens, or in the place of their order");
    ProfScope prof(ctx, SATK_EMBED, 12.0 * (double)n, 0.0);
    if (n == 0) return SAT_OK;
    int all = 1;   // bits of the largest key, which is `vocabulary`
    while (all < 31 && (order->vocabulary >> all) != 0) ++all;
    TokPass p = {};
    p.tokens = tokens, p.n = n, p.vocabulary = order->vocabulary, p.padding = padding, p.status = ctx->d_flag + 1;
    if (n <= TOK_SMALL) {
        static PerDeviceOnce set;
        if (set.need(ctx->device)) {
            SAT_CUDA(ctx, cudaFuncSetAttribute(k_tok_small, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(TokSmem)));
            set.mark(ctx->device);
        }
        // a block takes up to two rounds of keys before there is a second one, and then as many as eight blocks leave
        const int blocks = (int)std::min<int64_t>(TOK_CLUSTER, cdiv64(n, 2048)), rounds = (int)cdiv64(n, 1024 * blocks);
        p.keys_out = order->tokens, p.vals_out = order->index;
        sat_pdl(ctx->stream, k_tok_small, (unsigned)blocks, 1024, sizeof(TokSmem), (unsigned)blocks)(p, all, rounds, blocks);
        SAT_LAUNCHED(ctx);
        return SAT_OK;
    }
    const int passes = (all + TOK_BITS - 1) / TOK_BITS;
    const int32_t tiles = (int32_t)cdiv64(n, TOK_TILE);
    const size_t counts = ((size_t)tiles + 1) << TOK_BITS;
    SAT_TRY(sat_ensure(ctx, ctx->buf_tokens, counts * sizeof(int32_t) + (passes > 2 ? 2 : passes - 1) * (size_t)n * sizeof(int2)));
    int32_t *count = (int32_t *)ctx->buf_tokens.p;
    int2 *tmp = (int2 *)(count + counts);
    p.keys_out = order->tokens, p.vals_out = order->index;
    p.tiles = tiles, p.count = count;
    for (int k = 0, shift = 0; k < passes; ++k) {
        p.shift = shift;
        p.bits = (all - shift + passes - k - 1) / (passes - k);
        shift += p.bits;
        p.total = count + ((size_t)tiles << p.bits);
        p.first = k == 0;
        p.pairs_out = k == passes - 1 ? nullptr : tmp + (k & 1) * n;
        const int digits = 1 << p.bits;
        sat_pdl(ctx->stream, k_tok_count, (unsigned)tiles, TOK_WARPS * 32, (size_t)digits * 4)(p);
        SAT_LAUNCHED(ctx);
        sat_pdl(ctx->stream, k_tok_prefix, (unsigned)cdiv64(digits, 8), 256, 0)(p);
        SAT_LAUNCHED(ctx);
        sat_pdl(ctx->stream, k_tok_place, (unsigned)tiles, TOK_WARPS * 32, (size_t)digits * (4 + 2 * TOK_WARPS))(p);
        SAT_LAUNCHED(ctx);
        p.pairs = p.pairs_out;
    }
    return SAT_OK;
}

// =====================================================================================
// gradient of the table: the sorted positions are cut into runs of `len`; TPR lanes walk one, a piece of 16 bytes of the row each
// =====================================================================================
// A token belongs to the run that it begins in.  One that crosses a single border is walked to its end by that run, the next one leaves it out.  One that
// crosses more is long: every run adds up its own part, in `part` ([run][2]: 0 where the token begins, 1 where it goes on), and k_embed_join adds these in
// order.  Further blocks write the rows of tokens that did not occur.  Bound by memory: 65536 x 1024 bf16 into 131072 rows 117 us (4.7 TB/s), 1300000 x 100 fp32 into 612257 rows
// 179 (4.8 TB/s: rows of 400 bytes at random places, fetched by 64 bytes).  Four rows on their way and four blocks an SM: no faster.
#define EMB_AHEAD 8
#define EMB_LEN 256
struct EmbedBwd {
    const int32_t *tokens, *index;
    int64_t n;
    int32_t vocabulary, d;
    int64_t ld_g, ld_gt;
    float scale;
    int accumulate;
    float *g_table, *part;
    int32_t ld_part, slabs, len;
    int64_t runs;
    int64_t walk_blocks, zero_blocks;   // blocks of the walk, and those that write zeros, each for zero_rows tokens
    int32_t zero_rows;
    int *status;
};

// the sum of a token's rows, V columns of it, to its place in the table: scaled, or scaled and added
template <int V>
__device__ __forceinline__ void embed_put(const EmbedBwd &p, int32_t token, int32_t col, const float (&f)[V])
{
    float *o = p.g_table + (int64_t)token * p.ld_gt;
#pragma unroll
    for (int i = 0; i < V; i += 4) {
        const int32_t c = col + i;
        if (c >= p.d) break;
        float v[4] = {f[i] * p.scale, f[i + 1] * p.scale, f[i + 2] * p.scale, f[i + 3] * p.scale};
        if (p.accumulate) {
            float old[4];
            row_load(o, c, p.d, old);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] += old[k];
        }
        row_store(o, c, p.d, v);
    }
}

// Zeros for the tokens [v0, v0 + zero_rows) that do not occur
#define EMB_ZERO 2048
__device__ __forceinline__ int64_t embed_find(const EmbedBwd &p, int64_t lo, int64_t hi, int64_t v)   // the first position in [lo, hi) whose token is v or more
{
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (__ldg(p.tokens + mid) < v) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}
__device__ __forceinline__ void embed_zero(const EmbedBwd &p, int64_t v0)
{
    __shared__ uint32_t there[EMB_ZERO / 32];
    __shared__ int64_t ends[2];
    const int64_t v1 = v0 + p.zero_rows < p.vocabulary ? v0 + p.zero_rows : p.vocabulary;
    const int lane = threadIdx.x & 31, rows = (int)(v1 - v0);
    if (threadIdx.x < EMB_ZERO / 32) there[threadIdx.x] = 0;
    if (threadIdx.x % 32 == 0 && threadIdx.x < 64) ends[threadIdx.x / 32] = embed_find(p, 0, p.n, threadIdx.x ? v1 : v0);
    __syncthreads();
    const int64_t p0 = ends[0], p1 = ends[1];
    if (p1 - p0 <= 8 * (int64_t)rows + 256) {   // few positions: read them all
        for (int64_t i = p0 + threadIdx.x; i < p1; i += 256) {
            const int v = (int)(__ldg(p.tokens + i) - v0);
            if ((uint32_t)v < (uint32_t)rows && (i == p0 || __ldg(p.tokens + i - 1) != v + v0)) atomicOr(there + (v >> 5), 1u << (v & 31));
        }
    } else {
        for (int v = threadIdx.x; v < rows; v += 256) {
            const int64_t at = embed_find(p, p0, p1, v0 + v);
            if (at < p1 && __ldg(p.tokens + at) == v0 + v) atomicOr(there + (v >> 5), 1u << (v & 31));
        }
    }
    __syncthreads();
    const float zero[4] = {0.f, 0.f, 0.f, 0.f};
    const int32_t quads = (p.d + 3) / 4;
    const int side = quads < 32 ? 32 / quads : 1, mine = quads < 32 ? lane / quads : 0, quad = quads < 32 ? lane % quads : lane;   // narrow rows side by side in a warp
    for (int w = threadIdx.x >> 5; w * 32 < rows; w += 8) {
        const uint32_t none = ~there[w] & (rows - w * 32 >= 32 ? 0xffffffffu : (1u << (rows - w * 32)) - 1u);
        if (none == 0) continue;
        float *o = p.g_table + (v0 + w * 32) * p.ld_gt;
        for (int r = mine; r < 32; r += side) {
            if (!((none >> r) & 1u) || mine >= side) continue;
            for (int32_t c = 4 * quad; c < p.d; c += 128) row_store(o + (int64_t)r * p.ld_gt, c, p.d, zero);
        }
    }
}

// The long tokens.  A block looks at EMB_WINDOW borders and 128 columns; a warp adds up a token of up to 32 runs, the block one of more: as many runs at a
// time as rows of 128 columns or less lie in its warps side by side, these rows' sums in order at the end.
#define EMB_WINDOW 256
__global__ void __launch_bounds__(1024)
k_embed_join(EmbedBwd p)
{
    sat_grid_wait();
    constexpr int NT = 1024;
    __shared__ int32_t list[EMB_WINDOW], heavy[EMB_WINDOW];
    __shared__ int32_t n_list, n_heavy;
    __shared__ float4 red[NT];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) n_list = n_heavy = 0;
    __syncthreads();
    const int64_t b0 = (int64_t)blockIdx.x * EMB_WINDOW + 1;
    if (threadIdx.x < EMB_WINDOW && b0 + threadIdx.x < p.runs) {
        const int64_t e = (b0 + threadIdx.x) * p.len;
        const int32_t t = __ldg(p.tokens + e), before = __ldg(p.tokens + e - 1), back = e > p.len ? __ldg(p.tokens + e - p.len - 1) : -2,
                      forth = e + p.len < p.n ? __ldg(p.tokens + e + p.len) : -2;
        // its first border, and there is another one
        if (before == t && back != t && forth == t && (uint32_t)t < (uint32_t)p.vocabulary) list[atomicAdd(&n_list, 1)] = threadIdx.x;   // (in any order: they have nothing to do with one another)
    }
    __syncthreads();
    const int32_t col0 = (int32_t)blockIdx.y * 128, width = p.d - col0 < 128 ? p.d - col0 : 128;
    auto row = [&](int64_t run, int which, int32_t col) { return __ldcg(reinterpret_cast<const float4 *>(p.part + (run * 2 + which) * p.ld_part + col)); };
    auto add = [](float4 &s, const float4 &v) { s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w; };
    for (int i = warp; i < n_list; i += NT / 32) {
        const int64_t b = b0 + list[i];
        const int32_t t = __ldg(p.tokens + b * p.len);
        const bool in = b + lane < p.runs && __ldg(p.tokens + (b + lane) * p.len) == t;
        const unsigned runs = __ballot_sync(0xffffffffu, in);   // (from the lowest bit up)
        if (runs == 0xffffffffu) {
            if (lane == 0) heavy[atomicAdd(&n_heavy, 1)] = list[i];
            continue;
        }
        if (4 * lane >= width) continue;
        float4 s = row(b - 1, 0, col0 + 4 * lane);
        const int count = __popc(runs);
#pragma unroll 4
        for (int r = 0; r < count; ++r) add(s, row(b + r, 1, col0 + 4 * lane));
        const float f[4] = {s.x, s.y, s.z, s.w};
        embed_put<4>(p, t, col0 + 4 * lane, f);
    }
    __syncthreads();
    const int quads = (width + 3) / 4, side = NT / quads, mine = threadIdx.x / quads, quad = threadIdx.x % quads;
    for (int i = 0; i < n_heavy; ++i) {
        const int64_t b = b0 + heavy[i];
        const int32_t t = __ldg(p.tokens + b * p.len);
        int64_t lo = b;   // the first run that does not begin with t
        for (int n = NT; n == NT; lo += n) {
            const int64_t r = lo + threadIdx.x;
            n = __syncthreads_count(r < p.runs && __ldg(p.tokens + (r < p.runs ? r : 0) * p.len) == t);
        }
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        if (mine < side) {
            if (mine == 0) s = row(b - 1, 0, col0 + 4 * quad);
            float4 all = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int64_t r0 = b + mine; r0 < lo; r0 += 64 * side) {   // (64 at a time: shorter chains of additions)
                const int64_t r1 = r0 + 64 * side < lo ? r0 + 64 * side : lo;
#pragma unroll 8
                for (int64_t r = r0; r < r1; r += side) add(s, row(r, 1, col0 + 4 * quad));
                add(all, s);
                s = make_float4(0.f, 0.f, 0.f, 0.f);
            }
            s = all;
        }
        red[threadIdx.x] = s;
        __syncthreads();
        int left = side;
        while (left > 1) {
            const int half = (left + 1) / 2;
            if (mine + half < left) add(red[threadIdx.x], red[threadIdx.x + half * quads]);
            __syncthreads();
            left = half;
        }
        if (mine == 0) {
            s = red[quad];
            const float f[4] = {s.x, s.y, s.z, s.w};
            embed_put<4>(p, t, col0 + 4 * quad, f);
        }
        __syncthreads();
    }
}

template <typename T, int TPR>
__global__ void __launch_bounds__(256, 3)
k_embed_bwd(EmbedBwd p, const T *__restrict__ g)
{
    sat_grid_wait();
    constexpr int V = RowVec<T>::V, GROUPS = 256 / TPR;
    const int lane = threadIdx.x & 31, t = lane % TPR;
    // blocks that walk and blocks that write zeros take turns while there are both
    int64_t block = blockIdx.x;
    {
        const int64_t both = 2 * (p.walk_blocks < p.zero_blocks ? p.walk_blocks : p.zero_blocks);
        const bool zeros = block < both ? (block & 1) != 0 : p.zero_blocks > p.walk_blocks;
        block = block < both ? block >> 1 : block - both / 2;
        if (zeros) {
            embed_zero(p, block * p.zero_rows);
            return;
        }
    }
    const unsigned mates = TPR == 32 ? 0xffffffffu : ((1u << (TPR & 31)) - 1u) << (lane - t);
    const int64_t item = block * GROUPS + threadIdx.x / TPR;   // neighbouring groups: the slabs of a run
    const int64_t run = sat_div(item, p.slabs);
    if (run >= p.runs) return;
    const int32_t col = ((int32_t)(item - run * p.slabs) * TPR + t) * V;
    const int64_t e0 = run * p.len, e1 = e0 + p.len < p.n ? e0 + p.len : p.n;
    // (all that is to be known of the borders is asked for at once; -2: no such position)
    auto token = [&](int64_t e) { return e >= 0 && e < p.n ? __ldg(p.tokens + e) : -2; };
    const int32_t first = token(e0), last = token(e1 - 1), before = token(e0 - 1), behind = token(e1), back = token(e0 - p.len - 1), forth = token(e1 + p.len);
    const bool goes_on = before == first, leaves = behind == last;
    // a token that crosses another border than this one is long
    const bool first_long = goes_on && (back == first || behind == first), last_long = leaves && (before == last || forth == last);
    const int64_t end = leaves && !last_long ? (e1 + p.len < p.n ? e1 + p.len : p.n) : e1;   // (the token ends before that)
    const bool skip = goes_on && !first_long;
    float acc[V] = {};
    int32_t cur = first;
    bool begun_here = !goes_on;
    auto put = [&](bool is_last) {   // the sum of `cur`
        if ((uint32_t)cur >= (uint32_t)p.vocabulary || col >= p.d || (!begun_here && skip)) return;
        if (!begun_here || (is_last && last_long)) {
            float *o = p.part + (run * 2 + (begun_here ? 0 : 1)) * p.ld_part + col;
#pragma unroll
            for (int i = 0; i < V; i += 4) *reinterpret_cast<float4 *>(o + i) = make_float4(acc[i], acc[i + 1], acc[i + 2], acc[i + 3]);
        } else {
            embed_put<V>(p, cur, col, acc);
        }
    };
    // Eight rows are on their way at any time.  The lanes hold eight entries each of three batches: the tokens of the one that is added up, the positions of the
    // one whose rows are asked for in their place one by one, and the one behind that.  What is to be known of an entry is worked out by its lane: where its row
    // is (none: -1), whether another token begins with it, whether the walk ends before it.
    const int slot = lane % EMB_AHEAD;
    uint4 raw[EMB_AHEAD];
    const T *gc = g + col;
    const bool inside = col < p.d;
    auto entries = [&](int64_t e, int32_t &tok, int32_t &idx) {
        tok = e + slot < p.n ? __ldg(p.tokens + e + slot) : -1;   // (asked for without waiting for the borders' tokens)
        idx = e + slot < p.n ? __ldg(p.index + e + slot) : -1;
        if (e + slot >= end || (e + slot >= e1 && tok != last)) tok = -1;   // behind what this run walks
        if ((uint32_t)tok >= (uint32_t)p.vocabulary || (skip && tok == first)) {
            idx = -1;
        } else if ((uint32_t)idx >= (uint32_t)p.n) {   // (the arrays are the caller's)
            atomicOr(p.status, 8);
            idx = -1;
        }
    };
    auto fetch = [&](int32_t i) { return i >= 0 && inside ? *reinterpret_cast<const uint4 *>(gc + (int64_t)i * p.ld_g) : make_uint4(0u, 0u, 0u, 0u); };
    int32_t tok0, tok1, idx1;
    {
        int32_t idx0;
        entries(e0, tok0, idx0);
        entries(e0 + EMB_AHEAD, tok1, idx1);
#pragma unroll
        for (int u = 0; u < EMB_AHEAD; ++u) raw[u] = fetch(__shfl_sync(mates, idx0, u, EMB_AHEAD));
    }
    for (int64_t e = e0; e < end; e += EMB_AHEAD) {
        int32_t tok2, idx2;
        entries(e + 2 * EMB_AHEAD, tok2, idx2);
        int32_t left = __shfl_up_sync(mates, tok0, 1, EMB_AHEAD);
        if (slot == 0) left = cur;
        const unsigned other = __ballot_sync(mates, tok0 != left) >> (lane & ~(EMB_AHEAD - 1)), none = __ballot_sync(mates, tok0 == -1) >> (lane & ~(EMB_AHEAD - 1));
        const int count = __ffs((none & ((1u << EMB_AHEAD) - 1u)) | (1u << EMB_AHEAD)) - 1;
#pragma unroll
        for (int u = 0; u < EMB_AHEAD; ++u) {
            const uint4 now = raw[u];
            raw[u] = fetch(__shfl_sync(mates, idx1, u, EMB_AHEAD));
            if (u >= count) continue;
            if ((other >> u) & 1u) {
                put(false);
                cur = __shfl_sync(mates, tok0, u, EMB_AHEAD);
                begun_here = true;
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] = 0.f;
            }
            float f[V];
            RowVec<T>::unpack(now, f);
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] += f[i];
        }
        if (count < EMB_AHEAD) break;
        tok0 = tok1, tok1 = tok2, idx1 = idx2;
    }
    put(true);
}

template <typename T>
static void embed_bwd_launch(sat_ctx *ctx, EmbedBwd &p, int tpr, const void *g)
{
    p.walk_blocks = cdiv64(p.runs * p.slabs, 256 / tpr);
    p.zero_blocks = p.accumulate ? 0 : cdiv64(p.vocabulary, p.zero_rows);
    const unsigned blocks = (unsigned)(p.walk_blocks + p.zero_blocks);
    if (tpr == 8) sat_pdl(ctx->stream, k_embed_bwd<T, 8>, blocks, 256, 0)(p, (const T *)g);
    else if (tpr == 16) sat_pdl(ctx->stream, k_embed_bwd<T, 16>, blocks, 256, 0)(p, (const T *)g);
    else sat_pdl(ctx->stream, k_embed_bwd<T, 32>, blocks, 256, 0)(p, (const T *)g);
}

extern "C" sat_status sat_embed_bwd(sat_ctx *ctx, const sat_token_order *order, int32_t d, int type, const void *g, int32_t ld_g, float scale, float *g_table,
                                    int32_t ld_gt, int accumulate)
{
    CHECK_CTX(ctx);
    SAT_TRY(order_check(ctx, order, "sat_embed_bwd"));
    if (!ok_type(type)) return sat_fail(ctx, SAT_EINVAL, "sat_embed_bwd: unknown element type");
    if (d <= 0 || d > 65535 * 128 || !ok_ld_of(type, ld_g, d) || !ok_ld(ld_gt, d) || !g_table || !aligned16(g_table) || (order->n > 0 && (!g || !aligned16(g))))
        return sat_fail(ctx, SAT_EINVAL, "sat_embed_bwd: null / misaligned tensor, bad width or leading dimension");
    if (accumulate != 0 && accumulate != 1) return sat_fail(ctx, SAT_EINVAL, "sat_embed_bwd: accumulate is 0 or 1");
    EmbedBwd p = {};
    p.tokens = order->tokens, p.index = order->index, p.n = order->n, p.vocabulary = order->vocabulary, p.d = d, p.ld_g = ld_g, p.ld_gt = ld_gt;
    p.scale = scale, p.accumulate = accumulate, p.g_table = g_table, p.ld_part = (d + 7) & ~7;
    p.status = ctx->d_flag + 1;
    if (p.n == 0 && accumulate) return SAT_OK;
    // lanes of a row: as many as it has pieces of 16 bytes; runs: as many as fill the SMs four times with the 24 warps that they hold, of 8 positions at least and EMB_LEN at most (a run's sum
    // is additions one after the other)
    const int32_t v = 16 / type_bytes(type), pieces = (d + v - 1) / v;
    const int tpr = pieces <= 8 ? 8 : pieces <= 16 ? 16 : 32;
    p.slabs = (pieces + tpr - 1) / tpr;
    p.len = (int32_t)std::min<int64_t>(EMB_LEN, std::max<int64_t>(8, cdiv64(p.n * p.slabs, (int64_t)ctx->sms * 96 * (32 / tpr))));
    p.zero_rows = (int32_t)std::min<int64_t>(EMB_ZERO, std::max<int64_t>(32, cdiv64(order->vocabulary, ctx->sms * 3)));
    p.runs = cdiv64(p.n, p.len);
    if (p.runs * p.slabs >= INT32_MAX) return sat_fail(ctx, SAT_EINVAL, "sat_embed_bwd: too many rows of this width");
    if (p.runs > 2) {   // (a long token crosses two borders)
        SAT_TRY(sat_ensure(ctx, ctx->buf_embed, (size_t)p.runs * 2 * p.ld_part * sizeof(float)));
        p.part = (float *)ctx->buf_embed.p;
    }
    ProfScope prof(ctx, SATK_EMBED, (double)type_bytes(type) * p.n * d + 4.0 * (double)order->vocabulary * d, (double)p.n * d);
    if (type == SAT_F32) embed_bwd_launch<float>(ctx, p, tpr, g);
    else if (type == SAT_BF16) embed_bwd_launch<__nv_bfloat16>(ctx, p, tpr, g);
    else embed_bwd_launch<__half>(ctx, p, tpr, g);
    SAT_LAUNCHED(ctx);
    if (p.runs > 2) {
        sat_pdl(ctx->stream, k_embed_join, dim3((unsigned)cdiv64(p.runs - 1, EMB_WINDOW), (unsigned)cdiv64(d, 128)), 1024, 0)(p);
        SAT_LAUNCHED(ctx);
    }
    return SAT_OK;
}

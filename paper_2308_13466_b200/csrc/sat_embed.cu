// Embedding lookup with scaling, and its gradient by sorted tokens:
//     out[i] = scale table[t_i]            g_table[v] (+)= scale sum of g[i] over the i with t_i = v, in ascending order of i
// The tokens are sorted once (sat_token_sort: keys of 32 bits, by digits, stable), the gradient then walks them in that order.
#include "sat_rows.h"

#include <algorithm>

// =====================================================================================
// lookup: a thread per 16 bytes of a row, bound by memory
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
//   k_tok_count   how often every digit occurs in each tile of keys, and (first pass) which tokens occur at all
//   k_tok_prefix  running sums over the tiles, digit by digit
//   k_tok_place   every key to its place
// Keys that pad or lie outside the vocabulary take the place of the token `vocabulary`, behind all others.
// =====================================================================================
#define TOK_TILE 4096
#define TOK_WARPS 8
#define TOK_ROUNDS (TOK_TILE / (TOK_WARPS * 32))
#define TOK_BITS 11

struct TokPass {
    const int32_t *tokens;      // first pass: the caller's tokens
    const int32_t *keys, *vals; // later ones: what the pass before left
    int32_t *keys_out, *vals_out;
    int64_t n;
    int32_t vocabulary, padding;
    int shift, bits, first, last;
    int32_t tiles;
    int32_t *count;             // [digits][tiles]; k_tok_prefix: running sums
    int32_t *total;             // [digits]
    uint8_t *seen;              // [vocabulary]
    int *status;
};

__device__ __forceinline__ int32_t tok_key(const TokPass &p, int64_t i)
{
    if (!p.first) return __ldg(p.keys + i);
    const int32_t t = __ldg(p.tokens + i);
    return t == p.padding || (uint32_t)t >= (uint32_t)p.vocabulary ? p.vocabulary : t;
}

__global__ void __launch_bounds__(TOK_WARPS * 32)
k_tok_count(TokPass p)
{
    sat_grid_wait();
    extern __shared__ int32_t tok_smem[];
    const int digits = 1 << p.bits;
    for (int i = threadIdx.x; i < digits; i += TOK_WARPS * 32) tok_smem[i] = 0;
    __syncthreads();
    if (p.first) {   // no token has been seen
        const int64_t per = ((int64_t)p.vocabulary + p.tiles - 1) / p.tiles, lo = per * blockIdx.x, hi = lo + per < p.vocabulary ? lo + per : p.vocabulary;
        for (int64_t i = lo + threadIdx.x; i < hi; i += TOK_WARPS * 32) p.seen[i] = 0;
    }
    for (int u = threadIdx.x; u < TOK_TILE; u += TOK_WARPS * 32) {
        const int64_t i = (int64_t)blockIdx.x * TOK_TILE + u;
        if (i >= p.n) break;
        if (p.first) {
            const int32_t t = p.tokens[i];
            if (t != p.padding && (uint32_t)t >= (uint32_t)p.vocabulary) atomicOr(p.status, 8);
        }
        atomicAdd(tok_smem + ((tok_key(p, i) >> p.shift) & (digits - 1)), 1);
    }
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
    // within the warp: keys of the same digit before this one, in this round and the rounds before
    int32_t key[TOK_ROUNDS];
    uint16_t rank[TOK_ROUNDS];
    const int64_t base = (int64_t)blockIdx.x * TOK_TILE + warp * (TOK_ROUNDS * 32);
#pragma unroll
    for (int r = 0; r < TOK_ROUNDS; ++r) {
        const int64_t i = base + r * 32 + lane;
        key[r] = i < p.n ? tok_key(p, i) : -1;
    }
#pragma unroll
    for (int r = 0; r < TOK_ROUNDS; ++r) {
        const int digit = key[r] < 0 ? -1 : (key[r] >> p.shift) & (digits - 1);
        const unsigned same = __match_any_sync(0xffffffffu, digit);
        const int before = __popc(same & ((1u << lane) - 1));
        const int had = digit < 0 ? 0 : mine[digit];
        __syncwarp();
        if (digit >= 0 && before == 0) mine[digit] = (uint16_t)(had + __popc(same));
        __syncwarp();
        rank[r] = (uint16_t)(had + before);
        if (p.last) {   // (one lane for several of a kind, where they are side by side)
            const int32_t left = __shfl_up_sync(0xffffffffu, key[r], 1);
            if ((lane == 0 || left != key[r]) && (uint32_t)key[r] < (uint32_t)p.vocabulary) p.seen[key[r]] = 1;
        }
    }
    // first place of every digit: of all keys with lower digits, then of the tiles before this one
    int32_t run = 0;
    const int per = digits / (TOK_WARPS * 32) > 0 ? digits / (TOK_WARPS * 32) : 1, d0 = threadIdx.x * per;
    for (int i = 0; i < per; ++i) run += d0 + i < digits ? p.total[d0 + i] : 0;
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
    for (int i = 0; i < per; ++i)
        if (d0 + i < digits) {
            tok_smem[d0 + i] = s + p.count[(int64_t)(d0 + i) * p.tiles + blockIdx.x];
            s += p.total[d0 + i];
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
        p.keys_out[at] = key[r];
        p.vals_out[at] = p.first ? (int32_t)(base + r * 32 + lane) : __ldg(p.vals + base + r * 32 + lane);
    }
}

static sat_status order_check(sat_ctx *ctx, const sat_token_order *o, const char *who)
{
    if (!o || o->n < 0 || o->n >= INT32_MAX || !embed_vocabulary_ok(o->vocabulary)) return sat_fail(ctx, SAT_EINVAL, "%s: no order of tokens, or one of bad size", who);
    if (!o->seen || (o->n > 0 && (!o->tokens || !o->index))) return sat_fail(ctx, SAT_EINVAL, "%s: null array in the order of tokens", who);
    return SAT_OK;
}

extern "C" sat_status sat_token_sort(sat_ctx *ctx, const int32_t *tokens, int32_t padding, const sat_token_order *order)
{
    CHECK_CTX(ctx);
    SAT_TRY(order_check(ctx, order, "sat_token_sort"));
    const int64_t n = order->n;
    if (n > 0 && !tokens) return sat_fail(ctx, SAT_EINVAL, "sat_token_sort: null tokens");
    ProfScope prof(ctx, SATK_EMBED, 12.0 * (double)n, 0.0);
    if (n == 0) {
        SAT_CUDA(ctx, cudaMemsetAsync(order->seen, 0, (size_t)order->vocabulary, ctx->stream));
        return SAT_OK;
    }
    int all = 1;   // bits of the largest key, which is `vocabulary`
    while (all < 31 && (order->vocabulary >> all) != 0) ++all;
    const int passes = (all + TOK_BITS - 1) / TOK_BITS;
    const int32_t tiles = (int32_t)cdiv64(n, TOK_TILE);
    const size_t counts = ((size_t)tiles + 1) << TOK_BITS;
    SAT_TRY(sat_ensure(ctx, ctx->buf_tokens, (counts + (passes > 1 ? 2 * (size_t)n : 0)) * sizeof(int32_t)));
    int32_t *count = (int32_t *)ctx->buf_tokens.p, *tmp = count + counts;
    TokPass p = {};
    p.tokens = tokens, p.n = n, p.vocabulary = order->vocabulary, p.padding = padding, p.tiles = tiles, p.count = count, p.seen = order->seen;
    p.status = ctx->d_flag + 1;
    for (int k = 0, shift = 0; k < passes; ++k) {
        p.shift = shift;
        p.bits = (all - shift + passes - k - 1) / (passes - k);
        shift += p.bits;
        p.total = count + ((size_t)tiles << p.bits);
        p.first = k == 0, p.last = k == passes - 1;
        const bool to_tmp = ((passes - 1 - k) & 1) != 0;   // the last pass ends in the caller's arrays
        p.keys_out = to_tmp ? tmp : order->tokens, p.vals_out = to_tmp ? tmp + n : order->index;
        const int digits = 1 << p.bits;
        sat_pdl(ctx->stream, k_tok_count, (unsigned)tiles, TOK_WARPS * 32, (size_t)digits * 4)(p);
        SAT_LAUNCHED(ctx);
        sat_pdl(ctx->stream, k_tok_prefix, (unsigned)cdiv64(digits, 8), 256, 0)(p);
        SAT_LAUNCHED(ctx);
        sat_pdl(ctx->stream, k_tok_place, (unsigned)tiles, TOK_WARPS * 32, (size_t)digits * (4 + 2 * TOK_WARPS))(p);
        SAT_LAUNCHED(ctx);
        p.keys = p.keys_out, p.vals = p.vals_out;
    }
    return SAT_OK;
}

// =====================================================================================
// gradient of the table: the sorted positions are cut into runs of EMB_RUN; TPR lanes walk one, a piece of 16 bytes of the row each
// =====================================================================================
// A token whose positions lie in one run has its sum written at once; the sums of one that crosses runs go to `part` ([run][2]: 0 where it begins, 1 where
// it goes on), and k_embed_join adds these up in order.  Further blocks write the rows of tokens that did not occur.
#define EMB_RUN 32
#define EMB_AHEAD 8
struct EmbedBwd {
    const int32_t *tokens, *index;
    const uint8_t *seen;
    int64_t n;
    int32_t vocabulary, d;
    int64_t ld_g, ld_gt;
    float scale;
    int accumulate;
    float *g_table, *part;
    int32_t ld_part, slabs;
    int64_t runs;
    int64_t walk_blocks;   // blocks of the walk; the others write zeros
    int *status;
};

template <typename T>
__device__ __forceinline__ void embed_put(const EmbedBwd &p, int32_t token, int32_t col, const float (&f)[RowVec<T>::V])
{
    float *o = p.g_table + (int64_t)token * p.ld_gt;
#pragma unroll
    for (int i = 0; i < RowVec<T>::V; i += 4) {
        const int32_t c = col + i;
        if (c >= p.d) break;
        float v[4];
        const bool whole = c + 4 <= p.d;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = f[i + k] * p.scale;
        if (p.accumulate) {
            if (whole) {
                const float4 old = *reinterpret_cast<const float4 *>(o + c);
                v[0] += old.x, v[1] += old.y, v[2] += old.z, v[3] += old.w;
            } else {
                for (int k = 0; k < 3; ++k)
                    if (c + k < p.d) v[k] += o[c + k];
            }
        }
        row_store(o, c, p.d, v);
    }
}

template <typename T, int TPR>
__global__ void __launch_bounds__(256)
k_embed_bwd(EmbedBwd p, const T *__restrict__ g)
{
    sat_grid_wait();
    constexpr int V = RowVec<T>::V, GROUPS = 256 / TPR;
    if ((int64_t)blockIdx.x >= p.walk_blocks) {   // 32 tokens a warp
        const int lane = threadIdx.x & 31;
        const int64_t v0 = (((int64_t)blockIdx.x - p.walk_blocks) * 8 + (threadIdx.x >> 5)) * 32;
        unsigned none = __ballot_sync(0xffffffffu, v0 + lane < p.vocabulary && p.seen[v0 + lane < p.vocabulary ? v0 + lane : 0] == 0);
        const float zero[4] = {0.f, 0.f, 0.f, 0.f};
        while (none) {
            const int64_t v = v0 + __ffs(none) - 1;
            none &= none - 1;
            for (int32_t c = 4 * lane; c < p.d; c += 128) row_store(p.g_table + v * p.ld_gt, c, p.d, zero);
        }
        return;
    }
    const int64_t item = (int64_t)blockIdx.x * GROUPS + threadIdx.x / TPR;   // neighbouring groups: the slabs of a run
    const int64_t run = sat_div(item, p.slabs);
    if (run >= p.runs) return;
    const int32_t col = ((int32_t)(item - run * p.slabs) * TPR + threadIdx.x % TPR) * V;
    const int64_t e0 = run * EMB_RUN, e1 = e0 + EMB_RUN < p.n ? e0 + EMB_RUN : p.n;
    int32_t cur = __ldg(p.tokens + e0);
    bool goes_on = e0 > 0 && __ldg(p.tokens + e0 - 1) == cur;   // from the run before
    float acc[V] = {};
    float *part = p.part + run * 2 * p.ld_part + col;
    for (int64_t e = e0; e < e1; e += EMB_AHEAD) {
        uint4 raw[EMB_AHEAD];
        int32_t tok[EMB_AHEAD];
#pragma unroll
        for (int u = 0; u < EMB_AHEAD; ++u) {
            tok[u] = e + u < e1 ? __ldg(p.tokens + e + u) : -1;
            const int32_t i = e + u < e1 ? __ldg(p.index + e + u) : 0;
            const bool known = (uint32_t)tok[u] < (uint32_t)p.vocabulary, there = (uint32_t)i < (uint32_t)p.n;   // (the arrays are the caller's)
            if (known && !there) atomicOr(p.status, 8);
            raw[u] = known && there ? row_load_raw(g + (int64_t)i * p.ld_g, col, p.d) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int u = 0; u < EMB_AHEAD; ++u) {
            if (e + u >= e1) break;
            if (tok[u] != cur) {
                if ((uint32_t)cur < (uint32_t)p.vocabulary && col < p.d) {
                    if (goes_on) {
#pragma unroll
                        for (int i = 0; i < V; i += 4) *reinterpret_cast<float4 *>(part + p.ld_part + i) = make_float4(acc[i], acc[i + 1], acc[i + 2], acc[i + 3]);
                    } else {
                        embed_put<T>(p, cur, col, acc);
                    }
                }
                cur = tok[u];
                goes_on = false;
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] = 0.f;
            }
            float f[V];
            RowVec<T>::unpack(raw[u], f);
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] += f[i];
        }
    }
    if ((uint32_t)cur >= (uint32_t)p.vocabulary || col >= p.d) return;
    if (goes_on || (e1 < p.n && __ldg(p.tokens + e1) == cur)) {
        float *o = part + (goes_on ? p.ld_part : 0);
#pragma unroll
        for (int i = 0; i < V; i += 4) *reinterpret_cast<float4 *>(o + i) = make_float4(acc[i], acc[i + 1], acc[i + 2], acc[i + 3]);
    } else {
        embed_put<T>(p, cur, col, acc);
    }
}

// A block per border between two runs and 128 columns: where a token crosses the border and begins in the run before it, its sums are added up, eight warps
// taking every eighth run.
__global__ void __launch_bounds__(256)
k_embed_join(EmbedBwd p)
{
    sat_grid_wait();
    __shared__ float4 red[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t b = (int64_t)blockIdx.x;                       // border between runs b and b + 1
    const int64_t at = (b + 1) * EMB_RUN;
    const int32_t t = __ldg(p.tokens + at);
    if (__ldg(p.tokens + at - 1) != t || (uint32_t)t >= (uint32_t)p.vocabulary) return;
    if (__ldg(p.tokens + b * EMB_RUN) == t && b > 0 && __ldg(p.tokens + b * EMB_RUN - 1) == t) return;   // it began earlier
    const int32_t col = (int32_t)blockIdx.y * 128 + 4 * lane;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (col < p.d) {
        if (warp == 0) s = __ldcg(reinterpret_cast<const float4 *>(p.part + b * 2 * p.ld_part + col));
        for (int64_t r = b + 1 + warp; r < p.runs && __ldg(p.tokens + r * EMB_RUN) == t; r += 8) {
            const float4 v = __ldcg(reinterpret_cast<const float4 *>(p.part + (r * 2 + 1) * p.ld_part + col));
            s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
        }
    }
    red[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && col < p.d) {
        for (int w = 1; w < 8; ++w) s.x += red[w][lane].x, s.y += red[w][lane].y, s.z += red[w][lane].z, s.w += red[w][lane].w;
        const float f[4] = {s.x, s.y, s.z, s.w};
        embed_put<float>(p, t, col, f);
    }
}

template <typename T>
static void embed_bwd_launch(sat_ctx *ctx, EmbedBwd &p, const void *g)
{
    constexpr int V = RowVec<T>::V;
    const int32_t pieces = (p.d + V - 1) / V;
    const int tpr = pieces <= 8 ? 8 : pieces <= 16 ? 16 : 32;
    p.slabs = (pieces + tpr - 1) / tpr;
    p.walk_blocks = cdiv64(p.runs * p.slabs, 256 / tpr);
    const unsigned blocks = (unsigned)(p.walk_blocks + (p.accumulate ? 0 : cdiv64(p.vocabulary, 256)));
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
    p.tokens = order->tokens, p.index = order->index, p.seen = order->seen, p.n = order->n, p.vocabulary = order->vocabulary, p.d = d, p.ld_g = ld_g, p.ld_gt = ld_gt;
    p.scale = scale, p.accumulate = accumulate, p.g_table = g_table, p.runs = cdiv64(order->n, EMB_RUN), p.ld_part = (d + 7) & ~7;
    p.status = ctx->d_flag + 1;
    if (p.n == 0 && accumulate) return SAT_OK;
    if (p.runs * cdiv64(d, 32) >= INT32_MAX) return sat_fail(ctx, SAT_EINVAL, "sat_embed_bwd: too many rows of this width");
    if (p.runs > 1) {
        SAT_TRY(sat_ensure(ctx, ctx->buf_embed, (size_t)p.runs * 2 * p.ld_part * sizeof(float)));
        p.part = (float *)ctx->buf_embed.p;
    }
    ProfScope prof(ctx, SATK_EMBED, (double)type_bytes(type) * p.n * d + 4.0 * (double)order->vocabulary * d, (double)p.n * d);
    if (type == SAT_F32) embed_bwd_launch<float>(ctx, p, g);
    else if (type == SAT_BF16) embed_bwd_launch<__nv_bfloat16>(ctx, p, g);
    else embed_bwd_launch<__half>(ctx, p, g);
    SAT_LAUNCHED(ctx);
    if (p.runs > 1) {
        sat_pdl(ctx->stream, k_embed_join, dim3((unsigned)(p.runs - 1), (unsigned)cdiv64(d, 128)), 256, 0)(p);
        SAT_LAUNCHED(ctx);
    }
    return SAT_OK;
}

// C entry points of the paged 4-bit key/value cache (declared in include/ivf.h):
// argument checks and launches. No call synchronises with the host.
#include <hip/hip_runtime.h>

#include <math.h>

#include <algorithm>

#include "ctx.h"
#include "ivf.h"
#include "kv.h"

using namespace ivf;

namespace {

int block_shift(int32_t bs) { return bs == 16 ? 4 : bs == 32 ? 5 : bs == 64 ? 6 : bs == 128 ? 7 : 0; }

bool kv_dim(int32_t d) { return d == 64 || d == 96 || d == 128 || d == 192 || d == 256; }

ivf_status check_cache(ivf_ctx *ctx, const ivf_kv_cache *c, KvCache &k)
{
    if (!c) return fail(ctx, IVF_EINVAL, "null cache");
    if (!block_shift(c->block_size))
        return fail(ctx, IVF_EUNSUPPORTED, "block_size must be 16, 32, 64 or 128 (got %d)", c->block_size);
    if (!kv_dim(c->dim)) return fail(ctx, IVF_EUNSUPPORTED, "dim must be 64, 96, 128, 192 or 256 (got %d)", c->dim);
    if (c->dtype != IVF_F16 && c->dtype != IVF_BF16)
        return fail(ctx, IVF_EUNSUPPORTED, "the cache's type must be IVF_F16 or IVF_BF16 (got %d)", c->dtype);
    if (c->heads < 1 || c->heads > 4096) return fail(ctx, IVF_EINVAL, "heads must be in [1, 4096] (got %d)", c->heads);
    if (c->blocks < 1 || c->blocks > INT32_MAX)
        return fail(ctx, IVF_EINVAL, "blocks must be in [1, 2^31) (got %lld)", (long long)c->blocks);
    if (!c->records || !c->summary || !c->weight) return fail(ctx, IVF_EINVAL, "null pointer in the cache");
    if (!aligned16(c->records) || !aligned16(c->summary) || !aligned16(c->weight))
        return fail(ctx, IVF_EINVAL, "the cache's arrays must be 16-byte aligned");
    k.rec = (uint8_t *)c->records;
    k.summary = c->summary;
    k.weight = c->weight;
    k.blocks = c->blocks;
    k.bs = c->block_size;
    k.shift = block_shift(c->block_size);
    k.heads = c->heads;
    k.dim = c->dim;
    k.bf16 = c->dtype == IVF_BF16;
    return IVF_OK;
}

bool overlaps_cache(const KvCache &c, const void *p, size_t n)
{
    const size_t bh = (size_t)c.blocks * c.heads;
    return overlap(p, n, c.rec, bh * c.rec_bytes()) || overlap(p, n, c.summary, bh * c.dim) ||
           overlap(p, n, c.weight, bh * 4);
}

// Rows [T][heads][dim] of 16-bit elements by strides; *bytes: from the first to
// past the last.
ivf_status check_rows(ivf_ctx *ctx, const char *name, const void *p, int64_t ts, int64_t hs, int64_t T, int64_t heads,
                      int dim, size_t *bytes)
{
    if (!p) return fail(ctx, IVF_EINVAL, "null pointer argument: %s", name);
    if (!aligned16(p)) return fail(ctx, IVF_EINVAL, "%s must be 16-byte aligned", name);
    if (ts < 0 || hs < 0 || ts % 8 || hs % 8 || ts > INT32_MAX || hs > INT32_MAX)
        return fail(ctx, IVF_EINVAL, "%s: strides must be multiples of 8 elements in [0, 2^31)", name);
    *bytes = ((size_t)(T - 1) * ts + (size_t)(heads - 1) * hs + dim) * 2;
    return IVF_OK;
}

ivf_status check_tokens(ivf_ctx *ctx, const KvCache &c, int64_t T, int64_t heads)
{
    if (T < 0) return fail(ctx, IVF_EINVAL, "T must be >= 0");
    if (T > INT32_MAX || T * heads > INT32_MAX)
        return fail(ctx, IVF_EUNSUPPORTED, "too many tokens for one call");
    return IVF_OK;
}

ivf_status check_table(ivf_ctx *ctx, int64_t B, int32_t cols, int shift)
{
    if (B < 1 || B > INT32_MAX) return fail(ctx, IVF_EINVAL, "B must be in [1, 2^31)");
    if (cols < 1 || ((int64_t)cols << shift) > INT32_MAX)
        return fail(ctx, IVF_EINVAL, "table_cols * block_size must be in [1, 2^31)");
    return IVF_OK;
}

// The sizes of an attention call, and how it is carried out (T above 0).
ivf_status plan_attend(ivf_ctx *ctx, const KvCache &c, int32_t q_heads, int64_t T, int64_t B, int32_t cols, int32_t count,
                       int64_t longest, int num_cus, KvAttendPlan &p)
{
    if (q_heads < 1 || q_heads > 65536 || q_heads % c.heads)
        return fail(ctx, IVF_EINVAL, "q_heads must be a multiple of the cache's heads (got %d, %d)", q_heads, c.heads);
    ivf_status st = check_tokens(ctx, c, T, q_heads);
    if (st != IVF_OK || T == 0) return st;
    if ((st = check_table(ctx, B, cols, c.shift)) != IVF_OK) return st;
    if (count < 0 || count > kKvMaxCount)
        return fail(ctx, IVF_EINVAL, "count must be in [1, %d] with blocks, 0 without", kKvMaxCount);
    if (longest < 1) return fail(ctx, IVF_EINVAL, "longest must be >= 1");
    const int group = q_heads / c.heads;
    p = kv_attend_plan(c, group, T, B, cols, count, std::min(longest, T), num_cus);
    const int64_t tiles = (T * group + kv_prompt_rows(c.dim) - 1) / kv_prompt_rows(c.dim);
    if (p.units * 16 * c.heads > INT32_MAX) return fail(ctx, IVF_EUNSUPPORTED, "too many rows for one call");
    // a team of one: four units a workgroup
    if ((st = check_threads(ctx, (p.token_groups + 3) * c.heads * 64 * p.team)) != IVF_OK) return st;
    return check_threads(ctx, tiles * p.prompt_splits * c.heads * 512);
}

// The attention calls. terms: null, or what goes into the scores.
ivf_status attend(ivf_ctx *ctx, const ivf_kv_cache *cache, const void *q, int64_t q_token_stride, int64_t q_head_stride,
                  int32_t q_heads, int64_t T, const int32_t *start, const int32_t *request, const int32_t *position,
                  const int32_t *table, int64_t B, int32_t table_cols, const int32_t *blocks, int32_t count, float scale,
                  int64_t longest, const ivf_kv_terms *terms, void *out, float *out_lse)
{
    return guarded(ctx, "kv_attend", [&]() -> ivf_status {
        KvAttend a;
        ivf_status st = check_cache(ctx, cache, a.c);
        if (st != IVF_OK) return st;
        KvAttendPlan p = {};
        if ((st = plan_attend(ctx, a.c, q_heads, T, B, table_cols, count, longest, ctx->num_cus, p)) != IVF_OK) return st;
        if (T == 0) return IVF_OK;
        if (blocks ? count < 1 : count != 0)
            return fail(ctx, IVF_EINVAL, "count must be in [1, %d] with blocks, 0 without", kKvMaxCount);
        const float scale2 = fabsf(scale) * 1.44269504089f;  // of exponents to the base 2
        if (!isfinite(scale2)) return fail(ctx, IVF_EINVAL, "scale must be finite, and of magnitude below 2.3e38");
        const ivf_kv_terms none = {}, &given = terms ? *terms : none;
        KvTerms x = {given.cap, {}, given.slopes, given.first, given.prefix};
        if (x.cap != 0.f) {
            if (!(x.cap >= 0x1p-40f && x.cap <= 0x1p40f)) return fail(ctx, IVF_EINVAL, "cap must be 0, or from 2^-40 to 2^40");
            const float by_cap = fabsf(scale) / x.cap;
            if (!isfinite(by_cap) || (by_cap < 0x1p-126f && scale != 0.f))
                return fail(ctx, IVF_EINVAL, "scale / cap must be 0 or a normal number");
        }
        size_t qb;
        if ((st = check_rows(ctx, "q", q, q_token_stride, q_head_stride, T, q_heads, a.c.dim, &qb)) != IVF_OK) return st;
        if (!position || !table || !out || (blocks ? !request : !start)) return fail(ctx, IVF_EINVAL, "null pointer argument");
        const void *i32[] = {start, request, position, table, blocks, out_lse, x.slopes, x.first, x.prefix};
        if ((st = check_elements(ctx, i32, 4)) != IVF_OK) return st;
        if (!aligned16(out)) return fail(ctx, IVF_EINVAL, "out must be 16-byte aligned");
        const size_t rows = (size_t)T * q_heads;
        const Span ins[] = {{q, qb}, {start, (size_t)(B + 1) * 4}, {request, (size_t)T * 4}, {position, (size_t)T * 4},
                            {table, (size_t)B * table_cols * 4}, {blocks, (size_t)T * a.c.heads * count * 4}, {x.slopes, (size_t)q_heads * 4},
                            {x.first, (size_t)T * 4}, {x.prefix, (size_t)T * 4}};
        const Span outs[] = {{out, rows * a.c.dim * 2}, {out_lse, rows * 4}};
        if ((st = no_overlap(ctx, outs, 2, ins, 9)) != IVF_OK) return st;
        for (const Span &o : outs)
            if (overlaps_cache(a.c, o.p, o.n)) return fail(ctx, IVF_EINVAL, "outputs overlap the cache");
        const size_t need = p.token_bytes + p.prompt_bytes;
        if (need && (st = check_ws(ctx, need)) != IVF_OK) return st;
        DeviceGuard g(ctx->device);
        if (!g.ok) return fail(ctx, IVF_EDEVICE, "no usable device (context device %d)", ctx->device);
        a.q = {q, q_token_stride, q_head_stride};
        a.group = q_heads / a.c.heads;
        a.T = T;
        a.start = start;
        a.request = request;
        a.position = position;
        a.table = table;
        a.B = B;
        a.cols = table_cols;
        a.blocks = blocks;
        a.count = count;
        // a scale of 0 as the least number above it: masked scores stay -infinity
        a.scale = std::max(scale2, 0x1p-149f);
        a.q_flip = scale < 0.f ? 0x80008000u : 0u;
        const bool has_terms = x.cap != 0.f || x.slopes || x.first || x.prefix;
        if (x.cap != 0.f) a.scale = std::max(fabsf(scale) / x.cap, 0x1p-149f);
        x.cap *= 1.44269504089f;
        const float near[5] = {0.99999994f, -0.333323091f, 0.133101732f, -0.0521014817f, 0.0154754277f};
        for (int i = 0; i < 5; ++i) x.near[i] = near[i] * x.cap;
        a.out = out;
        a.lse = out_lse;
        a.small_rows = p.small_rows;
        a.unit_size = p.unit_size;
        a.team = p.team;
        a.unit_rows = p.unit_rows;
        a.per_unit = p.per_unit;
        a.units = (int)p.units;
        a.slots = (int)p.slots;
        KvAttend prompts = a;
        if (p.tokens) {
            char *ws = (char *)ctx->ws;
            a.splits = p.token_splits;
            a.part = (float *)ws;
            a.part_ml = (float2 *)(ws + p.token_ml);
            a.unit_parts = (int2 *)(ws + p.token_parts);
            TIMED("kv_attend", has_terms ? launch_kv_tokens_terms(a, x, p.token_groups, ctx->stream)
                                         : launch_kv_tokens(a, p.token_groups, ctx->stream));
        }
        if (p.prompt) {
            char *ws = (char *)ctx->ws + p.token_bytes;
            prompts.splits = p.prompt_splits;
            prompts.part = (float *)ws;
            prompts.part_ml = (float2 *)(ws + p.prompt_ml);
            TIMED("kv_prompt", has_terms ? launch_kv_prompt_terms(prompts, x, ctx->stream) : launch_kv_prompt(prompts, ctx->stream));
        }
        const KvAttend *join_prompts = p.prompt && p.prompt_splits > 1 ? &prompts : nullptr;
        const KvAttend *join_units = p.tokens && p.token_splits > 1 ? &a : nullptr;
        if (join_prompts || join_units) TIMED("kv_combine", launch_kv_combine(join_prompts, join_units, ctx->stream));
        ctx->last_stats = nullptr;
        return IVF_OK;
    });
}

}  // namespace

extern "C" {

ivf_status ivf_kv_plan(ivf_ctx *ctx, const int32_t *cached, const int32_t *added, int64_t B, int32_t block_size,
                       int32_t *table, int32_t table_cols, const int32_t *free_blocks, int64_t n_free, int64_t T,
                       int32_t *out_start, int64_t *out_slots, int32_t *out_request, int32_t *out_position,
                       int64_t *out_info)
{
    return guarded(ctx, "kv_plan", [&]() -> ivf_status {
        const int shift = block_shift(block_size);
        if (!shift) return fail(ctx, IVF_EUNSUPPORTED, "block_size must be 16, 32, 64 or 128 (got %d)", block_size);
        if (B < 0 || T < 0 || n_free < 0) return fail(ctx, IVF_EINVAL, "B, T and n_free must be >= 0");
        // an empty batch fills the outputs that are there; it needs no table (and a validation-only context, nothing)
        if (B == 0 && (ctx->device < 0 || (!out_start && !out_slots && !out_request && !out_position && !out_info)))
            return IVF_OK;
        if (B > kKvMaxRequests) return fail(ctx, IVF_EUNSUPPORTED, "at most %d requests", kKvMaxRequests);
        if (T > INT32_MAX) return fail(ctx, IVF_EUNSUPPORTED, "T must be < 2^31");
        ivf_status st = B == 0 ? IVF_OK : check_table(ctx, B, table_cols, shift);
        if (st != IVF_OK) return st;
        if (B && (!cached || !added || !table || !out_start || (n_free && !free_blocks) ||
                  (T && (!out_slots || !out_request || !out_position))))
            return fail(ctx, IVF_EINVAL, "null pointer argument");
        const void *i32[] = {cached, added, table, free_blocks, out_start, out_request, out_position};
        const void *i64[] = {out_slots, out_info};
        if ((st = check_elements(ctx, i32, 4)) != IVF_OK || (st = check_elements(ctx, i64, 8)) != IVF_OK) return st;
        const Span ins[] = {{cached, (size_t)B * 4}, {added, (size_t)B * 4}, {free_blocks, (size_t)n_free * 4}};
        const Span outs[] = {{table, B ? (size_t)B * table_cols * 4 : 0}, {out_start, (size_t)(B + 1) * 4},
                             {out_slots, (size_t)T * 8}, {out_request, (size_t)T * 4}, {out_position, (size_t)T * 4},
                             {out_info, 32}};
        if ((st = no_overlap(ctx, outs, 6, ins, 3)) != IVF_OK) return st;
        DeviceGuard g(ctx->device);
        if (!g.ok) return fail(ctx, IVF_EDEVICE, "no usable device (context device %d)", ctx->device);
        TIMED("kv_plan", launch_kv_plan(cached, added, (int)B, shift, table, B ? table_cols : 1, free_blocks, n_free, T,
                                        out_start, out_slots, out_request, out_position, out_info, ctx->num_cus,
                                        ctx->stream));
        ctx->last_stats = nullptr;
        return IVF_OK;
    });
}

ivf_status ivf_kv_fork(ivf_ctx *ctx, const int32_t *parent, const int32_t *child, int64_t n, int32_t *cached, int64_t B,
                       int32_t block_size, int32_t *table, int32_t table_cols, const int32_t *free_blocks,
                       int64_t n_free, int32_t *out_source, int32_t *out_to, int64_t *out_info)
{
    return guarded(ctx, "kv_fork", [&]() -> ivf_status {
        const int shift = block_shift(block_size);
        if (!shift) return fail(ctx, IVF_EUNSUPPORTED, "block_size must be 16, 32, 64 or 128 (got %d)", block_size);
        if (n < 0 || n_free < 0) return fail(ctx, IVF_EINVAL, "n and n_free must be >= 0");
        if (n == 0 && !out_info) return IVF_OK;
        ivf_status st = check_table(ctx, B, table_cols, shift);
        if (st != IVF_OK) return st;
        if (n > kKvMaxRequests || B > kKvMaxRequests)
            return fail(ctx, IVF_EUNSUPPORTED, "at most %d forks and requests", kKvMaxRequests);
        if (!cached || !table || (n_free && !free_blocks) || (n && (!parent || !child || !out_source || !out_to)))
            return fail(ctx, IVF_EINVAL, "null pointer argument");
        const void *i32[] = {parent, child, cached, table, free_blocks, out_source, out_to};
        const void *i64[] = {out_info};
        if ((st = check_elements(ctx, i32, 4)) != IVF_OK || (st = check_elements(ctx, i64, 8)) != IVF_OK) return st;
        const Span ins[] = {{parent, (size_t)n * 4}, {child, (size_t)n * 4}, {free_blocks, (size_t)n_free * 4}};
        const Span outs[] = {{table, (size_t)B * table_cols * 4}, {cached, (size_t)B * 4}, {out_source, (size_t)n * 4},
                             {out_to, (size_t)n * 4}, {out_info, 16}};
        if ((st = no_overlap(ctx, outs, 5, ins, 3)) != IVF_OK) return st;
        DeviceGuard g(ctx->device);
        if (!g.ok) return fail(ctx, IVF_EDEVICE, "no usable device (context device %d)", ctx->device);
        TIMED("kv_fork", launch_kv_fork(parent, child, (int)n, cached, (int)B, shift, table, table_cols, free_blocks, n_free,
                                        out_source, out_to, out_info, ctx->num_cus, ctx->stream));
        ctx->last_stats = nullptr;
        return IVF_OK;
    });
}

ivf_status ivf_kv_copy(ivf_ctx *ctx, const ivf_kv_cache *cache, const ivf_kv_cache *source_cache, const int32_t *to,
                       const int32_t *source, int64_t n)
{
    return guarded(ctx, "kv_copy", [&]() -> ivf_status {
        KvCache dst, src;
        ivf_status st = check_cache(ctx, cache, dst);
        if (st != IVF_OK || (st = check_cache(ctx, source_cache, src)) != IVF_OK) return st;
        if (dst.bs != src.bs || dst.heads != src.heads || dst.dim != src.dim || dst.bf16 != src.bf16)
            return fail(ctx, IVF_EINVAL, "the caches' block_size, heads, dim and type must be the same");
        const bool same = dst.rec == src.rec && dst.summary == src.summary && dst.weight == src.weight;
        const size_t sh = (size_t)src.blocks * src.heads;
        if (!same && (overlaps_cache(dst, src.rec, sh * src.rec_bytes()) || overlaps_cache(dst, src.summary, sh * src.dim) ||
                      overlaps_cache(dst, src.weight, sh * 4)))
            return fail(ctx, IVF_EINVAL, "the caches overlap");
        if (n < 0) return fail(ctx, IVF_EINVAL, "n must be >= 0");
        if (n > INT32_MAX) return fail(ctx, IVF_EUNSUPPORTED, "n must be < 2^31");
        if (n == 0) return IVF_OK;
        if (!to || !source) return fail(ctx, IVF_EINVAL, "null pointer argument");
        const void *i32[] = {to, source};
        if ((st = check_elements(ctx, i32, 4)) != IVF_OK) return st;
        if (overlaps_cache(dst, to, (size_t)n * 4) || overlaps_cache(dst, source, (size_t)n * 4))
            return fail(ctx, IVF_EINVAL, "inputs overlap the cache");
        DeviceGuard g(ctx->device);
        if (!g.ok) return fail(ctx, IVF_EDEVICE, "no usable device (context device %d)", ctx->device);
        TIMED("kv_copy", launch_kv_copy(dst, src, to, source, n, ctx->num_cus, ctx->stream));
        ctx->last_stats = nullptr;
        return IVF_OK;
    });
}

size_t ivf_kv_reclaim_bytes(int64_t B, int32_t block_size, int32_t table_cols, int64_t blocks, int64_t moves)
{
    const int shift = block_shift(block_size);
    if (!shift || B < 0 || (B && check_table(nullptr, B, table_cols, shift) != IVF_OK) || blocks < 1 || blocks > INT32_MAX ||
        moves < 0 || moves > INT32_MAX)
        return 0;
    size_t counts, rank;
    return kv_reclaim_workspace(blocks, B ? B * table_cols : 0, moves, &counts, &rank);
}

ivf_status ivf_kv_reclaim(ivf_ctx *ctx, const int32_t *cached, int64_t B, int32_t block_size, int32_t *table,
                          int32_t table_cols, int64_t blocks, int64_t moves, int32_t *out_free, int32_t *out_source,
                          int32_t *out_to, int64_t *out_info)
{
    return guarded(ctx, "kv_reclaim", [&]() -> ivf_status {
        const int shift = block_shift(block_size);
        if (!shift) return fail(ctx, IVF_EUNSUPPORTED, "block_size must be 16, 32, 64 or 128 (got %d)", block_size);
        if (B < 0) return fail(ctx, IVF_EINVAL, "B must be >= 0");
        ivf_status st = B == 0 ? IVF_OK : check_table(ctx, B, table_cols, shift);
        if (st != IVF_OK) return st;
        if (blocks < 1 || blocks > INT32_MAX)
            return fail(ctx, IVF_EINVAL, "blocks must be in [1, 2^31) (got %lld)", (long long)blocks);
        if (moves < 0 || moves > INT32_MAX) return fail(ctx, IVF_EINVAL, "moves must be in [0, 2^31)");
        if ((B && (!cached || !table)) || (moves && (!out_source || !out_to)))
            return fail(ctx, IVF_EINVAL, "null pointer argument");
        if (!moves) out_source = out_to = nullptr;
        if (!moves && !out_free && !out_info) return IVF_OK;
        const void *i32[] = {cached, table, out_free, out_source, out_to};
        const void *i64[] = {out_info};
        if ((st = check_elements(ctx, i32, 4)) != IVF_OK || (st = check_elements(ctx, i64, 8)) != IVF_OK) return st;
        const Span ins[] = {{cached, (size_t)B * 4}};
        const Span outs[] = {{table, B ? (size_t)B * table_cols * 4 : 0}, {out_free, (size_t)blocks * 4},
                             {out_source, (size_t)moves * 4}, {out_to, (size_t)moves * 4}, {out_info, 24}};
        if ((st = no_overlap(ctx, outs, 5, ins, 1)) != IVF_OK) return st;
        KvReclaim a = {};
        a.cached = cached;
        a.B = B;
        a.shift = shift;
        a.table = table;
        a.cols = B ? table_cols : 1;
        a.blocks = blocks;
        a.moves = moves;
        a.free = out_free;
        a.source = out_source;
        a.to = out_to;
        a.info = out_info;
        size_t counts = 0, rank = 0;
        const size_t need = kv_reclaim_workspace(blocks, a.B * a.cols, moves, &counts, &rank);
        if (need) {
            if ((st = check_ws(ctx, need)) != IVF_OK) return st;
            a.bits = (uint32_t *)ctx->ws;
            a.counts = (uint32_t *)((char *)ctx->ws + counts);
            a.rank = (int32_t *)((char *)ctx->ws + rank);
        }
        DeviceGuard g(ctx->device);
        if (!g.ok) return fail(ctx, IVF_EDEVICE, "no usable device (context device %d)", ctx->device);
        TIMED("kv_reclaim", launch_kv_reclaim(a, ctx->num_cus, ctx->stream));
        ctx->last_stats = nullptr;
        return IVF_OK;
    });
}

ivf_status ivf_kv_append(ivf_ctx *ctx, const ivf_kv_cache *cache, const void *k, int64_t k_token_stride,
                         int64_t k_head_stride, const void *v, int64_t v_token_stride, int64_t v_head_stride,
                         const int64_t *slots, int64_t T)
{
    return guarded(ctx, "kv_append", [&]() -> ivf_status {
        KvCache c;
        ivf_status st = check_cache(ctx, cache, c);
        if (st != IVF_OK) return st;
        if ((st = check_tokens(ctx, c, T, c.heads)) != IVF_OK) return st;
        if (T == 0) return IVF_OK;
        if ((st = check_threads(ctx, kv_cache_threads(c, T, T <= kKvFewTokens ? T : 0))) != IVF_OK) return st;
        size_t kb, vb;
        if ((st = check_rows(ctx, "k", k, k_token_stride, k_head_stride, T, c.heads, c.dim, &kb)) != IVF_OK) return st;
        if ((st = check_rows(ctx, "v", v, v_token_stride, v_head_stride, T, c.heads, c.dim, &vb)) != IVF_OK) return st;
        if (!slots) return fail(ctx, IVF_EINVAL, "null pointer argument: slots");
        const void *i64[] = {slots};
        if ((st = check_elements(ctx, i64, 8)) != IVF_OK) return st;
        if (overlaps_cache(c, k, kb) || overlaps_cache(c, v, vb) || overlaps_cache(c, slots, (size_t)T * 8))
            return fail(ctx, IVF_EINVAL, "inputs overlap the cache");
        DeviceGuard g(ctx->device);
        if (!g.ok) return fail(ctx, IVF_EDEVICE, "no usable device (context device %d)", ctx->device);
        TIMED("kv_append", launch_kv_append(c, {k, k_token_stride, k_head_stride}, {v, v_token_stride, v_head_stride},
                                            slots, T, ctx->stream));
        ctx->last_stats = nullptr;
        return IVF_OK;
    });
}

ivf_status ivf_kv_read(ivf_ctx *ctx, const ivf_kv_cache *cache, const int64_t *slots, int64_t T, void *out_k,
                       void *out_v, const int32_t *blocks, int64_t n, float *out_mean)
{
    return guarded(ctx, "kv_read", [&]() -> ivf_status {
        KvCache c;
        ivf_status st = check_cache(ctx, cache, c);
        if (st != IVF_OK) return st;
        if ((st = check_tokens(ctx, c, T, c.heads)) != IVF_OK) return st;
        if ((st = check_tokens(ctx, c, n, c.heads)) != IVF_OK) return st;
        if (!out_k && !out_v) T = 0;
        if (T == 0 && n == 0) return IVF_OK;
        if ((st = check_threads(ctx, kv_cache_threads(c, T, n))) != IVF_OK) return st;
        if ((T && !slots) || (n && (!blocks || !out_mean))) return fail(ctx, IVF_EINVAL, "null pointer argument");
        const void *i32[] = {blocks}, *i64[] = {slots};
        if ((st = check_elements(ctx, i32, 4)) != IVF_OK || (st = check_elements(ctx, i64, 8)) != IVF_OK) return st;
        if (!aligned16(out_k) || !aligned16(out_v) || !aligned16(out_mean))
            return fail(ctx, IVF_EINVAL, "outputs must be 16-byte aligned");
        const size_t row = (size_t)c.heads * c.dim;
        const Span ins[] = {{slots, (size_t)T * 8}, {blocks, (size_t)n * 4}};
        const Span outs[] = {{out_k, T * row * 2}, {out_v, T * row * 2}, {out_mean, n * row * 4}};
        if ((st = no_overlap(ctx, outs, 3, ins, 2)) != IVF_OK) return st;
        for (const Span &o : outs)
            if (overlaps_cache(c, o.p, o.n)) return fail(ctx, IVF_EINVAL, "outputs overlap the cache");
        DeviceGuard g(ctx->device);
        if (!g.ok) return fail(ctx, IVF_EDEVICE, "no usable device (context device %d)", ctx->device);
        TIMED("kv_read", launch_kv_read(c, slots, T, out_k, out_v, blocks, n, out_mean, ctx->stream));
        ctx->last_stats = nullptr;
        return IVF_OK;
    });
}

ivf_status ivf_kv_select(ivf_ctx *ctx, const ivf_kv_cache *cache, const void *q, int64_t q_token_stride,
                         int64_t q_head_stride, int32_t q_heads, int64_t T, const int32_t *request,
                         const int32_t *position, const int32_t *table, int64_t B, int32_t table_cols, int32_t first,
                         int32_t last, int32_t count, int32_t *out_blocks)
{
    return guarded(ctx, "kv_select", [&]() -> ivf_status {
        KvSelect a;
        ivf_status st = check_cache(ctx, cache, a.c);
        if (st != IVF_OK) return st;
        if (q_heads < 1 || q_heads > 65536 || q_heads % a.c.heads)
            return fail(ctx, IVF_EINVAL, "q_heads must be a multiple of the cache's heads (got %d, %d)", q_heads, a.c.heads);
        if (first < 0 || last < 1 || count > kKvMaxCount || (int64_t)first + last > count)
            return fail(ctx, IVF_EINVAL, "first >= 0, last >= 1 and first + last <= count <= %d are wanted", kKvMaxCount);
        if ((st = check_tokens(ctx, a.c, T, q_heads)) != IVF_OK) return st;
        if (T == 0) return IVF_OK;
        if ((st = check_table(ctx, B, table_cols, a.c.shift)) != IVF_OK) return st;
        if (table_cols > kKvMaxSelectCols)
            return fail(ctx, IVF_EUNSUPPORTED, "at most %d blocks of a request", kKvMaxSelectCols);
        size_t qb;
        if ((st = check_rows(ctx, "q", q, q_token_stride, q_head_stride, T, q_heads, a.c.dim, &qb)) != IVF_OK) return st;
        const void *i32[] = {request, position, table, out_blocks};
        for (const void *p : i32)
            if (!p) return fail(ctx, IVF_EINVAL, "null pointer argument");
        if ((st = check_elements(ctx, i32, 4)) != IVF_OK) return st;
        const Span ins[] = {{q, qb}, {request, (size_t)T * 4}, {position, (size_t)T * 4}, {table, (size_t)B * table_cols * 4}};
        const Span outs[] = {{out_blocks, (size_t)T * a.c.heads * count * 4}};
        if ((st = no_overlap(ctx, outs, 1, ins, 4)) != IVF_OK) return st;
        if (overlaps_cache(a.c, outs[0].p, outs[0].n)) return fail(ctx, IVF_EINVAL, "outputs overlap the cache");
        DeviceGuard g(ctx->device);
        if (!g.ok) return fail(ctx, IVF_EDEVICE, "no usable device (context device %d)", ctx->device);
        a.q = {q, q_token_stride, q_head_stride};
        a.group = q_heads / a.c.heads;
        a.T = T;
        a.request = request;
        a.position = position;
        a.table = table;
        a.B = B;
        a.cols = table_cols;
        a.first = first;
        a.last = last;
        a.count = count;
        a.out = out_blocks;
        TIMED("kv_select", launch_kv_select(a, ctx->stream));
        ctx->last_stats = nullptr;
        return IVF_OK;
    });
}

size_t ivf_kv_attend_bytes(const ivf_kv_cache *cache, int32_t q_heads, int64_t T, int64_t B, int32_t table_cols,
                           int32_t count, int64_t longest)
{
    KvCache c;
    if (check_cache(nullptr, cache, c) != IVF_OK) return 0;
    int num_cus = 256, dev = 0;
    if (hipGetDevice(&dev) == hipSuccess) {
        int n = 0;
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && n > 0) num_cus = n;
    }
    KvAttendPlan p = {};
    if (plan_attend(nullptr, c, q_heads, T, B, table_cols, count, longest, num_cus, p) != IVF_OK) return 0;
    return p.token_bytes + p.prompt_bytes;
}

ivf_status ivf_kv_attend(ivf_ctx *ctx, const ivf_kv_cache *cache, const void *q, int64_t q_token_stride,
                         int64_t q_head_stride, int32_t q_heads, int64_t T, const int32_t *start,
                         const int32_t *request, const int32_t *position, const int32_t *table, int64_t B,
                         int32_t table_cols, const int32_t *blocks, int32_t count, float scale, int64_t longest,
                         void *out, float *out_lse)
{
    return attend(ctx, cache, q, q_token_stride, q_head_stride, q_heads, T, start, request, position, table, B, table_cols,
                  blocks, count, scale, longest, nullptr, out, out_lse);
}

ivf_status ivf_kv_attend_terms(ivf_ctx *ctx, const ivf_kv_cache *cache, const void *q, int64_t q_token_stride,
                               int64_t q_head_stride, int32_t q_heads, int64_t T, const int32_t *start,
                               const int32_t *request, const int32_t *position, const int32_t *table, int64_t B,
                               int32_t table_cols, const int32_t *blocks, int32_t count, float scale, int64_t longest,
                               const ivf_kv_terms *terms, void *out, float *out_lse)
{
    return attend(ctx, cache, q, q_token_stride, q_head_stride, q_heads, T, start, request, position, table, B, table_cols,
                  blocks, count, scale, longest, terms, out, out_lse);
}

}  // extern "C"

// cache_api.hip -- the C ABI of the paged cache (include/fma.h): plans, argument
// checks, launches.  Host code only.
#include <math.h>
#include <string.h>

#include <new>

#include "api_status.hpp"
#include "cache.hpp"
#include "fma_kernels.hpp"

using namespace fma_dev;

struct fma_cache_plan_s {
    fma_cache_desc_t desc;
    int levels, sets;
    int64_t wlen, blocks;
    float scale;
};

namespace {

// Tokens and sequences of one call.
constexpr int64_t kMaxRows = 1 << 21;
constexpr int32_t kMaxSequences = 1 << 20;

fma_status_t check_pool(const char *fn, const char *name, const void *p, size_t align)
{
    if (!p) return set_status(FMA_ERR_NULL, "%s: %s is NULL", fn, name);
    if (!is_aligned(p, align)) return set_status(FMA_ERR_ALIGN, "%s: %s is not %zu-byte aligned", fn, name, align);
    return FMA_OK;
}

struct Call {
    const char *fn;
    fma_cache_plan_t p;
    const fma_cache_batch_t *b;
    const fma_view_t *q, *k, *v, *out;
    const float *wk, *wv;
};

// The attention of a call (a.write: with the new tokens' way into the cache).
hipError_t launch_attention(const CacheArgs &a, CacheRoute route, int cus, hipStream_t st)
{
    if (route == CACHE_TOKENS) return launch_cache_token(a, st);
    const ChunkShape c = chunk_shape(a);
    return route == CACHE_KEYS ? launch_cache_keys(a, c, cus, st) : launch_cache_rows(a, c, st);
}

// Checks everything of a call; *skip: no rows, nothing to do.
fma_status_t check_call(const Call &c, CacheArgs &a, bool *skip)
{
    const char *fn = c.fn;
    if (!c.p || !c.b) return set_status(FMA_ERR_NULL, "%s: plan and batch must not be NULL", fn);
    const fma_cache_desc_t &d = c.p->desc;
    const fma_cache_batch_t &b = *c.b;
    if (b.sequences < 0 || b.max_chunk < 0 || b.rows < 0 || b.num_pages < 0 || b.num_summaries < 0 || b.table_stride < 0)
        return set_status(FMA_ERR_SHAPE, "%s: negative size", fn);
    if (b.rows > kMaxRows || b.sequences > kMaxSequences)
        return set_status(FMA_ERR_SHAPE, "%s: more than %lld rows or %d sequences in a call", fn, (long long)kMaxRows,
                          kMaxSequences);
    if (b.num_pages > 0x7fffffffLL || b.num_summaries > 0x7fffffffLL)
        return set_status(FMA_ERR_SHAPE, "%s: more than 2^31 - 1 pages", fn);
    *skip = b.sequences == 0 || b.rows == 0 || b.max_chunk == 0;
    if (*skip) return FMA_OK;
    const int e = d.dtype == FMA_BF16 ? 2 : 4, sets = c.p->sets;
    const View q = {c.q, 1, d.heads, b.rows, d.head_dim, e, "q"}, out = {c.out, 1, d.heads, b.rows, d.head_dim, e, "out"};
    const View k = {c.k, 1, d.kv_heads, b.rows, d.head_dim, e, "k"}, v = {c.v, 1, d.kv_heads, b.rows, d.head_dim, e, "v"};
    fma_status_t st;
    const bool writes = c.k || c.v || !c.q, attends = c.q || c.out;
    if (attends && ((st = check_view(fn, q, false)) || (st = check_view(fn, out, true)))) return st;
    if (writes && ((st = check_view(fn, k, false)) || (st = check_view(fn, v, false)))) return st;
    if ((st = check_pool(fn, "k_pages", b.k_pages, 16)) || (st = check_pool(fn, "v_pages", b.v_pages, 16)) ||
        (st = check_pool(fn, "page_table", b.page_table, 4)) || (st = check_pool(fn, "cu_tokens", b.cu_tokens, 4)) ||
        (st = check_pool(fn, "start", b.start, 4)))
        return st;
    if (sets && ((st = check_pool(fn, "summaries", b.summaries, 16)) ||
                 (st = check_pool(fn, "summary_table", b.summary_table, 4))))
        return st;
    if (sets && writes && ((st = check_pool(fn, "wk", c.wk, 4)) || (st = check_pool(fn, "wv", c.wv, 4)))) return st;
    const size_t page = (size_t)d.kv_heads * d.block * d.head_dim * e;
    const size_t sum = (size_t)d.kv_heads * 2 * sets * d.head_dim * sizeof(float);
    const size_t pool = page * (size_t)b.num_pages, sums = sum * (size_t)b.num_summaries;
    if (ranges_meet(b.k_pages, pool, b.v_pages, pool) ||
        (sets && (ranges_meet(b.summaries, sums, b.k_pages, pool) || ranges_meet(b.summaries, sums, b.v_pages, pool))))
        return set_status(FMA_ERR_ARG, "%s: the pools overlap", fn);
    const View *views[4] = {&q, &out, &k, &v};
    for (int i = attends ? 0 : 2; i < (writes ? 4 : 2); ++i) {
        const View &x = *views[i];
        if (ranges_meet(x.v->data, x.extent(), b.k_pages, pool) || ranges_meet(x.v->data, x.extent(), b.v_pages, pool) ||
            (sets && ranges_meet(x.v->data, x.extent(), b.summaries, sums)))
            return set_status(FMA_ERR_ARG, "%s: %s overlaps a pool", fn, x.name);
    }
    if (attends && !out.same(q) && views_meet(out, q)) return set_status(FMA_ERR_ARG, "%s: out overlaps q", fn);
    if (attends && writes && (views_meet(out, k) || views_meet(out, v)))
        return set_status(FMA_ERR_ARG, "%s: out overlaps k or v", fn);

    memset(&a, 0, sizeof(a));
    if (attends) {
        a.q = c.q->data, a.qt = c.q->token_stride, a.qh = c.q->head_stride;
        a.out = c.out->data, a.ot = c.out->token_stride, a.oh = c.out->head_stride;
    }
    if (writes) {
        a.k = c.k->data, a.kt = c.k->token_stride, a.kh = c.k->head_stride;
        a.v = c.v->data, a.vt = c.v->token_stride, a.vh = c.v->head_stride;
    }
    a.kp = b.k_pages, a.vp = b.v_pages, a.sum = b.summaries;
    a.npages = b.num_pages, a.nsums = b.num_summaries;
    a.table = b.page_table, a.stable = b.summary_table, a.tstride = b.table_stride;
    a.cu = b.cu_tokens, a.start = b.start;
    a.wk = c.wk, a.wv = c.wv, a.w_stride = d.weights_per_head ? c.p->wlen : 0;
    a.S = b.sequences, a.max_chunk = b.max_chunk, a.rows = (int)b.rows;
    const int64_t table = b.table_stride > d.max_seq_len / d.block ? d.max_seq_len : b.table_stride * d.block;
    a.limit = (int)(table < d.max_seq_len ? table : d.max_seq_len);
    a.heads = d.heads, a.kv_heads = d.kv_heads, a.group = d.heads / d.kv_heads;
    a.r = d.block, a.rank = d.rank, a.levels = c.p->levels, a.sets = sets;
    a.head_dim = d.head_dim, a.bf16 = d.dtype == FMA_BF16;
    a.scale_log2 = c.p->scale * (float)M_LOG2E;
    if (!cache_launches_fit(a, writes, attends, compute_units()))
        return set_status(FMA_ERR_SHAPE, "%s: too many rows and heads for one call", fn);
    (void)hipGetLastError();
    return FMA_OK;
}

}  // namespace

extern "C" {

fma_status_t fma_cache_plan(const fma_cache_desc_t *d, fma_cache_plan_t *out)
{
    const char *fn = "fma_cache_plan";
    if (!d || !out) return set_status(FMA_ERR_NULL, "%s: desc and out_plan must not be NULL", fn);
    *out = nullptr;
    if (d->struct_size != (int32_t)sizeof(fma_cache_desc_t))
        return set_status(FMA_ERR_ARG, "%s: struct_size %d != sizeof(fma_cache_desc_t) %zu", fn, d->struct_size,
                          sizeof(fma_cache_desc_t));
    if (d->dtype != FMA_F32 && d->dtype != FMA_BF16) return set_status(FMA_ERR_ARG, "%s: unknown dtype %d", fn, d->dtype);
    if (d->heads < 1 || d->kv_heads < 1 || d->heads % d->kv_heads)
        return set_status(FMA_ERR_SHAPE, "%s: kv_heads %d does not divide heads %d", fn, d->kv_heads, d->heads);
    if (d->heads > 0x4000) return set_status(FMA_ERR_SHAPE, "%s: more than %d heads", fn, 0x4000);
    if (d->head_dim != 32 && d->head_dim != 64 && d->head_dim != 128)
        return set_status(FMA_ERR_UNSUPPORTED, "%s: head_dim %d not implemented (32, 64 or 128)", fn, d->head_dim);
    if (d->block <= 0) return set_status(FMA_ERR_SHAPE, "%s: block must be positive, got %d", fn, d->block);
    if ((d->block % 64 || d->block > 256) && d->block != 16 && d->block != 32)
        return set_status(FMA_ERR_UNSUPPORTED, "%s: block %d not implemented (16, 32 or a multiple of 64 up to 256)", fn,
                          d->block);
    if (d->max_seq_len < 1 || d->max_seq_len > 0x7fffffffLL - 1024)
        return set_status(FMA_ERR_SHAPE, "%s: max_seq_len %lld outside 1 .. 2^31 - 1025", fn, (long long)d->max_seq_len);
    if (d->rank < 0) return set_status(FMA_ERR_ARG, "%s: rank must be >= 1 (0 selects 1), got %d", fn, d->rank);
    if (d->weights_per_head != 0 && d->weights_per_head != 1)
        return set_status(FMA_ERR_ARG, "%s: weights_per_head must be 0 or 1", fn);
    if (d->norm != FMA_NORM_JOINT && d->norm != FMA_NORM_PER_LEVEL)
        return set_status(FMA_ERR_ARG, "%s: unknown norm %d", fn, d->norm);
    if (d->norm == FMA_NORM_PER_LEVEL)
        return set_status(FMA_ERR_UNSUPPORTED, "%s: per-level normalisation is not implemented for the cache", fn);
    if (!isfinite(d->softmax_scale)) return set_status(FMA_ERR_ARG, "%s: softmax_scale is not finite", fn);
    fma_cache_plan_s p;
    memset(&p, 0, sizeof(p));
    p.desc = *d;
    if (p.desc.rank == 0) p.desc.rank = 1;
    p.blocks = (d->max_seq_len + d->block - 1) / d->block;
    int L = 0;
    while ((1LL << L) < p.blocks) ++L;
    p.levels = L > 1 ? L - 1 : 0;
    if (p.levels > kMaxCoarse)
        return set_status(FMA_ERR_UNSUPPORTED, "%s: %d levels exceed the supported %d", fn, L, kMaxCoarse + 1);
    if ((int64_t)p.levels * p.desc.rank > kMaxSets)
        return set_status(FMA_ERR_UNSUPPORTED, "%s: %d levels x rank %d exceed the supported %d coarse sets", fn, p.levels,
                          p.desc.rank, kMaxSets);
    p.sets = p.levels * p.desc.rank;
    p.wlen = (int64_t)p.desc.rank * d->block * ((1LL << p.levels) - 1);
    p.scale = d->softmax_scale != 0.f ? d->softmax_scale : 1.0f / sqrtf((float)d->head_dim);
    fma_cache_plan_s *h = new (std::nothrow) fma_cache_plan_s(p);
    if (!h) return set_status(FMA_ERR_HOST_ALLOC, "%s: out of host memory", fn);
    *out = h;
    return set_status(FMA_OK, nullptr);
}

fma_status_t fma_cache_destroy(fma_cache_plan_t plan)
{
    delete plan;
    return set_status(FMA_OK, nullptr);
}

fma_status_t fma_cache_sizes(fma_cache_plan_t p, int32_t *sets, int64_t *weights_len, int64_t *blocks)
{
    if (!p || !sets || !weights_len || !blocks)
        return set_status(FMA_ERR_NULL, "fma_cache_sizes: plan and results must not be NULL");
    *sets = p->sets;
    *weights_len = p->wlen;
    *blocks = p->blocks;
    return set_status(FMA_OK, nullptr);
}

fma_status_t fma_cache_append(fma_cache_plan_t plan, const fma_cache_batch_t *batch, const fma_view_t *k,
                              const fma_view_t *v, const float *wk, const float *wv, void *stream)
{
    const Call c = {"fma_cache_append", plan, batch, nullptr, k, v, nullptr, wk, wv};
    CacheArgs a;
    bool skip = false;
    const fma_status_t st = check_call(c, a, &skip);
    if (st) return st;
    if (skip) return set_status(FMA_OK, nullptr);
    return status_of(c.fn, launch_cache_append(a, static_cast<hipStream_t>(stream)));
}

fma_status_t fma_cache_attend(fma_cache_plan_t plan, const fma_cache_batch_t *batch, const fma_view_t *q,
                              const fma_view_t *out, void *stream)
{
    const Call c = {"fma_cache_attend", plan, batch, q, nullptr, nullptr, out, nullptr, nullptr};
    if (plan && batch && (!q || !out)) return set_status(FMA_ERR_NULL, "%s: q and out must not be NULL", c.fn);
    CacheArgs a;
    bool skip = false;
    const fma_status_t st = check_call(c, a, &skip);
    if (st) return st;
    if (skip) return set_status(FMA_OK, nullptr);
    const int cus = compute_units();
    return status_of(c.fn, launch_attention(a, cache_route(a, cus), cus, static_cast<hipStream_t>(stream)));
}

fma_status_t fma_cache_step(fma_cache_plan_t plan, const fma_cache_batch_t *batch, const fma_view_t *q,
                            const fma_view_t *k, const fma_view_t *v, const float *wk, const float *wv,
                            const fma_view_t *out, void *stream)
{
    const Call c = {"fma_cache_step", plan, batch, q, k, v, out, wk, wv};
    if (plan && batch && (!q || !k || !v || !out))
        return set_status(FMA_ERR_NULL, "%s: q, k, v and out must not be NULL", c.fn);
    CacheArgs a;
    bool skip = false;
    const fma_status_t st = check_call(c, a, &skip);
    if (st) return st;
    if (skip) return set_status(FMA_OK, nullptr);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int cus = compute_units();
    const CacheRoute route = cache_route(a, cus);
    a.write = route != CACHE_ROWS && a.max_chunk <= a.r;
    hipError_t e = hipSuccess;
    if (!a.write) e = launch_cache_append(a, s);
    if (e == hipSuccess) e = launch_attention(a, route, cus, s);
    return status_of(c.fn, e);
}

}  // extern "C"

// qk_api.hip -- the C ABI of the norm and rotation of queries and keys
// (include/fma.h): plans, argument checks, launches.  Host code only.
#include <math.h>
#include <string.h>

#include <new>

#include "api_status.hpp"
#include "qk_norm_rope.hpp"

using namespace fma_dev;

struct fma_qk_plan_s {
    fma_qk_desc_t desc;
    double turns[kMaxPairs];   // rates of an axis' pairs, turns per position
};

namespace {

constexpr int64_t kMaxRows = 1 << 28;

QkView device_view(const fma_view_t *v) { return {v->data, v->batch_stride, v->head_stride, v->token_stride}; }

// Everything a call's sizes decide; *skip: there is nothing to do.
fma_status_t check_sizes(const char *fn, fma_qk_plan_t p, int32_t batch, int64_t tokens, bool *skip)
{
    if (!p) return set_status(FMA_ERR_NULL, "%s: plan is NULL", fn);
    if (batch < 0 || tokens < 0) return set_status(FMA_ERR_SHAPE, "%s: negative batch / tokens", fn);
    *skip = batch == 0 || tokens == 0;
    if (!*skip && tokens >= kMaxRows / batch)
        return set_status(FMA_ERR_SHAPE, "%s: batch * tokens must stay below 2^28", fn);
    return FMA_OK;
}

fma_status_t check_floats(const char *fn, const char *name, const void *x)
{
    if (!is_aligned(x, 4)) return set_status(FMA_ERR_ALIGN, "%s: %s is not 4-byte aligned", fn, name);
    return FMA_OK;
}

// dst[i] may be src[i] itself; apart from that no dst meets any src or another dst
fma_status_t check_apart(const char *fn, const View *dst, int ndst, const View *src, int nsrc, bool in_place)
{
    for (int i = 0; i < ndst; ++i) {
        for (int j = 0; j < nsrc; ++j) {
            if (j % ndst == i && in_place && dst[i].same(src[j])) continue;
            if (views_meet(dst[i], src[j]))
                return set_status(FMA_ERR_ARG, "%s: %s overlaps %s", fn, dst[i].name, src[j].name);
        }
        for (int j = 0; j < i; ++j)
            if (views_meet(dst[i], dst[j]))
                return set_status(FMA_ERR_ARG, "%s: %s overlaps %s", fn, dst[i].name, dst[j].name);
    }
    return FMA_OK;
}

void fill(const fma_qk_plan_s *p, QkArgs &a, int32_t batch, int64_t tokens)
{
    const fma_qk_desc_t &d = p->desc;
    memset(&a, 0, sizeof(a));
    a.rows = (long long)batch * tokens;
    a.tokens = (int)tokens;
    a.heads = d.heads;
    a.kv_heads = d.kv_heads;
    a.rep = d.repeat_kv ? d.heads / d.kv_heads : 1;
    a.side = d.side;
    a.axes = d.axes;
    a.rotary = d.rotary_dim;
    a.interleaved = d.interleaved;
    a.dtype_bf16 = d.dtype == FMA_BF16;
    a.head_dim = d.head_dim;
    a.eps = d.eps;
    memcpy(a.turns, p->turns, sizeof(a.turns));
}

}  // namespace

extern "C" {

fma_status_t fma_qk_plan(const fma_qk_desc_t *d, const double *inv_freq, fma_qk_plan_t *out)
{
    const char *fn = "fma_qk_plan";
    if (!d || !out) return set_status(FMA_ERR_NULL, "%s: desc and out_plan must not be NULL", fn);
    *out = nullptr;
    if (d->struct_size != (int32_t)sizeof(fma_qk_desc_t))
        return set_status(FMA_ERR_ARG, "%s: struct_size %d != sizeof(fma_qk_desc_t) %zu", fn, d->struct_size,
                          sizeof(fma_qk_desc_t));
    if (d->dtype != FMA_F32 && d->dtype != FMA_BF16) return set_status(FMA_ERR_ARG, "%s: unknown dtype %d", fn, d->dtype);
    if (d->heads < 1 || d->kv_heads < 1 || d->heads % d->kv_heads)
        return set_status(FMA_ERR_SHAPE, "%s: kv_heads %d does not divide heads %d", fn, d->kv_heads, d->heads);
    if (d->heads > 0x4000) return set_status(FMA_ERR_SHAPE, "%s: more than %d heads", fn, 0x4000);
    if (d->head_dim != 32 && d->head_dim != 64 && d->head_dim != 128)
        return set_status(FMA_ERR_UNSUPPORTED, "%s: head_dim %d not implemented (32, 64 or 128)", fn, d->head_dim);
    if (d->axes != 1 && d->axes != 2) return set_status(FMA_ERR_ARG, "%s: axes must be 1 or 2", fn);
    if (d->rotary_dim < 0 || d->rotary_dim > d->head_dim)
        return set_status(FMA_ERR_SHAPE, "%s: rotary_dim %d outside 0 .. %d", fn, d->rotary_dim, d->head_dim);
    if (d->rotary_dim % (16 * d->axes))
        return set_status(FMA_ERR_UNSUPPORTED, "%s: rotary_dim %d not implemented (a multiple of 16 per axis)", fn,
                          d->rotary_dim);
    if (d->side < 0) return set_status(FMA_ERR_SHAPE, "%s: side is negative", fn);
    if ((d->interleaved != 0 && d->interleaved != 1) || (d->repeat_kv != 0 && d->repeat_kv != 1))
        return set_status(FMA_ERR_ARG, "%s: interleaved and repeat_kv must be 0 or 1", fn);
    if (!isfinite(d->eps) || d->eps < 0.f) return set_status(FMA_ERR_ARG, "%s: eps must be finite and not negative", fn);
    const int half = d->rotary_dim / 2 / d->axes;
    if (!inv_freq && half > 0 && !(isfinite(d->base) && d->base > 0.0))
        return set_status(FMA_ERR_ARG, "%s: base must be finite and positive", fn);
    fma_qk_plan_s p;
    memset(&p, 0, sizeof(p));
    p.desc = *d;
    for (int i = 0; i < half; ++i) {
        const double rate = inv_freq ? inv_freq[i] : pow(d->base, -(double)i / half);
        if (!isfinite(rate)) return set_status(FMA_ERR_ARG, "%s: inv_freq[%d] is not finite", fn, i);
        p.turns[i] = rate / (2.0 * M_PI);
    }
    fma_qk_plan_s *h = new (std::nothrow) fma_qk_plan_s(p);
    if (!h) return set_status(FMA_ERR_HOST_ALLOC, "%s: out of host memory", fn);
    *out = h;
    return set_status(FMA_OK, nullptr);
}

fma_status_t fma_qk_destroy(fma_qk_plan_t plan)
{
    delete plan;
    return set_status(FMA_OK, nullptr);
}

fma_status_t fma_qk_norm_rope(fma_qk_plan_t p, int32_t batch, int64_t tokens, const fma_view_t *q, const fma_view_t *k,
                              const fma_view_t *v, const float *gamma_q, const float *gamma_k,
                              const int32_t *positions, const fma_view_t *q_out, const fma_view_t *k_out,
                              const fma_view_t *v_out, void *stream)
{
    const char *fn = "fma_qk_norm_rope";
    bool skip = false;
    fma_status_t st = check_sizes(fn, p, batch, tokens, &skip);
    if (st) return st;
    if (skip) return set_status(FMA_OK, nullptr);
    const fma_qk_desc_t &d = p->desc;
    if (!v != !v_out) return set_status(FMA_ERR_NULL, "%s: v and v_out must be given together", fn);
    const int e = d.dtype == FMA_BF16 ? 2 : 4, ko = d.repeat_kv ? d.heads : d.kv_heads, n = v ? 3 : 2;
    const View in[3] = {{q, batch, d.heads, tokens, d.head_dim, e, "q"},
                        {k, batch, d.kv_heads, tokens, d.head_dim, e, "k"},
                        {v, batch, d.kv_heads, tokens, d.head_dim, e, "v"}};
    const View out[3] = {{q_out, batch, d.heads, tokens, d.head_dim, e, "q_out"},
                         {k_out, batch, ko, tokens, d.head_dim, e, "k_out"},
                         {v_out, batch, ko, tokens, d.head_dim, e, "v_out"}};
    for (int i = 0; i < n; ++i)
        if ((st = check_view(fn, in[i], false)) || (st = check_view(fn, out[i], true))) return st;
    if ((st = check_floats(fn, "gamma_q", gamma_q)) || (st = check_floats(fn, "gamma_k", gamma_k)) ||
        (st = check_floats(fn, "positions", positions)))
        return st;
    if (d.axes == 2 && d.rotary_dim && !positions && d.side <= 0)
        return set_status(FMA_ERR_SHAPE, "%s: a map without positions needs the plan's side", fn);
    if ((st = check_apart(fn, out, n, in, n, true))) return st;
    QkArgs a;
    fill(p, a, batch, tokens);
    a.q = device_view(q);
    a.k = device_view(k);
    a.qo = device_view(q_out);
    a.ko = device_view(k_out);
    a.has_v = v != nullptr;
    if (v) {
        a.v = device_view(v);
        a.vo = device_view(v_out);
    }
    a.gamma_q = gamma_q;
    a.gamma_k = gamma_k;
    a.pos = positions;
    (void)hipGetLastError();
    return status_of(fn, launch_qk(a, static_cast<hipStream_t>(stream)));
}

fma_status_t fma_qk_backward_workspace_size(fma_qk_plan_t p, int32_t batch, int64_t tokens, size_t *bytes)
{
    const char *fn = "fma_qk_backward_workspace_size";
    bool skip = false;
    const fma_status_t st = check_sizes(fn, p, batch, tokens, &skip);
    if (st) return st;
    if (!bytes) return set_status(FMA_ERR_NULL, "%s: bytes is NULL", fn);
    *bytes = 0;
    if (!skip) {
        // calls without values split the heads their own way: room for either
        long long g = 0;
        for (int kv = 1; kv <= 2; ++kv) {
            const long long x = qk_backward_groups((long long)batch * tokens, p->desc.heads + kv * p->desc.kv_heads,
                                                   p->desc.head_dim);
            if (x > g) g = x;
        }
        *bytes = (size_t)g * 2 * p->desc.head_dim * sizeof(float);
    }
    return set_status(FMA_OK, nullptr);
}

fma_status_t fma_qk_norm_rope_backward(fma_qk_plan_t p, int32_t batch, int64_t tokens, const fma_view_t *q,
                                       const fma_view_t *k, const float *gamma_q, const float *gamma_k,
                                       const int32_t *positions, const fma_view_t *g_q, const fma_view_t *g_k,
                                       const fma_view_t *g_v, const fma_view_t *dq, const fma_view_t *dk,
                                       const fma_view_t *dv, float *dgamma_q, float *dgamma_k, void *workspace,
                                       size_t workspace_bytes, void *stream)
{
    const char *fn = "fma_qk_norm_rope_backward";
    bool skip = false;
    fma_status_t st = check_sizes(fn, p, batch, tokens, &skip);
    if (st) return st;
    const fma_qk_desc_t &d = p->desc;
    if ((st = check_floats(fn, "dgamma_q", dgamma_q)) || (st = check_floats(fn, "dgamma_k", dgamma_k)) ||
        (st = check_floats(fn, "gamma_q", gamma_q)) || (st = check_floats(fn, "gamma_k", gamma_k)) ||
        (st = check_floats(fn, "positions", positions)))
        return st;
    QkArgs a;
    fill(p, a, batch, tokens);
    a.dgamma_q = dgamma_q;
    a.dgamma_k = dgamma_k;
    (void)hipGetLastError();
    if (skip) {   // no rows: the gammas' gradients are zero
        if (!dgamma_q && !dgamma_k) return set_status(FMA_OK, nullptr);
        return status_of(fn, launch_qk_backward(a, static_cast<hipStream_t>(stream)));
    }
    if (!g_v != !dv) return set_status(FMA_ERR_NULL, "%s: g_v and dv must be given together", fn);
    const int e = d.dtype == FMA_BF16 ? 2 : 4, ko = d.repeat_kv ? d.heads : d.kv_heads, n = dv ? 3 : 2;
    // (in check_apart's order: a gradient may take the place of the one it comes
    // from or of its own input)
    const View in[6] = {{g_q, batch, d.heads, tokens, d.head_dim, e, "g_q"},
                        {g_k, batch, ko, tokens, d.head_dim, e, "g_k"},
                        {n == 3 ? g_v : q, batch, n == 3 ? ko : d.heads, tokens, d.head_dim, e, n == 3 ? "g_v" : "q"},
                        {n == 3 ? q : k, batch, n == 3 ? d.heads : d.kv_heads, tokens, d.head_dim, e, n == 3 ? "q" : "k"},
                        {k, batch, d.kv_heads, tokens, d.head_dim, e, "k"}};
    const View out[3] = {{dq, batch, d.heads, tokens, d.head_dim, e, "dq"},
                         {dk, batch, d.kv_heads, tokens, d.head_dim, e, "dk"},
                         {dv, batch, d.kv_heads, tokens, d.head_dim, e, "dv"}};
    const int nin = n + 2;
    for (int i = 0; i < nin; ++i)
        if ((st = check_view(fn, in[i], false))) return st;
    for (int i = 0; i < n; ++i)
        if ((st = check_view(fn, out[i], true))) return st;
    if (d.axes == 2 && d.rotary_dim && !positions && d.side <= 0)
        return set_status(FMA_ERR_SHAPE, "%s: a map without positions needs the plan's side", fn);
    if ((st = check_apart(fn, out, n, in, nin, true))) return st;
    const int tasks = d.heads + (dv ? 2 : 1) * d.kv_heads;
    const size_t need = (size_t)qk_backward_groups(a.rows, tasks, d.head_dim) * 2 * d.head_dim * sizeof(float);
    if (!workspace || workspace_bytes < need)
        return set_status(FMA_ERR_WORKSPACE, "%s: workspace of %zu bytes, need %zu", fn,
                          workspace ? workspace_bytes : (size_t)0, need);
    if (!is_aligned(workspace, 16)) return set_status(FMA_ERR_ALIGN, "%s: workspace is not 16-byte aligned", fn);
    for (int i = 0; i < nin; ++i)
        if (ranges_meet(workspace, need, in[i].v->data, in[i].extent()))
            return set_status(FMA_ERR_ARG, "%s: workspace overlaps %s", fn, in[i].name);
    for (int i = 0; i < n; ++i)
        if (ranges_meet(workspace, need, out[i].v->data, out[i].extent()))
            return set_status(FMA_ERR_ARG, "%s: workspace overlaps %s", fn, out[i].name);
    a.q = device_view(q);
    a.k = device_view(k);
    a.qo = device_view(g_q);
    a.ko = device_view(g_k);
    a.dq = device_view(dq);
    a.dk = device_view(dk);
    a.has_v = dv != nullptr;
    if (dv) {
        a.vo = device_view(g_v);
        a.dv = device_view(dv);
    }
    a.gamma_q = gamma_q;
    a.gamma_k = gamma_k;
    a.pos = positions;
    a.part = static_cast<float *>(workspace);
    return status_of(fn, launch_qk_backward(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"

// api_status.hpp -- what the entry points in several files share: the calling
// thread's error message and checks of pointers and strided views.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fma.h"

namespace fma_dev {

// Keeps the message for fma_last_error() and returns st; without a format
// clears it and returns FMA_OK.
fma_status_t set_status(fma_status_t st, const char *fmt, ...) __attribute__((format(printf, 2, 3)));

inline fma_status_t status_of(const char *fn, hipError_t e)
{
    if (e != hipSuccess) return set_status(FMA_ERR_HIP, "%s: HIP error %d (%s)", fn, (int)e, hipGetErrorString(e));
    return set_status(FMA_OK, nullptr);
}

inline bool is_aligned(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

inline bool ranges_meet(const void *a, size_t na, const void *b, size_t nb)
{
    if (!a || !b || na == 0 || nb == 0) return false;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + nb && y < x + na;
}

// A view with its sizes: [batch][heads][tokens][dim] of esize bytes.
struct View {
    const fma_view_t *v;
    int64_t batch, heads, tokens;
    int dim, esize;
    const char *name;

    int64_t size(int a) const { return a == 0 ? batch : a == 1 ? heads : tokens; }
    int64_t stride(int a) const { return a == 0 ? v->batch_stride : a == 1 ? v->head_stride : v->token_stride; }
    // bytes from the first element to the end of the last
    size_t extent() const
    {
        int64_t n = dim;
        for (int a = 0; a < 3; ++a) n += (size(a) - 1) * stride(a);
        return (size_t)n * esize;
    }
    bool same(const View &o) const
    {
        if (v->data != o.v->data || batch != o.batch || heads != o.heads || tokens != o.tokens) return false;
        for (int a = 0; a < 3; ++a)
            if (size(a) > 1 && stride(a) != o.stride(a)) return false;
        return true;
    }
};

// Pointer, strides and (outputs) that no two rows share an element.
inline fma_status_t check_view(const char *fn, const View &x, bool output)
{
    if (!x.v || !x.v->data) return set_status(FMA_ERR_NULL, "%s: %s is NULL", fn, x.name);
    if (!is_aligned(x.v->data, 16)) return set_status(FMA_ERR_ALIGN, "%s: %s is not 16-byte aligned", fn, x.name);
    int64_t span = x.dim;   // elements that the axes seen so far reach over
    bool seen[3] = {false, false, false};
    for (int a = 0; a < 3; ++a) {
        if (x.size(a) <= 1) continue;
        if (x.stride(a) < 0) return set_status(FMA_ERR_SHAPE, "%s: %s has a negative stride", fn, x.name);
        if (x.stride(a) * x.esize % 16)
            return set_status(FMA_ERR_ALIGN, "%s: a stride of %s is not a multiple of 16 bytes", fn, x.name);
        if (x.stride(a) > INT64_MAX / 64 / x.size(a))
            return set_status(FMA_ERR_SHAPE, "%s: %s reaches past the address space", fn, x.name);
    }
    for (int k = 0; output && k < 3; ++k) {   // axes by growing stride
        int best = -1;
        for (int a = 0; a < 3; ++a)
            if (!seen[a] && x.size(a) > 1 && (best < 0 || x.stride(a) < x.stride(best))) best = a;
        if (best < 0) break;
        seen[best] = true;
        if (x.stride(best) < span)
            return set_status(FMA_ERR_ARG, "%s: rows of the output %s overlap", fn, x.name);
        span += (x.size(best) - 1) * x.stride(best);
    }
    return FMA_OK;
}

// Whether two views may share memory.  Views whose byte ranges meet still
// do not share any if they are heads of one packed row: equal token and batch
// strides, and heads that lie side by side within a token's row.
inline bool views_meet(const View &x, const View &y)
{
    if (!ranges_meet(x.v->data, x.extent(), y.v->data, y.extent())) return false;
    const int64_t row = x.tokens > 1 ? x.stride(2) : x.batch > 1 ? x.stride(0) : 0;
    if (row <= 0 || x.tokens != y.tokens || x.batch != y.batch) return true;
    for (int a = 0; a < 3; a += 2)
        if (x.size(a) > 1 && x.stride(a) != y.stride(a)) return true;
    if (x.tokens > 1 && x.batch > 1 && x.stride(0) < x.tokens * row) return true;
    const intptr_t apart = reinterpret_cast<intptr_t>(y.v->data) - reinterpret_cast<intptr_t>(x.v->data);
    const View &first = apart < 0 ? y : x, &second = apart < 0 ? x : y;
    const int64_t off = (apart < 0 ? -apart : apart) / x.esize;   // of the second's rows behind the first's
    auto length = [](const View &w) { return (w.heads > 1 ? (w.heads - 1) * w.stride(1) : 0) + w.dim; };
    return !(length(first) <= off && off + length(second) <= row);
}

}  // namespace fma_dev

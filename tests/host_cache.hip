// The paged cache's tiling, compiled for the host from the library's own header.
#include "cache.hpp"

using namespace fma_dev;

extern "C" void host_cache_tiling(int r, int S, int max_chunk, int rows, int tm, long long *out)
{
    CacheArgs a = {};
    a.r = r, a.S = S, a.max_chunk = max_chunk, a.rows = rows;
    const Tiling t = make_tiling(a, tm);
    out[0] = t.tm, out[1] = t.tpb, out[2] = t.per_seq, out[3] = t.units;
}

extern "C" int host_cache_tile_of(int r, int tm, int tpb, int pos)
{
    Tiling t = {};
    t.tm = tm, t.tpb = tpb;
    return tile_of(t, r, pos);
}

extern "C" void host_cache_route(int r, int group, int kv_heads, int max_chunk, int rows, int d, int bf16, int cus,
                                 int *out)
{
    CacheArgs a = {};
    a.head_dim = d, a.bf16 = bf16;
    a.r = r, a.group = group, a.kv_heads = kv_heads, a.max_chunk = max_chunk, a.rows = rows;
    const ChunkShape c = chunk_shape(a);
    out[0] = cache_route(a, cus), out[1] = c.gs, out[2] = c.split, out[3] = c.tm;
}

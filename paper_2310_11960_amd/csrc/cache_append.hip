// cache_append.hip -- new tokens into the paged cache: rows to their pages, and
// the summaries of the blocks that they complete.
//
// One workgroup per (touched block, key head) copies the block's new rows and, if
// the block is complete now, sums its rows per coarse set.  A chunk of more than
// a block can complete several: the sums over a group's blocks are then added
// up by a second pass, one block after the other.
#include "cache_device.hpp"

namespace fma_dev {

namespace {

constexpr int kThreads = 256;

template <bool BF16, int D>
__global__ __launch_bounds__(kThreads) void cache_append_kernel(CacheArgs a, Tiling t, int prior)
{
    __shared__ SumSmem<D, kThreads> sm;
    Tile x;
    if (!find_tile(a, t, blockIdx.x, x)) return;
    const int h = blockIdx.y, b = x.pos / a.r;
    const int page = page_of(a, x.seq, b);
    copy_rows<BF16, D, kThreads>(a, x, h, page);
    if (a.sets && (x.pos + x.n) % a.r == 0) summarize<BF16, D, kThreads>(a, x, h, b, page, prior != 0, sm);
}

// Block parts to running sums, in place: thread (sequence, head, column) walks
// the blocks that the call completed.
__global__ __launch_bounds__(kThreads) void cache_scan_kernel(CacheArgs a)
{
    const int seq = blockIdx.x, h = blockIdx.y;
    const int col = blockIdx.z * kThreads + threadIdx.x, cols = 2 * a.sets * a.head_dim;
    if (col >= cols) return;
    const int c0 = a.cu[seq], c1 = a.cu[seq + 1], s = a.start[seq];
    if (!sequence_fits(a, c0, c1, s)) return;
    const int l = col / a.head_dim % a.sets / a.rank;
    if (l == 0) return;   // a group of level 1 is one block
    const int b0 = s / a.r, b1 = (s + c1 - c0) / a.r;
    if (b0 == b1) return;
    auto at = [&](int b) -> float * {
        const int p = b >= 0 ? summary_of(a, seq, b) : -1;
        return p < 0 ? nullptr : a.sum + ((long long)p * a.kv_heads + h) * cols + col;
    };
    const float *const prev = at(b0 - 1);
    float acc = prev ? *prev : 0.f;
    for (int b = b0; b < b1; ++b) {
        float *const p = at(b);
        const float own = p ? *p : 0.f;
        acc = b & ((1 << l) - 1) ? acc + own : own;
        if (p) *p = acc;
        else acc = 0.f;
    }
}

template <bool BF16, int D>
hipError_t append_d(const CacheArgs &a, hipStream_t st)
{
    const Tiling t = make_tiling(a, a.r);
    const bool single = a.max_chunk <= a.r;   // a chunk completes one block at most
    hipLaunchKernelGGL((cache_append_kernel<BF16, D>), dim3((unsigned)t.units, a.kv_heads), dim3(kThreads), 0, st, a, t,
                       (int)single);
    if (!single && a.levels > 1)
        hipLaunchKernelGGL(cache_scan_kernel, dim3(a.S, a.kv_heads, (2 * a.sets * D + kThreads - 1) / kThreads),
                           dim3(kThreads), 0, st, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_append(const CacheArgs &a, hipStream_t st)
{
    if (a.S == 0 || a.rows == 0 || a.max_chunk == 0) return hipSuccess;
    switch (a.head_dim) {
    case 32: return a.bf16 ? append_d<true, 32>(a, st) : append_d<false, 32>(a, st);
    case 64: return a.bf16 ? append_d<true, 64>(a, st) : append_d<false, 64>(a, st);
    case 128: return a.bf16 ? append_d<true, 128>(a, st) : append_d<false, 128>(a, st);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace fma_dev

// cache_append.hip -- new tokens into the paged cache: rows to their pages, and
// the summaries of the blocks that they complete.
//
// Where no chunk is longer than a block, a chunk completes one block at most and
// one workgroup per (touched block, key head) writes its sums at once
// (summarize).  Longer chunks take two passes:
//   1. a wave per (touched block, key head, keys or values) streams the block's
//      rows, to the page and through LDS into matrix products: the block's part
//      of every set is X^T W^T, W [sets][r] the block's piece of the weights;
//   2. the parts become running sums over the blocks of a group, in place.
//
// What bounds it: bytes.  The rows are read once and written once; the weights
// (r floats per set) come from L2.
#include "cache_device.hpp"

namespace fma_dev {

namespace {

constexpr int kThreads = 256;

template <bool BF16, int D>
__global__ __launch_bounds__(kThreads) void cache_append_kernel(CacheArgs a, Tiling t)
{
    __shared__ __attribute__((aligned(16))) char lds[kThreads / 64][kSumTile<BF16>];
    Tile x;
    const CacheGroup g = cache_group(a.kv_heads);
    if (!find_tile(a, t, g.unit, x)) return;
    const int h = g.head, b = x.pos / a.r;
    const int page = page_of(a, x.seq, b);
    copy_rows<BF16, D, kThreads>(a, x, h, page);
    if (!a.sets || (x.pos + x.n) % a.r) return;
    const int dst = summary_of(a, x.seq, b), before = b > 0 ? summary_of(a, x.seq, b - 1) : -1;
    if (dst >= 0) summarize<BF16, D, kThreads / 64>(a, x, h, b, page, dst, before, lds[threadIdx.x >> 6]);
}

// Pass 1.  Workgroup: a block and two key heads (waves 0, 1: keys, values of the
// first, ..).  32 rows at a time; the next tile's rows are on their way while
// one is multiplied.
template <bool BF16, int D>
__global__ __launch_bounds__(kThreads) void cache_blocks_kernel(CacheArgs a, Tiling t)
{
    constexpr int ND = D / 32;
    __shared__ __attribute__((aligned(16))) char lds[kThreads / 64][32 * D * (BF16 ? 2 : 4)];
    Tile x;
    const CacheGroup g = cache_group((a.kv_heads + 1) / 2);
    if (!find_tile(a, t, g.unit, x)) return;
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = 2 * g.head + (wave >> 1), kv = wave & 1;
    if (h >= a.kv_heads) return;
    const int b = x.pos / a.r;
    const bool done = a.sets && x.pos + x.n == (b + 1) * a.r;
    const int dst = done ? summary_of(a, x.seq, b) : -1;
    char *const tile = lds[wave];
    BlockRows<BF16, D, D> rows(a, x, h, kv, page_of(a, x.seq, b), 0, lane);

    for (int s0 = 0; s0 == 0 || s0 < a.sets; s0 += 32) {
        const bool col = dst >= 0 && s0 + l32 < a.sets;
        const float *const w = col ? block_weights(a, kv, h, s0 + l32, b) : nullptr;
        f32x16 o[ND];
#pragma unroll
        for (int db = 0; db < ND; ++db) o[db] = f32x16{0};
        rows.fetch(0, dst >= 0);
        for (int row0 = 0; row0 < a.r; row0 += 32) {
            float wf[16];
            if (dst >= 0) {
                tile_weights(w, col, row0, a.r, hh, wf);
                rows.stage(tile);
            }
            if (s0 == 0) rows.keep(row0, x.pos);
            if (row0 + 32 < a.r) rows.fetch(row0 + 32, dst >= 0);
            if (dst >= 0) tile_sums<BF16, D>(tile, wf, lane, o);
        }
        if (dst < 0) break;
        if (col) {
            float *const to = a.sum + ((((long long)dst * a.kv_heads + h) * 2 + kv) * a.sets + s0 + l32) * D;
#pragma unroll
            for (int db = 0; db < ND; ++db)
#pragma unroll
                for (int j = 0; j < 16; j += 4)
                    *reinterpret_cast<f32x4 *>(to + 32 * db + grow(j, hh)) = f32x4{o[db][j], o[db][j + 1], o[db][j + 2], o[db][j + 3]};
        }
    }
}

// Pass 2: a thread per channel of a set walks the blocks that the call completed,
// kScan of them on their way at a time (a wave's block is uniform).  Runs of
// kScan blocks that start at a multiple of kScan hold whole groups of up to kScan
// blocks and go to workgroups of their own; the levels above are walked from run
// to run by the first of them.
// Two prompts of 98K tokens together, 16 heads: 93 us with 16 blocks on their
// way, 53 with 64, XX with the runs apart.
__global__ __launch_bounds__(kThreads) void cache_scan_kernel(CacheArgs a, int runs)
{
    const int seq = blockIdx.x / (unsigned)runs, run = blockIdx.x - seq * runs, h = blockIdx.y, lane = threadIdx.x & 63;
    const int cols = 2 * a.sets * a.head_dim, at = blockIdx.z * kThreads + threadIdx.x;
    const int col = at < cols ? at : 0;   // (whole waves stay: every lane holds a block's page)
    const int c0 = listed(a.cu, seq), c1 = listed(a.cu, seq + 1), s = listed(a.start, seq);
    if (!sequence_fits(a, c0, c1, s)) return;
    const int l = col / a.head_dim % a.sets / a.rank;
    const int first = s / a.r, b1 = (s + c1 - c0) / a.r, run0 = (first / kScan + run) * kScan;
    const bool tall = (1 << l) > kScan;
    bool live = at < cols && l > 0 && (!tall || run == 0);   // a group of level 1 is one block
    float *const base = a.sum + (long long)h * cols;
    const long long page = (long long)a.kv_heads * cols;
    float acc = 0.f;
    if (run == 0 && first > 0) {
        const int prev = summary_of(a, seq, first - 1);
        if (prev >= 0) acc = (base + prev * page)[col];
    }
    for (int b = run == 0 ? first : run0; b < b1;) {
        const int end = b / kScan * kScan + kScan;   // the walk's pieces end with the runs
        const int n = (end < b1 ? end : b1) - b;
        const int mine = lane < n ? summary_of(a, seq, b + lane) : -1;   // lane i: page of block b + i
        float own[kScan];
#pragma unroll
        for (int i = 0; i < kScan; ++i) {
            own[i] = 0.f;
            const int p = __builtin_amdgcn_readlane(mine, i);
            if (p >= 0 && live) own[i] = (base + p * page)[col];
        }
#pragma unroll
        for (int i = 0; i < kScan; ++i) {
            const int p = __builtin_amdgcn_readlane(mine, i);
            acc = (b + i) & ((1 << l) - 1) ? acc + own[i] : own[i];
            if (p < 0)
                acc = 0.f;   // the sums of a missing page count as zero (and none follows the last block)
            else if (live)
                (base + p * page)[col] = acc;
        }
        live = live && tall;
        if (__builtin_amdgcn_ballot_w64(live) == 0) break;
        b = end;
    }
}

template <bool BF16, int D>
hipError_t append_d(const CacheArgs &a, hipStream_t st)
{
    const Tiling t = make_tiling(a, a.r);
    if (a.max_chunk <= a.r) {
        hipLaunchKernelGGL((cache_append_kernel<BF16, D>), dim3((unsigned)(t.units * a.kv_heads)), dim3(kThreads), 0, st, a, t);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((cache_blocks_kernel<BF16, D>), dim3((unsigned)(t.units * ((a.kv_heads + 1) / 2))), dim3(kThreads),
                       0, st, a, t);
    if (a.levels > 1)
        hipLaunchKernelGGL(cache_scan_kernel, dim3((unsigned)a.S * scan_runs(a), a.kv_heads, (2 * a.sets * D + kThreads - 1) / kThreads),
                           dim3(kThreads), 0, st, a, scan_runs(a));
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_append(const CacheArgs &a, hipStream_t st)
{
    switch (a.head_dim) {
    case 32: return a.bf16 ? append_d<true, 32>(a, st) : append_d<false, 32>(a, st);
    case 64: return a.bf16 ? append_d<true, 64>(a, st) : append_d<false, 64>(a, st);
    case 128: return a.bf16 ? append_d<true, 128>(a, st) : append_d<false, 128>(a, st);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace fma_dev

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
// blocks and go to workgroups of their own.  Groups of more blocks (tall ones):
//   SCAN_ALL     the first run's workgroup walks on through the others;
//   or, for chunks of several runs,
//   SCAN_TOTALS  every run that another follows leaves its total in its last
//                block's row,
//   SCAN_CHAIN   one thread per channel makes these the sums at the runs' ends,
//   SCAN_RUNS    every run starts from the sum at the end of the one before.
// Two prompts of 98K tokens together, 16 heads: 93 us with 16 blocks on their
// way, 53 with 64, 59 with the runs apart and tall groups walked, 39 in three steps.
enum ScanStep { SCAN_ALL, SCAN_TOTALS, SCAN_CHAIN, SCAN_RUNS };

// blocks b .. b + n - 1 of a channel on their way: mine, lane i's page of block b + i
__device__ __attribute__((always_inline)) inline void scan_fetch(const float *base, long long page, int col, int mine, int n,
                                                                 bool live, float (&own)[kScan])
{
#pragma unroll
    for (int i = 0; i < kScan; i += 8) {
        if (i < n) {
#pragma unroll
            for (int k = i; k < i + 8; ++k) {
                const int p = __builtin_amdgcn_readlane(mine, k);
                own[k] = p >= 0 && live ? (base + p * page)[col] : 0.f;
            }
        }
    }
}

template <int STEP>
__global__ __launch_bounds__(kThreads) void cache_scan_kernel(CacheArgs a, int runs)
{
    const int per = STEP == SCAN_CHAIN ? 1 : runs;   // workgroups along a sequence
    const int seq = blockIdx.x / (unsigned)per, run = blockIdx.x - seq * per, h = blockIdx.y, lane = threadIdx.x & 63;
    const int cols = 2 * a.sets * a.head_dim, at = blockIdx.z * kThreads + threadIdx.x;
    const int col = at < cols ? at : 0;   // (whole waves stay: every lane holds a block's page)
    const int c0 = listed(a.cu, seq), c1 = listed(a.cu, seq + 1), s = listed(a.start, seq);
    if (!sequence_fits(a, c0, c1, s)) return;
    const int l = col / a.head_dim % a.sets / a.rank;
    const int first = s / a.r, b1 = (s + c1 - c0) / a.r, run0 = (first / kScan + run) * kScan;
    const bool tall = (1 << l) > kScan;
    bool live = at < cols && l > 0;   // a group of level 1 is one block
    float *const base = a.sum + (long long)h * cols;
    const long long page = (long long)a.kv_heads * cols;
    auto sum_at = [&](int b) {
        const int p = b >= 0 ? summary_of(a, seq, b) : -1;
        return p >= 0 ? (base + p * page)[col] : 0.f;
    };
    float own[kScan];
    if constexpr (STEP == SCAN_CHAIN) {
        live = live && tall;
        if (__builtin_amdgcn_ballot_w64(live) == 0) return;
        // the ends of the runs that others follow, kScan at a time
        float acc = 0.f;
        for (int e = run0 + kScan - 1; e < b1 - 1; e += kScan * kScan) {
            const int end = e + lane * kScan, mine = end < b1 - 1 ? summary_of(a, seq, end) : -1;
            const int n = (b1 - 2 - e) / kScan + 1 < kScan ? (b1 - 2 - e) / kScan + 1 : kScan;
            scan_fetch(base, page, col, mine, n, live, own);
#pragma unroll
            for (int i = 0; i < kScan; i += 8) {
                if (i < n) {
#pragma unroll
                    for (int k = i; k < i + 8; ++k) {
                        if (k >= n) continue;
                        const int p = __builtin_amdgcn_readlane(mine, k);
                        // (the run of end e + k kScan starts a group, or goes on with one)
                        acc = (e + (k - 1) * kScan + 1) & ((1 << l) - 1) ? acc + own[k] : own[k];
                        if (p < 0)
                            acc = 0.f;
                        else if (live)
                            (base + p * page)[col] = acc;
                    }
                }
            }
        }
        return;
    }
    int b = run == 0 ? first : run0;
    if (b >= b1) return;
    if constexpr (STEP == SCAN_TOTALS) live = live && tall && b / kScan * kScan + kScan < b1;
    if constexpr (STEP == SCAN_ALL) live = live && (!tall || run == 0);
    if (__builtin_amdgcn_ballot_w64(live) == 0) return;
    // the sum before the piece, where a group goes on through its start
    float acc = live && (b & ((1 << l) - 1)) && (run == 0 || STEP == SCAN_RUNS) ? sum_at(b - 1) : 0.f;
    while (b < b1) {
        const int end = b / kScan * kScan + kScan;   // the walk's pieces end with the runs
        const int n = (end < b1 ? end : b1) - b;
        const int mine = lane < n ? summary_of(a, seq, b + lane) : -1;
        const int keep = STEP == SCAN_RUNS && tall && end < b1 ? n - 1 : n;   // (a run's end is there already)
        scan_fetch(base, page, col, mine, n, live, own);
#pragma unroll
        for (int i = 0; i < kScan; i += 8) {
            if (i < n) {
#pragma unroll
                for (int k = i; k < i + 8; ++k) {
                    if (k >= n) continue;
                    const int p = __builtin_amdgcn_readlane(mine, k);
                    acc = (b + k) & ((1 << l) - 1) ? acc + own[k] : own[k];
                    if (p < 0)
                        acc = 0.f;   // the sums of a missing page count as zero
                    else if (live && (STEP == SCAN_TOTALS ? k == n - 1 : k < keep))
                        (base + p * page)[col] = acc;
                }
            }
        }
        live = live && tall && STEP == SCAN_ALL;
        if (__builtin_amdgcn_ballot_w64(live) == 0) break;
        b = end;
    }
}

template <int STEP>
void launch_scan(const CacheArgs &a, int runs, hipStream_t st)
{
    const dim3 grid((unsigned)a.S * (STEP == SCAN_CHAIN ? 1 : runs), a.kv_heads, (2 * a.sets * a.head_dim + kThreads - 1) / kThreads);
    hipLaunchKernelGGL((cache_scan_kernel<STEP>), grid, dim3(kThreads), 0, st, a, runs);
}

void launch_scans(const CacheArgs &a, hipStream_t st)
{
    const int runs = scan_runs(a);
    if (runs > 3 && (1 << (a.levels - 1)) > kScan) {
        launch_scan<SCAN_TOTALS>(a, runs, st);
        launch_scan<SCAN_CHAIN>(a, runs, st);
        launch_scan<SCAN_RUNS>(a, runs, st);
    } else {
        launch_scan<SCAN_ALL>(a, runs, st);
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
    if (a.levels > 1) launch_scans(a, st);
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

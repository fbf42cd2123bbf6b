// cache.hpp -- arguments, launchers and shared device code of the paged cache
// (internal to the library).
#pragma once

#include "fma_device.hpp"

namespace fma_dev {

struct CacheArgs {
    // rows of tokens: element strides of tokens and heads
    const void *q, *k, *v;         // k == NULL: every key is in the pages
    void *out;
    int write;                     // the attention's launch puts k and v into the pages as well
    long long qt, qh, kt, kh, vt, vh, ot, oh;
    void *kp, *vp;                 // pages [npages][kv_heads][r][d]
    float *sum;                    // summary pages [nsums][kv_heads][2][sets][d]
    long long npages, nsums;
    const int32_t *table, *stable; // [S][tstride]
    long long tstride;
    const int32_t *cu, *start;
    const float *wk, *wv;
    long long w_stride;            // floats between heads' weights (0 = shared)
    int S, max_chunk, rows, limit; // limit: longest sequence that fits
    int heads, kv_heads, group;    // group: query heads of a key head
    int r, rank, levels, sets;
    int head_dim, bf16;
    float scale_log2;              // softmax scale * log2(e)
};

// How a launch's workgroups meet the sequences' tokens: tiles of tm positions
// that do not cross base blocks, tpb of them per block.
struct Tiling {
    int tm, tpb;
    int per_seq;   // > 0: workgroup u takes tile u % per_seq of sequence u / per_seq; 0: it searches
    long long units;
};

__host__ __device__ inline int tile_of(const Tiling &t, int r, int pos) { return pos / r * t.tpb + pos % r / t.tm; }

// Tiles of tm positions over chunks of at most a.max_chunk tokens.  A chunk of w
// tokens meets 1 + ceil((w - 1) / tm) tiles at most where tiles of tm fill a
// block; where a block ends with a shorter one, no more than w tpb / r + 3; so
// rows / tm + 2 S (rows tpb / r + 3 S) bound any batch, and a tile has at least one
// row.  One tile range per sequence, without a search, where that leaves at most
// twice as many idle workgroups.
inline Tiling make_tiling(const CacheArgs &a, int tm)
{
    Tiling t;
    t.tm = tm < a.r ? tm : a.r;
    t.tpb = (a.r + t.tm - 1) / t.tm;
    const bool even = t.tpb * t.tm == a.r;
    const long long most = a.max_chunk < a.rows ? a.max_chunk : a.rows;
    long long each = even ? (most + t.tm - 2) / t.tm + 1 : most * t.tpb / a.r + 3;
    if (each > most) each = most;
    long long bound = even ? a.rows / t.tm + 2LL * a.S : (long long)a.rows * t.tpb / a.r + 3LL * a.S;
    if (bound > a.rows) bound = a.rows;
    t.per_seq = each * a.S <= 2 * bound + 64 ? (int)each : 0;
    t.units = t.per_seq ? each * a.S : bound;
    return t;
}

// Which kernel attends:
//   TOKENS  at most token_rows(a) query rows meet a key head's rows, too few for a
//           32-column matrix operand: the vector ALU (cache_token.hip).  64
//           sequences, TOKENS against KEYS: one row 20.8 against 40.8 us (fp32),
//           two rows 16.1 against 19.9 (bf16, d = 64), four rows 20.4 against 23.6
//           (d = 128) and 13.8 against 18.0 (fp32), but 14.8 against 12.3 (bf16,
//           d = 64: the products of eight channels cost more than the loads);
//   KEYS    32 rows a workgroup, whose waves take different keys
//           (cache_attend.hip): pieces whose rows with one key head fit one
//           such tile, and calls whose workgroups all run at once, or nearly;
//   ROWS    128 rows a workgroup, whose waves take different rows and share the
//           keys in LDS (cache_chunk.hip).
// Which of these two, by workgroups of ROWS in eighths of the CUs (a workgroup of
// KEYS has a quarter of the rows; its registers leave room for three or four on a
// CU at d = 32, two at 64, one at 128).  One piece, r = 128, KEYS against ROWS in
// us, at 256 CUs:
//   bf16, d = 32:   192 24.4 against 27.6, 224 28.5 against 28.3
//         d = 64:   128 27.7 against 31.2, 144 34.3 against 32.2, 192 37.2 against 32.8
//         d = 128:   64 36.8 against 41.4,  80 48.2 against 41.9, 192 66.4 against 44.2
//   fp32, d = 64:   160 54.2 against 56.6, 192 61.2 against 57.9
//         d = 128:  128 92.8 against 98.0, 144  110 against 98.6
// The first two put new tokens into the cache as well, where no chunk is longer
// than a block (the far field of such a chunk has nothing of its own).
enum CacheRoute { CACHE_TOKENS, CACHE_KEYS, CACHE_ROWS };

// Query heads of a workgroup and workgroups per key head; the tile of CACHE_ROWS.
struct ChunkShape {
    int gs, split, tm;
};
inline ChunkShape chunk_shape(const CacheArgs &a)
{
    ChunkShape c;
    c.split = (a.group + 31) / 32;
    c.gs = (a.group + c.split - 1) / c.split;
    int tpb = (a.r * c.gs + 127) / 128;   // equal tiles of at most 128 rows
    while ((a.r + tpb - 1) / tpb * c.gs > 128) ++tpb;
    c.tm = (a.r + tpb - 1) / tpb;
    return c;
}

inline int token_rows(const CacheArgs &a) { return a.bf16 && a.head_dim <= 64 ? 2 : 4; }

inline int keys_eighths(const CacheArgs &a)
{
    if (a.head_dim == 32) return 7;
    return a.bf16 ? (a.head_dim == 64 ? 4 : 2) : (a.head_dim == 64 ? 5 : 4);
}

inline CacheRoute cache_route(const CacheArgs &a, int cus)
{
    const long long most = a.max_chunk < a.rows ? a.max_chunk : a.rows;
    if (most * a.group <= token_rows(a)) return CACHE_TOKENS;
    const ChunkShape c = chunk_shape(a);
    const long long groups = (long long)a.rows * c.gs / (c.tm * c.gs < 128 ? c.tm * c.gs : 128) * a.kv_heads * c.split;
    return most * c.gs <= 32 || 8 * groups <= (long long)keys_eighths(a) * cus ? CACHE_KEYS : CACHE_ROWS;
}

// Workgroups are numbered tile by tile, a tile's key heads one after the other: a
// sequence that has more to do than others (a finished block's sums) is not
// last with every head, and with a multiple of eight heads the neighbouring
// tiles of one head, which share rows, meet in one XCD's L2.
struct CacheGroup {
    unsigned unit;
    int head;
};
__device__ inline CacheGroup cache_group(int heads)
{
    CacheGroup g;
    g.unit = blockIdx.x / (unsigned)heads;
    g.head = (int)(blockIdx.x - g.unit * (unsigned)heads);
    return g;
}

// Tile positions of the launches and the key-head parts of a tile.
inline int token_tile(const CacheArgs &a) { return a.max_chunk < a.rows ? a.max_chunk : a.rows; }
inline int keys_tile(const ChunkShape &c) { return 32 / c.gs; }

// Runs of kScan aligned blocks that a chunk's complete blocks can touch.
constexpr int kScan = 64;   // lanes of a wave
inline int scan_runs(const CacheArgs &a)
{
    const int most = (a.max_chunk < a.rows ? a.max_chunk : a.rows) / a.r + 1;
    return (most + kScan - 1) / kScan + 1;
}

// Threads of a launch stay below 2^32.
inline bool cache_launches_fit(const CacheArgs &a, bool appends, bool attends, int cus)
{
    auto fits = [&](int tm, long long heads, int threads) {
        return make_tiling(a, tm).units <= 0xffffffffLL / threads / heads;
    };
    if (appends && (!fits(a.r, a.kv_heads, 256) || (long long)a.S * scan_runs(a) >= 1 << 24)) return false;
    if (!attends) return true;
    const ChunkShape c = chunk_shape(a);
    switch (cache_route(a, cus)) {
    case CACHE_TOKENS: return fits(token_tile(a), a.kv_heads, 512);
    case CACHE_KEYS: return fits(keys_tile(c), (long long)a.kv_heads * c.split, 512);
    default: return fits(c.tm, (long long)a.kv_heads * c.split, 256);
    }
}

hipError_t launch_cache_append(const CacheArgs &a, hipStream_t st);
hipError_t launch_cache_token(const CacheArgs &a, hipStream_t st);
hipError_t launch_cache_keys(const CacheArgs &a, const ChunkShape &c, int cus, hipStream_t st);
hipError_t launch_cache_rows(const CacheArgs &a, const ChunkShape &c, hipStream_t st);

// A workgroup's tile: positions [pos, pos + n) of sequence seq, the first in row
// `row` of the call's tensors.
struct Tile {
    int seq, pos, n, row;
    int start, end;     // tokens of the sequence before and after the call
    int row0;           // row of its first new token
};

// lengths and tables, which no kernel writes: scalar loads where the index is uniform
__device__ inline int listed(const int32_t *p, long long i)
{
    return ((const __attribute__((address_space(4))) int32_t *)(uintptr_t)p)[i];
}

__device__ inline bool sequence_fits(const CacheArgs &a, int c0, int c1, int s)
{
    return c0 >= 0 && c1 > c0 && c1 <= a.rows && c1 - c0 <= a.max_chunk && s >= 0 && s <= a.limit - (c1 - c0);
}

__device__ inline bool find_tile(const CacheArgs &a, const Tiling &t, unsigned unit, Tile &x)
{
    int c0 = 0, s = 0, len = 0, idx = 0;
    if (t.per_seq) {
        x.seq = unit / (unsigned)t.per_seq;
        idx = unit - x.seq * t.per_seq;
        c0 = listed(a.cu, x.seq);
        const int c1 = listed(a.cu, x.seq + 1);
        s = listed(a.start, x.seq);
        if (!sequence_fits(a, c0, c1, s)) return false;
        len = c1 - c0;
        if (idx > tile_of(t, a.r, s + len - 1) - tile_of(t, a.r, s)) return false;
    } else {
        // 64 sequences at a time: their tile counts, a running sum over the
        // lanes, and the first lane whose sum passes the unit
        const int lane = threadIdx.x & 63;
        int before = 0;
        bool found = false;
        for (int base = 0; base < a.S; base += 64) {
            const int i = base + lane;
            int n = 0, d0 = 0, d1 = 0, ds = 0;
            if (i < a.S) {
                d0 = a.cu[i];
                d1 = a.cu[i + 1];
                ds = a.start[i];
                if (sequence_fits(a, d0, d1, ds)) n = tile_of(t, a.r, ds + d1 - d0 - 1) - tile_of(t, a.r, ds) + 1;
            }
            int sum = n;
#pragma unroll
            for (int k = 1; k < 64; k *= 2) {
                const int y = __shfl_up(sum, k);
                if (lane >= k) sum += y;
            }
            const uint64_t past = __builtin_amdgcn_ballot_w64(before + sum > (int)unit);
            if (past) {
                const int l = __builtin_ctzll(past);
                x.seq = base + l;
                idx = (int)unit - before - __shfl(sum - n, l);
                c0 = __shfl(d0, l);
                len = __shfl(d1, l) - c0;
                s = __shfl(ds, l);
                found = true;
                break;
            }
            before += __shfl(sum, 63);
        }
        if (!found) return false;
    }
    const int tile = tile_of(t, a.r, s) + idx;
    const int b = tile / t.tpb, lo = b * a.r + (tile - b * t.tpb) * t.tm;
    int hi = lo + t.tm < (b + 1) * a.r ? lo + t.tm : (b + 1) * a.r;
    if (hi > s + len) hi = s + len;
    // (uniform, whichever way it was found: scalar registers for all that follows)
    auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    x.seq = uniform(x.seq);
    x.pos = uniform(lo > s ? lo : s);
    x.n = uniform(hi) - x.pos;
    x.start = uniform(s);
    x.end = uniform(s + len);
    x.row0 = uniform(c0);
    x.row = x.row0 + x.pos - x.start;
    return true;
}

// page of block b (-1: missing)
__device__ inline int page_of(const CacheArgs &a, int seq, int b)
{
    const int p = listed(a.table, seq * a.tstride + b);
    return p >= 0 && p < a.npages ? p : -1;
}
__device__ inline int summary_of(const CacheArgs &a, int seq, int b)
{
    const int p = listed(a.stable, seq * a.tstride + b);
    return p >= 0 && p < a.nsums ? p : -1;
}

}  // namespace fma_dev

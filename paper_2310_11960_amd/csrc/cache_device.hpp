// cache_device.hpp -- rows of the paged cache, and what entering tokens leave
// behind: page copies and the block summaries.
#pragma once

#include "cache.hpp"
#include "lds_rows.hpp"
#include "row_lanes.hpp"

namespace fma_dev {

namespace {

// Key or value row of position `pos` in the caller's tensors or its page.
__device__ inline long long page_row(const CacheArgs &a, int page, int h, int in)
{
    return (((long long)page * a.kv_heads + h) * a.r + in) * a.head_dim;
}

template <bool BF16>
__device__ inline const void *elem(const void *p, long long off)
{
    return static_cast<const char *>(p) + off * (BF16 ? 2 : 4);
}
template <bool BF16>
__device__ inline void *elem(void *p, long long off)
{
    return static_cast<char *>(p) + off * (BF16 ? 2 : 4);
}

template <bool BF16>
__device__ inline void load8f(const void *p, float (&x)[8])
{
    floats<BF16>(load_raw<BF16>(p), x);
}

// Rows 0 .. 31 of a tile that a lane's query sees, as bits: those of `there` up to
// row `last`; shifted so that accumulator element j of lane half hh is bit
// 8 (j >> 2) + (j & 3).
__device__ inline uint32_t seen_rows(uint32_t there, int last, int hh)
{
    const uint32_t upto = last >= 31 ? ~0u : last < 0 ? 0u : (2u << last) - 1;
    return (there & upto) >> (4 * hh);
}
__device__ inline bool seen(uint32_t rows, int j) { return rows >> (8 * (j >> 2) + (j & 3)) & 1u; }

// The far field of queries in block b: level by level group q - 2 and (odd q)
// group q - 3, each with all bases; groups that a finer level covers and
// empty levels take no place in the list.
struct FarList {
    int b, levels, n;
    __device__ FarList(const CacheArgs &a, int b_)
    {
        const int lq = b_ >= 2 ? 31 - __builtin_clz((unsigned)b_) : 0;
        b = b_;
        levels = lq < a.levels ? lq : a.levels;
        n = a.rank * (levels + __popc(b & ((1 << levels) - 1)));
    }
    // key row of source i (the value row is sets * D floats on); NULL if its page is missing
    __device__ const float *row(const CacheArgs &a, int seq, int h, int i) const
    {
        if (i >= n) return nullptr;
        int lv = 0, c = a.rank << (b & 1);
        while (i >= c) {
            i -= c;
            ++lv;
            c = a.rank << (b >> lv & 1);
        }
        const int two = i >= a.rank, g = (b >> lv) - 2 - two;
        const int sp = summary_of(a, seq, ((g + 1) << lv) - 1);
        if (sp < 0) return nullptr;
        return a.sum + (((long long)sp * a.kv_heads + h) * 2 * a.sets + lv * a.rank + i - two * a.rank) * a.head_dim;
    }
};

// A tile's new rows of key head h into their page (all in one block), NT threads.
template <bool BF16, int D, int NT>
__device__ inline void copy_rows(const CacheArgs &a, const Tile &x, int h, int page)
{
    if (page < 0) return;
    constexpr int C = D * (BF16 ? 2 : 4) / 16;   // 16-byte pieces of a row
    const int in = x.pos % a.r;
    for (int i = threadIdx.x; i < x.n * C; i += NT) {
        const int j = i / C, c = i % C;
        const uint4 k = static_cast<const uint4 *>(elem<BF16>(a.k, (x.row + j) * a.kt + h * a.kh))[c];
        const uint4 v = static_cast<const uint4 *>(elem<BF16>(a.v, (x.row + j) * a.vt + h * a.vh))[c];
        const long long o = page_row(a, page, h, in + j);
        static_cast<uint4 *>(elem<BF16>(a.kp, o))[c] = k;
        static_cast<uint4 *>(elem<BF16>(a.vp, o))[c] = v;
    }
}

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));   // the caller's weights

// One wave's share of a block's sums: C channels of the block's rows (keys or
// values of head h), 32 rows at a time, against the weights of 32 sets,
//   o[db] += X^T W^T      (rows: channels 32 db .., columns: sets),
// on the matrix cores.  fp32 weights meet bf16 rows exactly: each weight is
// split into three bf16 terms (8 + 8 + 8 bits), so the sums keep fp32 accuracy.
template <bool BF16, int D, int C>
struct BlockRows {
    static constexpr int LPR = C / 8, RPL = 64 / LPR, NL = 32 / RPL;   // rows of a load, loads of a tile
    static constexpr int RB = D * (BF16 ? 2 : 4), TB = C * (BF16 ? 2 : 4), LB = TB / LPR;   // bytes of a row, in a tile, a lane
    const char *in;        // row of position x.start + i at in + i * in_t
    char *pg;              // the block's page (rows of RB bytes)
    long long in_t;
    int page, pos_b, start, end, r, lr, lc;
    Raw8<BF16> raw[NL];

    __device__ BlockRows(const CacheArgs &a, const Tile &x, int h, int kv, int page_, int c0, int lane)   // c0: first channel
    {
        page = page_;
        pos_b = x.pos / a.r * a.r;
        start = x.start;
        end = x.pos + x.n;
        r = a.r;
        in_t = (kv ? a.vt : a.kt) * (BF16 ? 2 : 4);
        lr = lane / LPR;
        lc = lane % LPR;
        in = static_cast<const char *>(elem<BF16>(kv ? a.v : a.k, h * (kv ? a.vh : a.kh) + c0)) + x.row0 * in_t;
        pg = static_cast<char *>(elem<BF16>(kv ? a.vp : a.kp, page_row(a, page, h, 0) + c0));
    }
    __device__ int row_of(int row0, int i) const { return row0 + i * RPL + lr; }
    // rows row0 .. of the block, zero where there is none; old: with those from before the call
    __device__ void fetch(int row0, bool old)
    {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int row = row_of(row0, i), pos = pos_b + row;
            raw[i] = Raw8<BF16>();
            if (row >= r) continue;   // (r = 16: half a tile)
            if (pos >= start) {
                if (pos < end) raw[i] = load_raw<BF16>(in + (long long)(pos - start) * in_t + LB * lc);
            } else if (page >= 0 && old) {
                raw[i] = load_raw<BF16>(pg + row * RB + LB * lc);
            }
        }
    }
    // the new ones (from `first` on) to the page
    __device__ void keep(int row0, int first) const
    {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int row = row_of(row0, i), pos = pos_b + row;
            if (row < r && pos >= first && pos < end && page >= 0) store_raw<BF16>(pg + row * RB + LB * lc, raw[i]);
        }
    }
    // to a wave's LDS tile of 32 rows (bf16: chunks swizzled for the transposing reads)
    __device__ void stage(char *tile) const
    {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int tr = i * RPL + lr;
            if constexpr (BF16) {
                *reinterpret_cast<uint4 *>(tile + tr * TB + 16 * (lc ^ swzd<C>(tr))) =
                    make_uint4(raw[i].w[0], raw[i].w[1], raw[i].w[2], raw[i].w[3]);
            } else {
                float f[8];
                floats<BF16>(raw[i], f);
                f32x4 *to = reinterpret_cast<f32x4 *>(tile + tr * TB + 32 * lc);
                to[0] = f32x4{f[0], f[1], f[2], f[3]};
                to[1] = f32x4{f[4], f[5], f[6], f[7]};
            }
        }
    }
};

// weights of set e for the rows of block b
__device__ inline const float *block_weights(const CacheArgs &a, int kv, int h, int e, int b)
{
    const int l = e / a.rank, s = e - l * a.rank;
    const long long size = (long long)a.r << l;
    return (kv ? a.wv : a.wk) + h * a.w_stride + a.rank * (size - a.r) + s * size + (long long)(b & ((1 << l) - 1)) * a.r;
}

// this lane's weights of a tile: rows 8 i + 4 (lane >> 5) + j of it in w[4 i + j]
__device__ inline void tile_weights(const float *w, bool col, int row0, int r, int hh, float (&wf)[16])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f32x4u x = {0.f, 0.f, 0.f, 0.f};
        if (col && row0 + 8 * i < r) x = *reinterpret_cast<const f32x4u *>(w + row0 + 8 * i + 4 * hh);
#pragma unroll
        for (int j = 0; j < 4; ++j) wf[4 * i + j] = x[j];
    }
}

template <bool BF16, int C>
__device__ inline void tile_sums(const char *tile, const float (&wf)[16], int lane, f32x16 (&o)[C / 32])
{
    const int l32 = lane & 31, hh = lane >> 5;
    if constexpr (BF16) {
        const int gq = lane >> 4, s4 = lane & 15, jr = s4 >> 2, qq = s4 & 3;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            bf16x8 ws[3];   // each the rounding of what the ones before leave
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float left = wf[8 * hf + j];
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    ws[k][j] = static_cast<__bf16>(left);
                    left -= static_cast<float>(ws[k][j]);
                }
            }
#pragma unroll
            for (int db = 0; db < C / 32; ++db) {
                s16x4 r[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int row = 16 * hf + 8 * k + 4 * (gq >> 1) + jr;
                    const int off = row * C + ((8 * ((2 * (gq & 1) + (qq >> 1)) ^ swzd<C>(row)) + 4 * (qq & 1)) ^ (32 * db));
                    r[k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(reinterpret_cast<const __bf16 *>(tile) + off));
                }
                const s16x8 xv = {r[0][0], r[0][1], r[0][2], r[0][3], r[1][0], r[1][1], r[1][2], r[1][3]};
#pragma unroll
                for (int k = 0; k < 3; ++k)
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, xv), ws[k], o[db], 0, 0, 0);
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const float *xr = reinterpret_cast<const float *>(tile) + grow(j, hh) * C + l32;
#pragma unroll
            for (int db = 0; db < C / 32; ++db)
                o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(xr[32 * db], wf[j], o[db], 0, 0, 0);
        }
    }
}

// LDS of a wave that sums blocks 32 channels at a time
template <bool BF16>
constexpr int kSumTile = 32 * 32 * (BF16 ? 2 : 4);

// The summary of block b of key head h, complete with this call:
//   S_e(b) = (b starts a group of e's level ? 0 : S_e(b - 1))
//            + sum over its rows j of pi_e[b r mod s_l + j] x_j.
// A wave takes 32 channels of the keys or of the values, its sums start from the
// previous block's, and no two waves meet.  fp32 throughout: sums over up to 2^15
// blocks of a group are kept.  dst, before: the summary pages of b and b - 1.
template <bool BF16, int D, int NW>
__device__ inline void summarize(const CacheArgs &a, const Tile &x, int h, int b, int page, int dst, int before, char *tile)
{
    const int lane = threadIdx.x & 63, l32 = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll 1
    for (int task = wave; task < 2 * (D / 32); task += NW) {
        const int kv = task & 1, c0 = 32 * (task >> 1);
        BlockRows<BF16, D, 32> rows(a, x, h, kv, page, c0, lane);
#pragma unroll 1
        for (int s0 = 0; s0 < a.sets; s0 += 32) {
            const int e = s0 + l32;
            const bool col = e < a.sets;
            const float *const w = block_weights(a, kv, h, col ? e : 0, b);
            float next[16];
            rows.fetch(0, true);
            tile_weights(w, col, 0, a.r, hh, next);
            f32x16 o[1] = {f32x16{0}};
            if (col && before >= 0 && (b & ((1 << (e / a.rank)) - 1))) {
                const float *const from = a.sum + ((((long long)before * a.kv_heads + h) * 2 + kv) * a.sets + e) * D + c0;
#pragma unroll
                for (int j = 0; j < 16; j += 4) {
                    const f32x4 f = *reinterpret_cast<const f32x4 *>(from + grow(j, hh));
                    o[0][j] = f[0], o[0][j + 1] = f[1], o[0][j + 2] = f[2], o[0][j + 3] = f[3];
                }
            }
#pragma unroll 1
            for (int row0 = 0; row0 < a.r; row0 += 32) {
                float wf[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) wf[j] = next[j];
                rows.stage(tile);
                rows.fetch(row0 + 32, true);
                tile_weights(w, col, row0 + 32, a.r, hh, next);
                tile_sums<BF16, 32>(tile, wf, lane, o);
            }
            if (col) {
                float *const to = a.sum + ((((long long)dst * a.kv_heads + h) * 2 + kv) * a.sets + e) * D + c0;
#pragma unroll
                for (int j = 0; j < 16; j += 4)
                    *reinterpret_cast<f32x4 *>(to + grow(j, hh)) = f32x4{o[0][j], o[0][j + 1], o[0][j + 2], o[0][j + 3]};
            }
        }
    }
}

}  // namespace

}  // namespace fma_dev

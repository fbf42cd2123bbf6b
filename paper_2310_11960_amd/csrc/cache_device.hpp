// cache_device.hpp -- rows of the paged cache, and what entering tokens leave
// behind: page copies and the block summaries.
#pragma once

#include "cache.hpp"
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

constexpr int kSumSets = 4;   // sets that one walk over a block's rows adds up

template <int D, int NT>
struct SumSmem {
    float part[NT / 64][kSumSets][D];
};

// The summary of block b of key head h, complete with this call:
//   S_e(b) = sum over its rows j of pi_e[b r mod s_l + j] x_j
//            + (b starts a group of e's level ? 0 : S_e(b - 1)).
// Rows from x.start on come from the caller's tensors, the others from the
// block's page; d / 8 lanes hold a row, half of the waves the keys, the others
// the values.  fp32 throughout: sums over up to 2^15 blocks of a group are kept.
template <bool BF16, int D, int NT>
__device__ inline void summarize(const CacheArgs &a, const Tile &x, int h, int b, int page, SumSmem<D, NT> &sm)
{
    constexpr int LPR = D / 8, NW = NT / 64, HT = NT / 2, SLOTS = HT / LPR;
    const int dst = summary_of(a, x.seq, b);
    if (dst < 0) return;
    const int before = b > 0 ? summary_of(a, x.seq, b - 1) : -1;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, t = tid >= HT;
    const int ch = 8 * (tid % LPR), slot = (tid - t * HT) / LPR;
    const float *w = (t ? a.wv : a.wk) + h * a.w_stride;
    const long long row = (long long)a.sets * D;   // floats of one tensor's sums
    for (int e0 = 0; e0 < a.sets; e0 += kSumSets) {
        float acc[kSumSets][8];
        const float *we[kSumSets];
#pragma unroll
        for (int e = 0; e < kSumSets; ++e) {
            const int l = (e0 + e) / a.rank, s = (e0 + e) - l * a.rank;
            const long long size = (long long)a.r << l;
            we[e] = w + a.rank * (size - a.r) + s * size + (long long)(b & ((1 << l) - 1)) * a.r;
#pragma unroll
            for (int c = 0; c < 8; ++c) acc[e][c] = 0.f;
        }
        for (int j = slot; j < a.r; j += SLOTS) {
            const int pos = b * a.r + j;
            float f[8];
            if (pos >= x.start) {
                const long long o = (long long)(x.row0 + pos - x.start) * (t ? a.vt : a.kt) + h * (t ? a.vh : a.kh);
                load8f<BF16>(elem<BF16>(t ? a.v : a.k, o + ch), f);
            } else if (page >= 0) {
                load8f<BF16>(elem<BF16>(const_cast<const void *>(t ? a.vp : a.kp), page_row(a, page, h, j) + ch), f);
            } else {
                continue;
            }
#pragma unroll
            for (int e = 0; e < kSumSets; ++e) {
                const float wj = e0 + e < a.sets ? we[e][j] : 0.f;
#pragma unroll
                for (int c = 0; c < 8; ++c) acc[e][c] = fmaf(wj, f[c], acc[e][c]);
            }
        }
#pragma unroll
        for (int e = 0; e < kSumSets; ++e)
#pragma unroll
            for (int c = 0; c < 8; ++c) {
#pragma unroll
                for (int m = LPR; m < 64; m *= 2) acc[e][c] += __shfl_xor(acc[e][c], m);
                if (lane < LPR) sm.part[wave][e][ch + c] = acc[e][c];
            }
        __syncthreads();
        for (int i = tid; i < 2 * kSumSets * D; i += NT) {
            const int kv = i / (kSumSets * D), e = i / D % kSumSets, c = i % D;
            if (e0 + e < a.sets) {
                float s = 0.f;
#pragma unroll
                for (int k = 0; k < NW / 2; ++k) s += sm.part[kv * (NW / 2) + k][e][c];
                const long long o = kv * row + (long long)(e0 + e) * D + c;
                if (before >= 0 && (b & ((1 << ((e0 + e) / a.rank)) - 1)))
                    s += a.sum[((long long)before * a.kv_heads + h) * 2 * row + o];
                a.sum[((long long)dst * a.kv_heads + h) * 2 * row + o] = s;
            }
        }
        __syncthreads();
    }
}

}  // namespace

}  // namespace fma_dev

// cache_attend.hip -- FMA attention of new tokens over the paged cache, for pieces
// of few rows, and in the same launch their way into it where no chunk is longer
// than a block.
//
// A query of base block b attends to the tokens of blocks b - 1 and b up to its
// own and, at level l, to the summaries of groups q - 2 and (q odd) q - 3, q =
// b >> (l - 1): one softmax.  No later token and no sequence length enters.
//
// A workgroup takes at most 32 rows, one tile of positions times the query heads
// that share a key head, and deals the key tiles (32 near tokens, or 32 sources of
// the far list) to its waves; each keeps its own reference, sum and output
// (cache_tile.hpp) and they meet in LDS.  A wave's next tile is on its way in
// registers, whole rows by adjacent lanes, while it uses the one in LDS.
//
// What bounds it: the latency of a few dependent loads (lengths, pages, rows)
// and of two or three tiles per wave.
#include "cache_device.hpp"
#include "cache_tile.hpp"

namespace fma_dev {

namespace {

template <bool BF16, int D, int NW>
struct KeysSmem {
    static constexpr int TB = 32 * D * (BF16 ? 2 : 4);
    union {
        __attribute__((aligned(16))) char tile[NW][TB];   // keys, then values
        float o[NW * 32 * 33];
        __attribute__((aligned(16))) char sum[NW][kSumTile<BF16>];
    };
    float m[NW][32], l[NW][32];
};

template <bool BF16, int D, int NW>
__global__ __launch_bounds__(64 * NW) void cache_keys_kernel(CacheArgs a, Tiling t, int split, int gs)
{
    constexpr int NT = 64 * NW, ND = D / 32, RB = D * (BF16 ? 2 : 4);
    constexpr int LPR = D / 8, RPL = 64 / LPR, NL = 32 / RPL;   // lanes of a row, rows of a load, loads of a tile
    __shared__ KeysSmem<BF16, D, NW> sm;
    Tile x;
    const CacheGroup g = cache_group(a.kv_heads * split);
    if (!find_tile(a, t, g.unit, x)) return;
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = g.head / split, g0 = (g.head - h * split) * gs;
    const int ng = gs < a.group - g0 ? gs : a.group - g0;   // this workgroup's query heads
    const int b = x.pos / a.r, pos_b = b * a.r, klo = b > 0 ? pos_b - a.r : 0, kend = x.pos + x.n;
    const int page = page_of(a, x.seq, b), page0 = b > 0 ? page_of(a, x.seq, b - 1) : -1;
    const bool completes = a.write && g0 == 0 && a.sets && kend % a.r == 0;
    const int dst = completes ? summary_of(a, x.seq, b) : -1, before = completes && b > 0 ? summary_of(a, x.seq, b - 1) : -1;
    const int near = (kend - klo + 31) / 32;
    const FarList list(a, b);
    const int tiles = near + (list.n + 31) / 32;

    // Tile i's rows, eight channels a lane (zeros for rows that are not there), and
    // which of them are.  Positions from `fresh` on come from the caller's tensors.
    const int lr = lane / LPR, lc = lane % LPR, fresh = a.k ? x.start : kend;
    const int lane_off = lr * RB + RB / LPR * lc;
    Raw8<BF16> rk[NL], rv[NL];
    uint32_t there;
    auto fetch = [&](int i) __attribute__((always_inline)) {
        if (i < near) {
            const int k0 = klo + 32 * i;
            const bool own = k0 >= pos_b;   // (blocks of a multiple of 32: tiles do not cross them)
            const int pg = own ? page : page0;
            if ((a.r & 31) == 0 && pg >= 0 && k0 + 32 <= fresh && k0 + 32 <= kend) {   // a whole tile of a page
                const long long off = page_row(a, pg, h, k0 - (own ? pos_b : klo));
                const char *const k = static_cast<const char *>(elem<BF16>(const_cast<const void *>(a.kp), off)) + lane_off;
                const char *const v = static_cast<const char *>(elem<BF16>(const_cast<const void *>(a.vp), off)) + lane_off;
#pragma unroll
                for (int j = 0; j < NL; ++j) rk[j] = load_raw<BF16>(k + j * RPL * RB);
#pragma unroll
                for (int j = 0; j < NL; ++j) rv[j] = load_raw<BF16>(v + j * RPL * RB);
                there = ~0u;
                return;
            }
#pragma unroll
            for (int j = 0; j < NL; ++j) {
                const int pos = k0 + j * RPL + lr;
                const int p = pos >= pos_b ? page : page0;
                rk[j] = Raw8<BF16>();
                rv[j] = Raw8<BF16>();
                if (pos >= kend || (pos < fresh && p < 0)) continue;
                if (pos >= fresh) {
                    const long long n = x.row0 + pos - x.start;
                    rk[j] = load_raw<BF16>(elem<BF16>(a.k, n * a.kt + h * a.kh + 8 * lc));
                    rv[j] = load_raw<BF16>(elem<BF16>(a.v, n * a.vt + h * a.vh + 8 * lc));
                } else {
                    const long long off = page_row(a, p, h, pos - (pos >= pos_b ? pos_b : klo)) + 8 * lc;
                    rk[j] = load_raw<BF16>(elem<BF16>(const_cast<const void *>(a.kp), off));
                    rv[j] = load_raw<BF16>(elem<BF16>(const_cast<const void *>(a.vp), off));
                }
            }
            const int lo = k0 + l32;
            there = (uint32_t)__builtin_amdgcn_ballot_w64(lo < kend && (lo >= fresh || (lo >= pos_b ? page : page0) >= 0));
        } else {
            // fp32 sums, rounded to the cache's type as the dense path keeps them; lane l32
            // looks row l32 up
            const float *const mine = list.row(a, x.seq, h, 32 * (i - near) + l32);
            there = (uint32_t)__builtin_amdgcn_ballot_w64(mine != nullptr);
            const long long at = mine ? mine - a.sum : 0;
#pragma unroll
            for (int j = 0; j < NL; ++j) {
                const int row = j * RPL + lr;
                const long long off = (long long)(uint32_t)__shfl((int)at, row) | (long long)__shfl((int)(at >> 32), row) << 32;
                float k[8], v[8];
#pragma unroll
                for (int c = 0; c < 8; ++c) k[c] = v[c] = 0.f;
                if (there >> row & 1) {
                    load8f<false>(a.sum + off + 8 * lc, k);
                    load8f<false>(a.sum + off + (long long)a.sets * D + 8 * lc, v);
                }
                rk[j] = rounded<BF16>(k);
                rv[j] = rounded<BF16>(v);
            }
        }
    };
    auto put = [&](char *to, const Raw8<BF16> (&r)[NL]) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < NL; ++k) {
            const int row = k * RPL + lr, sw = chunk_swz<BF16, D>(row);
            if constexpr (BF16) {
                *reinterpret_cast<uint4 *>(to + row * RB + 16 * (lc ^ sw)) = make_uint4(r[k].w[0], r[k].w[1], r[k].w[2], r[k].w[3]);
            } else {
                float f[8];
                floats<BF16>(r[k], f);
                *reinterpret_cast<f32x4 *>(to + row * RB + 16 * ((2 * lc) ^ sw)) = f32x4{f[0], f[1], f[2], f[3]};
                *reinterpret_cast<f32x4 *>(to + row * RB + 16 * ((2 * lc + 1) ^ sw)) = f32x4{f[4], f[5], f[6], f[7]};
            }
        }
    };
    // this lane's query: row l32 of the tile, position by position
    const int rows = x.n * ng, qi = l32 < rows ? l32 / ng : 0, gi = l32 < rows ? l32 - qi * ng : 0, qpos = x.pos + qi;
    QueryTile<BF16, D> qt(lane, a.scale_log2);
    qt.load(elem<BF16>(a.q, (long long)(x.row + qi) * a.qt + (h * a.group + g0 + gi) * a.qh), a.scale_log2);
    if (a.write && g0 == 0) copy_rows<BF16, D, NT>(a, x, h, page);
    qt.start(lane);
    f32x16 o[ND];
#pragma unroll
    for (int db = 0; db < ND; ++db) o[db] = f32x16{0};
    float m = -INFINITY, l = 0.f;
    uint32_t late = 0;   // near tiles (16 at most) that come at the end
    char *const tile = sm.tile[wave];
#pragma unroll 1
    for (int i = wave; i < tiles; i += NW) {
        fetch(i);
        const uint32_t vm = there;
        if (vm == 0) continue;
        uint4 kf[QueryTile<BF16, D>::NC];
        put(tile, rk);
        qt.keys(tile, kf);
        put(tile, rv);
        const int last = i < near ? qpos - klo - 32 * i : 31;
        const bool all = vm == ~0u && (i >= near || klo + 32 * i + 31 <= x.pos);
        if (!all && i < near && qt.odd_rows(tile)) {
            late |= 1u << i;
            continue;
        }
        qt.meet(kf, tile, seen_rows(vm, last, hh), all, o, m, l);
    }
    for (; late; late &= late - 1)
        late_rows<BF16, D>(a, x, h, klo + 32 * __builtin_ctz(late), qt, qpos, o, m, l);

    // the waves' parts: a common reference, then 32 channels at a time
    l = pair_sum(l);
    if (hh == 0) {
        sm.m[wave][l32] = m;
        sm.l[wave][l32] = l;
    }
    __syncthreads();
    float top = -INFINITY, den = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, sm.m[w][l32]);
    // (a wave without a score adds its zeros, or a NaN score's NaN)
    auto weight = [&](float mw) { return mw == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mw - top); };
#pragma unroll
    for (int w = 0; w < NW; ++w) den = fmaf(sm.l[w][l32], weight(sm.m[w][l32]), den);
    const float f = den == 0.f ? 0.f : weight(m) / den;   // a row that sees nothing is zero
    // as many 32-channel pieces at a time as the rows leave room for
    const int most = 32 / rows < ND ? 32 / rows : ND;
    for (int db0 = 0; db0 < ND; db0 += most) {
        const int n = most < ND - db0 ? most : ND - db0;
        __syncthreads();
        if (l32 < rows) {
#pragma unroll
            for (int db = 0; db < ND; ++db) {
                if (db < db0 || db >= db0 + n) continue;
                float *const to = sm.o + (((db - db0) * NW + wave) * rows + l32) * 33 + 4 * hh;
#pragma unroll
                for (int j = 0; j < 16; ++j) to[8 * (j >> 2) + (j & 3)] = o[db][j] * f;
            }
        }
        __syncthreads();
        for (int i = tid; i < 16 * rows * n; i += NT) {   // two channels a thread
            const int c = 2 * (i & 15), row = (i >> 4) % rows, db = (i >> 4) / rows, ri = row / ng;
            const float *const from = sm.o + (db * NW * rows + row) * 33 + c;
            float y0 = 0.f, y1 = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                y0 += from[w * rows * 33];
                y1 += from[w * rows * 33 + 1];
            }
            const long long off = (long long)(x.row + ri) * a.ot + (h * a.group + g0 + row - ri * ng) * a.oh + 32 * (db0 + db) + c;
            if constexpr (BF16)
                *static_cast<uint32_t *>(elem<BF16>(a.out, off)) = pack_bf16(y0, y1);
            else
                *static_cast<float2 *>(elem<BF16>(a.out, off)) = make_float2(y0, y1);
        }
    }
    if (dst >= 0) {
        __syncthreads();
        summarize<BF16, D, NW>(a, x, h, b, page, dst, before, sm.sum[wave]);
    }
}

template <bool BF16, int D, int NW>
hipError_t keys_w(const CacheArgs &a, const ChunkShape &c, const Tiling &t, hipStream_t st)
{
    hipLaunchKernelGGL((cache_keys_kernel<BF16, D, NW>), dim3((unsigned)(t.units * a.kv_heads * c.split)), dim3(64 * NW), 0, st,
                       a, t, c.split, c.gs);
    return hipGetLastError();
}

// Eight waves where their tiles' latency counts and no other workgroup waits for
// the CU (bf16 up to d = 64, up to one workgroup per CU: 4 pieces of 64 tokens,
// 16 heads, 13.0 us against 14.4 with four), else four (64 drafts of 5 tokens, 16
// heads: 24.5 us against 39.5; d = 128, 32 drafts of 8 heads: 16.2 against 21.2).
template <bool BF16, int D>
hipError_t keys_d(const CacheArgs &a, const ChunkShape &c, int cus, hipStream_t st)
{
    const Tiling t = make_tiling(a, keys_tile(c));
    const long long tiles = a.rows / t.tm > a.S ? a.rows / t.tm : a.S;   // about (t.units bounds any batch)
    if constexpr (BF16 && D <= 64)
        if (tiles * a.kv_heads * c.split <= cus) return keys_w<BF16, D, 8>(a, c, t, st);
    return keys_w<BF16, D, 4>(a, c, t, st);
}

}  // namespace

hipError_t launch_cache_keys(const CacheArgs &a, const ChunkShape &c, int cus, hipStream_t st)
{
    switch (a.head_dim) {
    case 32: return a.bf16 ? keys_d<true, 32>(a, c, cus, st) : keys_d<false, 32>(a, c, cus, st);
    case 64: return a.bf16 ? keys_d<true, 64>(a, c, cus, st) : keys_d<false, 64>(a, c, cus, st);
    case 128: return a.bf16 ? keys_d<true, 128>(a, c, cus, st) : keys_d<false, 128>(a, c, cus, st);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace fma_dev

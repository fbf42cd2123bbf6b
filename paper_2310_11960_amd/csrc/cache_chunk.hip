// cache_chunk.hip -- FMA attention of longer pieces over the paged cache: up to
// 128 query rows of one base block against the rows they share.
//
// A workgroup's waves take 32 query rows each (positions times the query heads of
// one key head) and meet every 32-row tile of keys in LDS: the previous and the
// own block's tokens, which stream through two stages by direct-to-LDS loads
// a tile ahead, then the far list, loaded once at the start.  A wave leaves
// out the tiles behind its last query.  Products and softmax: cache_tile.hpp.
//
// What bounds it: issue.  A 32 x 32 piece at d = 64 takes 256 cycles of matrix
// products and about 450 of vector work, the exponentials 256 of them.  4 pieces of
// 4096 tokens, 12 heads, rank 4: 49 us.
#include "cache_device.hpp"
#include "cache_tile.hpp"
#include "row_groups.hpp"

namespace fma_dev {

namespace {

constexpr int kStages = 2;   // near tiles in LDS

// Rows of a block's tokens: position p of [lo, hi) at k + (p - first) * sk, v likewise.
template <bool BF16>
struct NearRows {
    const char *k, *v;
    long long sk, sv;   // bytes
    int first, lo, hi;
    bool paged;
    __device__ NearRows() {}
    __device__ NearRows(const CacheArgs &a, const Tile &x, int h, int page, int first_, int end)
    {
        first = first_;
        hi = end;
        paged = page >= 0;
        if (paged) {
            const long long off = page_row(a, page, h, 0);
            k = static_cast<const char *>(elem<BF16>(const_cast<const void *>(a.kp), off));
            v = static_cast<const char *>(elem<BF16>(const_cast<const void *>(a.vp), off));
            sk = sv = a.head_dim * (BF16 ? 2 : 4);
            lo = first;
        } else {   // the caller's tensors, for the new ones
            const long long n = x.row0 + first - x.start;
            k = static_cast<const char *>(elem<BF16>(a.k, n * a.kt + h * a.kh));
            v = static_cast<const char *>(elem<BF16>(a.v, n * a.vt + h * a.vh));
            sk = a.kt * (BF16 ? 2 : 4);
            sv = a.vt * (BF16 ? 2 : 4);
            lo = !a.k ? end : first > x.start ? first : x.start;
        }
    }
};

template <bool BF16, int D, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(NW < 4 ? 1 : BF16 ? (D == 128 ? 2 : 4) : (D == 32 ? 4 : 1))))
void cache_chunk_kernel(CacheArgs a, Tiling t, int split, int gs, int far_cap)
{
    constexpr int ND = D / 32, RB = D * (BF16 ? 2 : 4), TB = 32 * RB;   // row, tile bytes
    constexpr int CPR = RB / 16, RPL = 64 / CPR, NLD = TB / 1024;   // 16-byte chunks of a row, rows of a load, loads
    constexpr int ML = (2 * NLD + NW - 1) / NW, FL = 2 * NLD / NW;  // a wave's loads of a tile, at most and at least
    extern __shared__ __attribute__((aligned(16))) char smem[];
    char *const ring = smem;                                        // [kStages][2][TB]
    char *const far_k = smem + kStages * 2 * TB, *const far_v = far_k + far_cap * RB;
    uint32_t *const far_ok = reinterpret_cast<uint32_t *>(far_v + far_cap * RB);
    Tile x;
    const CacheGroup g = cache_group(a.kv_heads * split);
    if (!find_tile(a, t, g.unit, x)) return;
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = g.head / split, g0 = (g.head - h * split) * gs;
    const int ng = gs < a.group - g0 ? gs : a.group - g0;
    const int b = x.pos / a.r, pos_b = b * a.r, klo = b > 0 ? pos_b - a.r : 0, kend = x.pos + x.n;
    const int near = (kend - klo + 31) / 32;
    const FarList list(a, b);
    const NearRows<BF16> prev(a, x, h, b > 0 ? page_of(a, x.seq, b - 1) : -1, klo, pos_b);
    const NearRows<BF16> own(a, x, h, page_of(a, x.seq, b), pos_b, kend);

    // near tile i to stage st: load j of the tile (keys, then values) by wave j % NW
    const int lrow = lane / CPR, lchunk = lane % CPR;
    const char *const any = static_cast<const char *>(elem<BF16>(a.q, (long long)x.row * a.qt + (h * a.group + g0) * a.qh));
    auto issue = [&](int i, int st) __attribute__((always_inline)) {
        const int k0 = klo + 32 * i;
        const bool whole = k0 >= pos_b;   // (blocks of a multiple of 32: tiles do not cross them)
        const char *const sk = whole ? own.k : prev.k, *const sv = whole ? own.v : prev.v;
        const int first = whole ? own.first : prev.first;
        const bool plain = (a.r & 31) == 0 && (whole ? own.paged && k0 + 32 <= own.hi : prev.paged);
#pragma unroll
        for (int jj = 0; jj < ML; ++jj) {
            const int j = wave + NW * jj;
            if (ML != FL && j >= 2 * NLD) break;
            const int val = j >= NLD, row = (j - val * NLD) * RPL + lrow, ch = 16 * (lchunk ^ chunk_swz<BF16, D>(row));
            const char *p;
            if (plain) {
                p = (val ? sv : sk) + (k0 - first) * RB + (row * RB + ch);
            } else {
                // a row that is not there repeats one that is (its weight is 0, and
                // what the page holds in its place is no number to multiply)
                bool o = k0 + row >= pos_b;
                o = (o ? own.lo < own.hi : prev.lo < prev.hi) ? o : !o;
                const int lo = o ? own.lo : prev.lo, hi = o ? own.hi : prev.hi;
                const int pos = k0 + row < lo ? lo : k0 + row >= hi ? hi - 1 : k0 + row;
                const long long step = val ? (o ? own.sv : prev.sv) : (o ? own.sk : prev.sk);
                p = (val ? (o ? own.v : prev.v) : (o ? own.k : prev.k)) + (pos - (o ? own.first : prev.first)) * step;
                p = (lo < hi ? p : any) + ch;
            }
            dma16(p, lds_u32(ring + (2 * st + val) * TB) + (j - val * NLD) * 1024);
        }
    };
    // which rows of near tile i are there
    auto rows_there = [&](int i) {
        const int k0 = klo + 32 * i;
        auto bits = [&](int lo, int hi) {
            lo = lo - k0 < 0 ? 0 : lo - k0;
            hi = hi - k0 > 32 ? 32 : hi - k0;
            return lo >= hi ? 0u : (hi - lo == 32 ? ~0u : ((1u << (hi - lo)) - 1) << lo);
        };
        return bits(prev.lo, prev.hi) | bits(own.lo, own.hi);
    };
    // far rows first .. of the list, fp32, to LDS in the cache's type (bf16: rounded, as
    // the dense path keeps them); whole tiles, rows beyond the list as missing ones
    auto far_rows = [&](int first) {
        constexpr int LPR = D / 8, RPP = 64 * NW / LPR, U = 2;   // U passes' pages, then their rows
        const int left = (list.n - first + 31) / 32 * 32, rows = left < far_cap ? left : far_cap, lc = tid % LPR;
        for (int row0 = tid / LPR; row0 < rows; row0 += U * RPP) {
            const float *far[U];
            f32x4 f[U][2][2];
#pragma unroll
            for (int u = 0; u < U; ++u) far[u] = row0 + u * RPP < rows ? list.row(a, x.seq, h, first + row0 + u * RPP) : nullptr;
#pragma unroll
            for (int u = 0; u < U; ++u) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    f[u][k >> 1][k & 1] = f32x4{0.f, 0.f, 0.f, 0.f};
                    if (far[u]) f[u][k >> 1][k & 1] = *reinterpret_cast<const f32x4 *>(far[u] + (k >> 1) * a.sets * D + 8 * lc + 4 * (k & 1));
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int row = row0 + u * RPP, sw = chunk_swz<BF16, D>(row);
                if (row >= rows) continue;
                if (lc == 0) far_ok[row] = far[u] != nullptr;
#pragma unroll
                for (int kv = 0; kv < 2; ++kv) {
                    char *const to = (kv ? far_v : far_k) + row * RB;
                    const f32x4 lo = f[u][kv][0], hi = f[u][kv][1];
                    if constexpr (BF16) {
                        *reinterpret_cast<uint4 *>(to + 16 * (lc ^ sw)) = make_uint4(pack_bf16(lo[0], lo[1]), pack_bf16(lo[2], lo[3]),
                                                                                   pack_bf16(hi[0], hi[1]), pack_bf16(hi[2], hi[3]));
                    } else {
                        *reinterpret_cast<f32x4 *>(to + 16 * ((2 * lc) ^ sw)) = lo;
                        *reinterpret_cast<f32x4 *>(to + 16 * ((2 * lc + 1) ^ sw)) = hi;
                    }
                }
            }
        }
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i)
        if (i < near) issue(i, i);

    // this lane's query
    const int rows = x.n * ng, row = 32 * wave + l32, qi = row < rows ? row / ng : 0, gi = row < rows ? row - qi * ng : 0;
    const int qpos = x.pos + qi;
    const int wfirst = x.pos + 32 * wave / ng;   // positions of the wave's first and last rows
    const int wtop = 32 * wave + 31 < rows ? 32 * wave + 31 : rows - 1, wlast = x.pos + wtop / ng;
    const bool active = 32 * wave < rows;
    QueryTile<BF16, D> qt(lane, a.scale_log2);
    qt.load(elem<BF16>(a.q, (long long)(x.row + qi) * a.qt + (h * a.group + g0 + gi) * a.qh), a.scale_log2);
    if (list.n) far_rows(0);
    qt.start(lane);
    f32x16 o[ND];
#pragma unroll
    for (int db = 0; db < ND; ++db) o[db] = f32x16{0};
    float m = -INFINITY, l = 0.f;
    uint32_t late = 0;   // near tiles (16 at most) that come at the end

    const int tiles = near + (list.n + 31) / 32;
#pragma unroll 1
    for (int i = 0; i < tiles; ++i) {
        const char *kt, *vt;
        uint32_t vm;
        int last;       // rows of the tile that lie behind this lane's query start there
        bool all;       // every query of the wave sees every row
        if (i < near) {
            const int st = i % kStages, k0 = klo + 32 * i;
            if (i + kStages - 2 < near)   // the tiles behind this one may be on their way
                wait_vm<(kStages - 2) * FL>();
            else
                wait_vm<0>();
            __syncthreads();
            if (i + kStages - 1 < near) issue(i + kStages - 1, (i + kStages - 1) % kStages);
            vm = rows_there(i);
            if (!active || k0 > wlast || vm == 0) continue;
            kt = ring + 2 * st * TB;
            vt = kt + TB;
            last = qpos - k0;
            all = vm == ~0u && k0 + 31 <= wfirst;
        } else {
            const int f = 32 * (i - near), at = f % far_cap;
            if (f > 0 && at == 0) {   // (more far rows than LDS holds)
                __syncthreads();
                far_rows(f);
                __syncthreads();
            }
            if (!active) continue;
            vm = (uint32_t)__builtin_amdgcn_ballot_w64(far_ok[at + l32] != 0);
            if (vm == 0) continue;
            kt = far_k + at * RB;
            vt = far_v + at * RB;
            last = 31;
            all = vm == ~0u;
        }
        if (!all && i < near && qt.odd_rows(vt)) {
            late |= 1u << i;
            continue;
        }
        qt.meet(kt, vt, seen_rows(vm, last, hh), all, o, m, l);
    }
    if (!active) return;
    for (; late; late &= late - 1)
        late_rows<BF16, D>(a, x, h, klo + 32 * __builtin_ctz(late), qt, qpos, o, m, l);
    l = pair_sum(l);
    const float inv = l == 0.f ? 0.f : 1.f / l;   // a row that sees nothing is zero
    auto out_row = [&](int r) {
        const int i = r / ng;
        return (long long)(x.row + i) * a.ot + (h * a.group + g0 + r - i * ng) * a.oh;
    };
#pragma unroll
    for (int db = 0; db < ND; ++db) {
        if constexpr (BF16) {
            uint32_t u[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) u[k] = pack_bf16(o[db][2 * k] * inv, o[db][2 * k + 1] * inv);
            gather_rows(u);
            const int c = 32 * db + 8 * store_chunk(lane), r0 = 32 * wave + (lane & 15), r1 = r0 + 16;
            if (r0 < rows) *reinterpret_cast<uint4 *>(elem<BF16>(a.out, out_row(r0) + c)) = make_uint4(u[0], u[1], u[2], u[3]);
            if (r1 < rows) *reinterpret_cast<uint4 *>(elem<BF16>(a.out, out_row(r1) + c)) = make_uint4(u[4], u[5], u[6], u[7]);
        } else if (row < rows) {
            const long long off = (long long)(x.row + qi) * a.ot + (h * a.group + g0 + gi) * a.oh + 32 * db;
#pragma unroll
            for (int j = 0; j < 16; j += 4)
                *reinterpret_cast<f32x4 *>(elem<BF16>(a.out, off + grow(j, hh))) =
                    f32x4{o[db][j] * inv, o[db][j + 1] * inv, o[db][j + 2] * inv, o[db][j + 3] * inv};
        }
    }
}

template <bool BF16, int D, int NW>
hipError_t chunk_w(const CacheArgs &a, const ChunkShape &c, const Tiling &t, hipStream_t st)
{
    constexpr int RB = D * (BF16 ? 2 : 4);
    int far = (2 * a.sets + 31) / 32 * 32;   // the longest list
    constexpr int kMost = RB == 512 ? 32 : 64;   // at a time, within 160 KB
    if (far > kMost) far = kMost;
    const int lds = kStages * 2 * 32 * RB + far * (2 * RB + 4);
    if (lds > 65536) {
        const void *const fn = reinterpret_cast<const void *>(cache_chunk_kernel<BF16, D, NW>);
        const hipError_t e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((cache_chunk_kernel<BF16, D, NW>), dim3((unsigned)(t.units * a.kv_heads * c.split)), dim3(64 * NW), lds,
                       st, a, t, c.split, c.gs, far);
    return hipGetLastError();
}

template <bool BF16, int D>
hipError_t chunk_d(const CacheArgs &a, const ChunkShape &c, hipStream_t st)
{
    const Tiling t = make_tiling(a, c.tm);
    switch ((t.tm * c.gs + 31) / 32) {
    case 1: return chunk_w<BF16, D, 1>(a, c, t, st);
    case 2: return chunk_w<BF16, D, 2>(a, c, t, st);
    case 3: return chunk_w<BF16, D, 3>(a, c, t, st);
    default: return chunk_w<BF16, D, 4>(a, c, t, st);
    }
}

}  // namespace

hipError_t launch_cache_rows(const CacheArgs &a, const ChunkShape &c, hipStream_t st)
{
    switch (a.head_dim) {
    case 32: return a.bf16 ? chunk_d<true, 32>(a, c, st) : chunk_d<false, 32>(a, c, st);
    case 64: return a.bf16 ? chunk_d<true, 64>(a, c, st) : chunk_d<false, 64>(a, c, st);
    case 128: return a.bf16 ? chunk_d<true, 128>(a, c, st) : chunk_d<false, 128>(a, c, st);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace fma_dev

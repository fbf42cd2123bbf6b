// cache_chunk.hip -- FMA attention of longer pieces over the paged cache: up to
// 128 query rows of one base block against the rows they share.
//
// A workgroup's waves take 32 query rows each (positions times the query heads of
// one key head) and meet every 32-row tile of keys in LDS: the previous and the
// own block's tokens, whole rows from their pages or the caller's tensors, then
// the far list.  The next tile's rows are in registers while one is used.
// Products and softmax as in cache_attend.hip, with the running maximum of each
// query; a wave leaves out the tiles behind its last query.
//
// What bounds it: per 32 x 32 piece the exponentials and conversions cost as many
// cycles as the matrix products (256 + ~350 at d = 64), and a query of a block of
// 128 meets 6 .. 9 tiles, so bytes and arithmetic weigh about the same.
#include "cache_device.hpp"
#include "wave_ops.hpp"

namespace fma_dev {

namespace {

template <bool BF16, int D>
struct ChunkSmem {
    static constexpr int P = BF16 ? 2 * D : 4 * D + 16;   // row pitch (fp32: off the banks of a 256-byte stride)
    __attribute__((aligned(16))) char k[2][32 * P], v[2][32 * P];
    uint32_t ok[2][32];   // the row is there
};

template <bool BF16, int D, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(NW < 4 ? 1 : D == 128 ? 2 : 3))) void cache_chunk_kernel(CacheArgs a, Tiling t, int split, int gs)
{
    constexpr int NT = 64 * NW, ND = D / 32, NC = BF16 ? D / 16 : D / 8;
    constexpr int LPR = D / 8, RPP = NT / LPR, NP = (32 + RPP - 1) / RPP;   // rows a pass, passes a tile
    constexpr int P = ChunkSmem<BF16, D>::P;
    __shared__ ChunkSmem<BF16, D> sm;
    Tile x;
    const CacheGroup g = cache_group(a.kv_heads * split);
    if (!find_tile(a, t, g.unit, x)) return;
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = g.head / split, g0 = (g.head - h * split) * gs;
    const int ng = gs < a.group - g0 ? gs : a.group - g0;
    const int b = x.pos / a.r, pos_b = b * a.r;
    const int page = page_of(a, x.seq, b), page0 = b > 0 ? page_of(a, x.seq, b - 1) : -1;
    const int klo = b > 0 ? pos_b - a.r : 0, kend = x.pos + x.n;
    const int near = (kend - klo + 31) / 32;
    const FarList list(a, b);
    const int tiles = near + (list.n + 31) / 32;

    // tile i's rows into registers (fp32 far rows as they are), then to LDS
    const int lr = tid / LPR, lc = tid % LPR;
    Raw8<BF16> rk[NP], rv[NP];
    bool there[NP];
    auto fetch = [&](int i) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int row = lr + p * RPP;
            rk[p] = Raw8<BF16>();
            rv[p] = Raw8<BF16>();
            there[p] = false;
            if (NP * RPP > 32 && row >= 32) continue;
            if (i < near) {
                const int pos = klo + 32 * i + row;
                if (pos >= kend) continue;
                if (a.k && pos >= x.start) {
                    const long long n = x.row0 + pos - x.start;
                    rk[p] = load_raw<BF16>(elem<BF16>(a.k, n * a.kt + h * a.kh + 8 * lc));
                    rv[p] = load_raw<BF16>(elem<BF16>(a.v, n * a.vt + h * a.vh + 8 * lc));
                    there[p] = true;
                } else {
                    const int pg = pos >= pos_b ? page : page0;
                    if (pg < 0) continue;
                    const long long off = page_row(a, pg, h, pos >= pos_b ? pos - pos_b : pos - klo) + 8 * lc;
                    rk[p] = load_raw<BF16>(elem<BF16>(const_cast<const void *>(a.kp), off));
                    rv[p] = load_raw<BF16>(elem<BF16>(const_cast<const void *>(a.vp), off));
                    there[p] = true;
                }
            } else {
                const float *far = list.row(a, x.seq, h, 32 * (i - near) + row);
                if (!far) continue;
                float f[8];
                load8f<false>(far + 8 * lc, f);
                rk[p] = rounded<BF16>(f);
                load8f<false>(far + (long long)a.sets * D + 8 * lc, f);
                rv[p] = rounded<BF16>(f);
                there[p] = true;
            }
        }
    };
    auto stage = [&](int st) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int row = lr + p * RPP;
            if (NP * RPP > 32 && row >= 32) continue;
            if constexpr (BF16) {
                const int o = row * P + 16 * (lc ^ swzd<D>(row));
                *reinterpret_cast<uint4 *>(sm.k[st] + o) = make_uint4(rk[p].w[0], rk[p].w[1], rk[p].w[2], rk[p].w[3]);
                *reinterpret_cast<uint4 *>(sm.v[st] + o) = make_uint4(rv[p].w[0], rv[p].w[1], rv[p].w[2], rv[p].w[3]);
            } else {
                float f[8];
                f32x4 *to = reinterpret_cast<f32x4 *>(sm.k[st] + row * P + 32 * lc);
                floats<BF16>(rk[p], f);
                to[0] = f32x4{f[0], f[1], f[2], f[3]};
                to[1] = f32x4{f[4], f[5], f[6], f[7]};
                to = reinterpret_cast<f32x4 *>(sm.v[st] + row * P + 32 * lc);
                floats<BF16>(rv[p], f);
                to[0] = f32x4{f[0], f[1], f[2], f[3]};
                to[1] = f32x4{f[4], f[5], f[6], f[7]};
            }
            if (lc == 0) sm.ok[st][row] = there[p];
        }
    };
    fetch(0);

    // this lane's query
    const int rows = x.n * ng, row = 32 * wave + l32, qi = row < rows ? row / ng : 0, gi = row < rows ? row - qi * ng : 0;
    const int qpos = x.pos + qi;
    const int wfirst = x.pos + 32 * wave / ng;   // positions of the wave's first and last rows
    const int wtop = 32 * wave + 31 < rows ? 32 * wave + 31 : rows - 1, wlast = x.pos + wtop / ng;
    const bool active = 32 * wave < rows;
    uint4 qo[NC];
    {
        const char *p = static_cast<const char *>(elem<BF16>(a.q, (long long)(x.row + qi) * a.qt + (h * a.group + g0 + gi) * a.qh)) + 16 * hh;
#pragma unroll
        for (int c = 0; c < NC; ++c) qo[c] = *reinterpret_cast<const uint4 *>(p + 32 * c);
    }

    f32x16 o[ND];
#pragma unroll
    for (int db = 0; db < ND; ++db) o[db] = f32x16{0};
    float m = -INFINITY, l = 0.f;
    const int koff = l32 * P + 16 * (hh ^ (BF16 ? swzd<D>(l32) : 0));
    int voff[2];
    {
        const int gq = lane >> 4, s4 = lane & 15, jr = s4 >> 2, qq = s4 & 3;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int r = 8 * k + 4 * (gq >> 1) + jr;
            voff[k] = r * D + 8 * ((2 * (gq & 1) + (qq >> 1)) ^ swzd<D>(r)) + 4 * (qq & 1);
        }
    }
    stage(0);
    for (int i = 0; i < tiles; ++i) {
        const int st = i & 1;
        __syncthreads();
        if (i + 1 < tiles) fetch(i + 1);
        const int k0 = klo + 32 * i;   // (near) position of the tile's first row
        if (active && (i >= near || k0 <= wlast)) {
            const uint32_t vm = (uint32_t)__builtin_amdgcn_ballot_w64(sm.ok[st][l32] != 0);
            f32x16 s = {0};
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                if constexpr (BF16) {
                    const bf16x8 kf = *reinterpret_cast<const bf16x8 *>(sm.k[st] + (koff ^ (32 * c)));
                    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, __builtin_bit_cast(bf16x8, qo[c]), s, 0, 0, 0);
                } else {
                    const f32x4 kf = *reinterpret_cast<const f32x4 *>(sm.k[st] + koff + 32 * c);
                    const f32x4 qf = __builtin_bit_cast(f32x4, qo[c]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[j], qf[j], s, 0, 0, 0);
                }
            }
            float mx = -INFINITY;
            if (vm == 0xffffffffu && (i >= near || k0 + 31 <= wfirst)) {
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    s[j] *= a.scale_log2;
                    mx = fmaxf(mx, s[j]);
                }
            } else {
                const int last = i < near ? qpos - k0 : 31;
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const int r = grow(j, hh);
                    s[j] = r <= last && (vm >> r & 1u) ? s[j] * a.scale_log2 : -INFINITY;
                    mx = fmaxf(mx, s[j]);
                }
            }
            mx = pair_max(mx);
            if (__builtin_amdgcn_ballot_w64(mx > m) != 0) {
                const float mnew = fmaxf(m, mx);
                const float corr = mnew == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mnew);
                m = mnew;
                l *= corr;
#pragma unroll
                for (int db = 0; db < ND; ++db)
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[db][j] *= corr;
            }
            const float ref = m == -INFINITY ? 0.f : m;   // a query that has seen nothing yet
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                s[j] = __builtin_amdgcn_exp2f(s[j] - ref);
                l += s[j];
            }
            if constexpr (BF16) {
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    const uint4 pw = make_uint4(pack_bf16(s[8 * hf], s[8 * hf + 1]), pack_bf16(s[8 * hf + 2], s[8 * hf + 3]),
                                                pack_bf16(s[8 * hf + 4], s[8 * hf + 5]),
                                                pack_bf16(s[8 * hf + 6], s[8 * hf + 7]));
                    const __bf16 *vt = reinterpret_cast<const __bf16 *>(sm.v[st]) + 16 * hf * D;
#pragma unroll
                    for (int db = 0; db < ND; ++db) {
                        const s16x4 r1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(vt + (voff[0] ^ (32 * db))));
                        const s16x4 r2 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(vt + (voff[1] ^ (32 * db))));
                        const s16x8 av = {r1[0], r1[1], r1[2], r1[3], r2[0], r2[1], r2[2], r2[3]};
                        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, av),
                                                                        __builtin_bit_cast(bf16x8, pw), o[db], 0, 0, 0);
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const float *vr = reinterpret_cast<const float *>(sm.v[st] + grow(j, hh) * P) + l32;
#pragma unroll
                    for (int db = 0; db < ND; ++db)
                        o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(vr[32 * db], s[j], o[db], 0, 0, 0);
                }
            }
        }
        if (i + 1 < tiles) stage(st ^ 1);
    }
    if (!active) return;
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

template <bool BF16, int D>
hipError_t chunk_d(const CacheArgs &a, const ChunkShape &c, hipStream_t st)
{
    const Tiling t = make_tiling(a, c.tm);
    const dim3 grid((unsigned)(t.units * a.kv_heads * c.split));
    switch ((t.tm * c.gs + 31) / 32) {
    case 1: hipLaunchKernelGGL((cache_chunk_kernel<BF16, D, 1>), grid, dim3(64), 0, st, a, t, c.split, c.gs); break;
    case 2: hipLaunchKernelGGL((cache_chunk_kernel<BF16, D, 2>), grid, dim3(128), 0, st, a, t, c.split, c.gs); break;
    case 3: hipLaunchKernelGGL((cache_chunk_kernel<BF16, D, 3>), grid, dim3(192), 0, st, a, t, c.split, c.gs); break;
    default: hipLaunchKernelGGL((cache_chunk_kernel<BF16, D, 4>), grid, dim3(256), 0, st, a, t, c.split, c.gs); break;
    }
    return hipGetLastError();
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

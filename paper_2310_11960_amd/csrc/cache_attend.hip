// cache_attend.hip -- FMA attention of new tokens over the paged cache, and in
// the same launch their way into it where no chunk is longer than a block.
//
// A query of base block b attends to the tokens of blocks b - 1 and b up to its
// own and, at level l, to the summaries of groups q - 2 and (q odd) q - 3, q =
// b >> (l - 1): one softmax.  No later token and no sequence length enters.
//
// A workgroup takes at most 32 rows, one tile of positions times the query heads
// that share a key head, and deals the key tiles (32 near tokens, or 32 slots of
// the far list) to its waves; each keeps its own running maximum, sum and
// output and they meet in LDS.  Per tile:
//   S^T = K Q^T (rows straight from the pages), P = exp2(c s - m),
//   O^T += V^T P^T (bf16: V through LDS, read transposed)
// on v_mfma_f32_32x32x16_bf16 or v_mfma_f32_32x32x2_f32.  P is rounded to bf16
// for the second product (V's type); far rows, kept in fp32, to bf16 as the
// dense path keeps them; maxima, sums and O are fp32.
#include "cache_device.hpp"
#include "wave_ops.hpp"

namespace fma_dev {

namespace {

template <bool BF16, int D, int NW>
struct AttendSmem {
    union {
        __attribute__((aligned(16))) char v[NW][32 * D * (BF16 ? 2 : 4)];
        float o[NW][32][33];
        __attribute__((aligned(16))) char sum[NW][kSumTile<BF16>];
    };
    float m[NW][32], l[NW][32];
};

template <bool BF16, int D, int NW>
__global__ __launch_bounds__(64 * NW) void cache_attend_kernel(CacheArgs a, Tiling t, int split, int gs)
{
    constexpr int NT = 64 * NW, ND = D / 32, NC = BF16 ? D / 16 : D / 8;   // 16-byte pieces of a lane's half row
    __shared__ AttendSmem<BF16, D, NW> sm;
    Tile x;
    const CacheGroup g = cache_group(a.kv_heads * split);
    if (!find_tile(a, t, g.unit, x)) return;
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = g.head / split, g0 = (g.head - h * split) * gs;
    const int ng = gs < a.group - g0 ? gs : a.group - g0;   // this workgroup's query heads
    const int b = x.pos / a.r, pos_b = b * a.r;
    const int page = page_of(a, x.seq, b), page0 = b > 0 ? page_of(a, x.seq, b - 1) : -1;
    if (a.write && g0 == 0) copy_rows<BF16, D, NT>(a, x, h, page);

    // this lane's query: row l32 of the tile, position by position
    const int qi = l32 / ng, qpos = x.pos + (qi < x.n ? qi : 0);
    uint4 qo[NC];
    {
        const long long o = (long long)(x.row + (qi < x.n ? qi : 0)) * a.qt + (h * a.group + g0 + l32 - qi * ng) * a.qh;
        const char *p = static_cast<const char *>(elem<BF16>(a.q, o)) + 16 * hh;
#pragma unroll
        for (int c = 0; c < NC; ++c) qo[c] = *reinterpret_cast<const uint4 *>(p + 32 * c);
    }

    const int klo = b > 0 ? pos_b - a.r : 0, kend = x.pos + x.n;
    const int near = (kend - klo + 31) / 32;
    const int lq = b >= 2 ? 31 - __builtin_clz((unsigned)b) : 0;   // levels whose far list is not empty
    const int nfar = 2 * a.rank * (lq < a.levels ? lq : a.levels);
    const int tiles = near + (nfar + 31) / 32;

    f32x16 o[ND];
#pragma unroll
    for (int db = 0; db < ND; ++db) o[db] = f32x16{0};
    float m = -INFINITY, l = 0.f;
    char *const vt = sm.v[wave];

    for (int i = wave; i < tiles; i += NW) {
        // this lane's source: row l32 of the tile
        uint4 kk[NC], vv[NC];
        bool valid;
        if (i < near) {
            const int pos = klo + 32 * i + l32;
            const bool fresh = a.k && pos >= x.start;
            const int pg = pos >= pos_b ? page : page0;
            valid = pos < kend && (fresh || pg >= 0);
            const char *kr, *vr;
            if (fresh) {
                const long long row = x.row0 + pos - x.start;
                kr = static_cast<const char *>(elem<BF16>(a.k, row * a.kt + h * a.kh));
                vr = static_cast<const char *>(elem<BF16>(a.v, row * a.vt + h * a.vh));
            } else {
                const long long off = page_row(a, pg, h, pos >= pos_b ? pos - pos_b : pos - klo);
                kr = static_cast<const char *>(elem<BF16>(const_cast<const void *>(a.kp), off));
                vr = static_cast<const char *>(elem<BF16>(const_cast<const void *>(a.vp), off));
            }
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                kk[c] = valid ? *reinterpret_cast<const uint4 *>(kr + 32 * c + 16 * hh) : make_uint4(0, 0, 0, 0);
                vv[c] = valid ? *reinterpret_cast<const uint4 *>(vr + 32 * c + 16 * hh) : make_uint4(0, 0, 0, 0);
            }
        } else {
            const int slot = 32 * (i - near) + l32, e = slot < nfar ? slot >> 1 : 0, lv = e / a.rank;
            const int q = b >> lv, fg = q - 2 - (slot & 1);
            valid = slot < nfar && fg >= 0 && (!(slot & 1) || (q & 1));
            const int sp = valid ? summary_of(a, x.seq, ((fg + 1) << lv) - 1) : -1;
            valid = sp >= 0;
            const float *kr = a.sum + (((long long)sp * a.kv_heads + h) * 2 * a.sets + e) * D;
            const float *vr = kr + (long long)a.sets * D;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                if constexpr (BF16) {
                    float kf[8], vf[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) kf[j] = vf[j] = 0.f;
                    if (valid) {
                        load8f<false>(kr + 16 * c + 8 * hh, kf);
                        load8f<false>(vr + 16 * c + 8 * hh, vf);
                    }
                    kk[c] = make_uint4(pack_bf16(kf[0], kf[1]), pack_bf16(kf[2], kf[3]), pack_bf16(kf[4], kf[5]),
                                       pack_bf16(kf[6], kf[7]));
                    vv[c] = make_uint4(pack_bf16(vf[0], vf[1]), pack_bf16(vf[2], vf[3]), pack_bf16(vf[4], vf[5]),
                                       pack_bf16(vf[6], vf[7]));
                } else {
                    kk[c] = valid ? reinterpret_cast<const uint4 *>(kr)[2 * c + hh] : make_uint4(0, 0, 0, 0);
                    vv[c] = valid ? reinterpret_cast<const uint4 *>(vr)[2 * c + hh] : make_uint4(0, 0, 0, 0);
                }
            }
        }
        const uint32_t vm = (uint32_t)__builtin_amdgcn_ballot_w64(valid);
        // V rows to this wave's LDS tile (bf16: chunks swizzled for the
        // transposing reads)
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int chunk = 2 * c + hh;
            if constexpr (BF16)
                *reinterpret_cast<uint4 *>(vt + l32 * 2 * D + 16 * (chunk ^ swzd<D>(l32))) = vv[c];
            else
                *reinterpret_cast<f32x4 *>(vt + l32 * 4 * D + 16 * chunk) = __builtin_bit_cast(f32x4, vv[c]);
        }
        f32x16 s = {0};
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            if constexpr (BF16) {
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kk[c]),
                                                            __builtin_bit_cast(bf16x8, qo[c]), s, 0, 0, 0);
            } else {
                // channel 8 c + 4 hh + j of both operands in product j
                const f32x4 kf = __builtin_bit_cast(f32x4, kk[c]), qf = __builtin_bit_cast(f32x4, qo[c]);
#pragma unroll
                for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[j], qf[j], s, 0, 0, 0);
            }
        }
        // causal: rows up to the query's own position; the far list is the past
        const uint32_t see = seen_rows(vm, i < near ? qpos - klo - 32 * i : 31, hh);
        float mx = -INFINITY;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            s[j] = seen(see, j) ? s[j] * a.scale_log2 : -INFINITY;
            mx = fmaxf(mx, s[j]);
        }
        const float mnew = fmaxf(m, pair_max(mx));
        const float ref = mnew == -INFINITY ? 0.f : mnew;   // a query that has seen nothing yet
        const float corr = __builtin_amdgcn_exp2f(m - ref);
        m = mnew;
        l *= corr;
#pragma unroll
        for (int db = 0; db < ND; ++db)
#pragma unroll
            for (int j = 0; j < 16; ++j) o[db][j] *= corr;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            s[j] = __builtin_amdgcn_exp2f(s[j] - ref);
            l += s[j];
        }
        if constexpr (BF16) {
            const int gq = lane >> 4, s4 = lane & 15, jr = s4 >> 2, qq = s4 & 3;
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                const uint4 pw = make_uint4(pack_bf16(s[8 * hf], s[8 * hf + 1]), pack_bf16(s[8 * hf + 2], s[8 * hf + 3]),
                                            pack_bf16(s[8 * hf + 4], s[8 * hf + 5]),
                                            pack_bf16(s[8 * hf + 6], s[8 * hf + 7]));
#pragma unroll
                for (int db = 0; db < ND; ++db) {
                    s16x4 r[2];
#pragma unroll
                    for (int x2 = 0; x2 < 2; ++x2) {
                        const int row = 8 * x2 + 4 * (gq >> 1) + jr;
                        const int off = (16 * hf + row) * D + ((8 * ((2 * (gq & 1) + (qq >> 1)) ^ swzd<D>(row)) + 4 * (qq & 1)) ^ (32 * db));
                        r[x2] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(reinterpret_cast<__bf16 *>(vt) + off));
                    }
                    const s16x8 av = {r[0][0], r[0][1], r[0][2], r[0][3], r[1][0], r[1][1], r[1][2], r[1][3]};
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, av),
                                                                    __builtin_bit_cast(bf16x8, pw), o[db], 0, 0, 0);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float *vr = reinterpret_cast<const float *>(vt) + grow(j, hh) * D + l32;
#pragma unroll
                for (int db = 0; db < ND; ++db)
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(vr[32 * db], s[j], o[db], 0, 0, 0);
            }
        }
    }

    // the waves' parts: a common maximum, then 32 channels at a time
    l = pair_sum(l);
    if (hh == 0) {
        sm.m[wave][l32] = m;
        sm.l[wave][l32] = l;
    }
    __syncthreads();
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, sm.m[w][l32]);
    const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
#pragma unroll
    for (int db = 0; db < ND; ++db) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 16; ++j) sm.o[wave][grow(j, hh)][l32] = o[db][j] * f;
        __syncthreads();
        for (int i = tid; i < 32 * x.n * ng; i += NT) {
            const int row = i >> 5, c = i & 31, ri = row / ng;
            float mm = -INFINITY, den = 0.f, num = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) mm = fmaxf(mm, sm.m[w][row]);
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                num += sm.o[w][c][row];
                den += sm.m[w][row] == -INFINITY ? sm.l[w][row]   // no score yet: 0, or NaN
                                                 : sm.l[w][row] * __builtin_amdgcn_exp2f(sm.m[w][row] - mm);
            }
            const float y = den == 0.f ? 0.f : num / den;   // a row that sees nothing is zero
            const long long off = (long long)(x.row + ri) * a.ot + (h * a.group + g0 + row - ri * ng) * a.oh + 32 * db + c;
            if constexpr (BF16)
                static_cast<__bf16 *>(a.out)[off] = static_cast<__bf16>(y);
            else
                static_cast<float *>(a.out)[off] = y;
        }
    }
    if (a.write && g0 == 0 && a.sets && kend % a.r == 0) {
        const int dst = summary_of(a, x.seq, b), before = b > 0 ? summary_of(a, x.seq, b - 1) : -1;
        __syncthreads();
        if (dst >= 0) summarize<BF16, D, NW>(a, x, h, b, page, dst, before, sm.sum[wave]);
    }
}

template <bool BF16, int D>
hipError_t attend_d(const CacheArgs &a, const ChunkShape &c, hipStream_t st)
{
    constexpr int NW = BF16 ? 8 : 4;
    const Tiling t = make_tiling(a, keys_tile(c));
    hipLaunchKernelGGL((cache_attend_kernel<BF16, D, NW>), dim3((unsigned)(t.units * a.kv_heads * c.split)), dim3(64 * NW), 0,
                       st, a, t, c.split, c.gs);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_keys(const CacheArgs &a, const ChunkShape &c, hipStream_t st)
{
    switch (a.head_dim) {
    case 32: return a.bf16 ? attend_d<true, 32>(a, c, st) : attend_d<false, 32>(a, c, st);
    case 64: return a.bf16 ? attend_d<true, 64>(a, c, st) : attend_d<false, 64>(a, c, st);
    case 128: return a.bf16 ? attend_d<true, 128>(a, c, st) : attend_d<false, 128>(a, c, st);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace fma_dev

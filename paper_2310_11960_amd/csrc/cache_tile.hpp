// cache_tile.hpp -- 32 queries against a 32-row tile of keys and values in LDS, on
// the matrix cores:
//   S^T = K Q^T (row reads), P = exp2(c s - m), l += the sum of P,
//   O^T += V^T P^T (bf16: transposing reads)
// on v_mfma_f32_32x32x16_bf16 or v_mfma_f32_32x32x2_f32.  m is the running maximum
// and l adds P as bf16 has rounded it, so that a dominating source weighs exactly
// 1.  (A reference that follows only when passed by 2^8 was 4 % faster at d = 64
// and its error against float64 up to 6 % larger.)  m, l and O are fp32; P is
// rounded to bf16 for the second product, V's type.
//
// A weight of 0 does not hide an infinity or a NaN in a matrix product.  Where
// queries may lie before rows of a tile and a value row holds one (odd_rows), the
// kernel leaves the tile out and takes its rows one by one at the end, each for
// the queries that see it (late_rows).  This costs a few registers and a look at
// one or two tiles of a wave: 12 long pieces at rank 4 88.6 -> 93.2 us.
#pragma once

#include "cache_device.hpp"
#include "wave_ops.hpp"

namespace fma_dev {

namespace {

// A row's 16-byte chunk c lies at chunk c ^ chunk_swz(row).
template <bool BF16, int D>
__device__ inline int chunk_swz(int row)
{
    if constexpr (BF16) return swzd<D>(row);
    else return row & (D == 32 ? 7 : 15);
}

template <bool BF16, int D>
struct QueryTile {
    static constexpr int ND = D / 32, NC = BF16 ? D / 16 : D / 8, RB = D * (BF16 ? 2 : 4);   // row bytes
    uint4 qo[NC];      // this lane's half of query lane & 31
    float scale;
    int hh, l32, koff, voff[2];

    __device__ QueryTile(int lane, float scale_log2)
    {
        hh = lane >> 5;
        l32 = lane & 31;
        scale = fabsf(scale_log2);
    }
    // before the first tile
    __device__ void start(int lane)
    {
        koff = l32 * RB + 16 * (hh ^ chunk_swz<BF16, D>(l32));
        const int gq = lane >> 4, s4 = lane & 15, jr = s4 >> 2, qq = s4 & 3;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int r = 8 * k + 4 * (gq >> 1) + jr;
            voff[k] = r * D + 8 * ((2 * (gq & 1) + (qq >> 1)) ^ swzd<D>(r)) + 4 * (qq & 1);
        }
    }
    // a negative scale turns the query's sign, so that the greatest product is
    // the greatest score
    __device__ void load(const void *row, float scale_log2)
    {
        const char *p = static_cast<const char *>(row) + 16 * hh;
        const uint32_t sign = scale_log2 < 0.f ? (BF16 ? 0x80008000u : 0x80000000u) : 0u;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            qo[c] = *reinterpret_cast<const uint4 *>(p + 32 * c);
            qo[c].x ^= sign, qo[c].y ^= sign, qo[c].z ^= sign, qo[c].w ^= sign;
        }
    }
    // whether value rows of a tile hold an infinity or a NaN
    __device__ __attribute__((always_inline)) bool odd_rows(const char *vt) const
    {
        float z[4] = {0.f, 0.f, 0.f, 0.f};   // x * 0 is 0 but for those
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const f32x4 x = *reinterpret_cast<const f32x4 *>(vt + (koff ^ (32 * c)));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (BF16) {
                    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
                    const bf16x2 none = {static_cast<__bf16>(0.f), static_cast<__bf16>(0.f)};
                    const float w = x[j];
                    z[j] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), none, z[j], false);
                } else {
                    z[j] = fmaf(x[j], 0.f, z[j]);
                }
            }
        }
        return __builtin_amdgcn_ballot_w64((z[0] + z[1]) + (z[2] + z[3]) != 0.f) != 0;
    }
    // rows kt, vt (RB bytes each, swizzled); see: seen_rows of this lane's query; all: every
    // query of the wave sees every row; odd: value rows to leave out.  o: O^T, channels 32 db + grow(j, lane >> 5);
    // m, l: reference and this lane's part of the sum, log2 units.  (They are the
    // kernel's own variables: as members they cost a second copy of o.)
    __device__ __attribute__((always_inline)) void meet(const char *kt, const char *vt, uint32_t see, bool all,
                                                        f32x16 (&o)[ND], float &m, float &l) const
    {
        uint4 kf[NC];
        keys(kt, kf);
        meet(kf, vt, see, all, o, m, l);
    }
    // this lane's half of key row lane & 31 of a tile
    __device__ __attribute__((always_inline)) void keys(const char *kt, uint4 (&kf)[NC]) const
    {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            if constexpr (BF16)
                kf[c] = *reinterpret_cast<const uint4 *>(kt + (koff ^ (32 * c)));
            else
                kf[c] = __builtin_bit_cast(uint4, *reinterpret_cast<const f32x4 *>(kt + (koff ^ (32 * c))));
        }
    }
    __device__ __attribute__((always_inline)) void meet(const uint4 (&kf)[NC], const char *vt, uint32_t see, bool all,
                                                        f32x16 (&o)[ND], float &m, float &l) const
    {
        f32x16 s = {0};
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            if constexpr (BF16) {
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[c]),
                                                            __builtin_bit_cast(bf16x8, qo[c]), s, 0, 0, 0);
            } else {
                const f32x4 k = __builtin_bit_cast(f32x4, kf[c]), q = __builtin_bit_cast(f32x4, qo[c]);
#pragma unroll
                for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_32x32x2f32(k[j], q[j], s, 0, 0, 0);
            }
        }
        if (!all) {
#pragma unroll
            for (int j = 0; j < 16; ++j) s[j] = seen(see, j) ? s[j] : -INFINITY;
        }
        float mx = s[0];
#pragma unroll
        for (int j = 1; j < 16; ++j) mx = __builtin_elementwise_maximum(mx, s[j]);
        mx = pair_max(mx) * scale;
        const bool up = mx > m || m == -INFINITY;
        if (__builtin_amdgcn_ballot_w64(up) != 0) {
            const float mnew = up ? mx : m;
            const float corr = mnew == m ? 1.f : __builtin_amdgcn_exp2f(m - mnew);   // (-inf: still nothing seen)
            m = mnew;
            l *= corr;
#pragma unroll
            for (int db = 0; db < ND; ++db)
#pragma unroll
                for (int j = 0; j < 16; ++j) o[db][j] *= corr;
        }
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int j = 0; j < 16; ++j) s[j] = __builtin_amdgcn_exp2f(fmaf(s[j], scale, -ref));
        if constexpr (BF16) {
            typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
            const bf16x2 ones = {static_cast<__bf16>(1.0f), static_cast<__bf16>(1.0f)};
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                uint32_t w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    w[k] = pack_bf16(s[8 * hf + 2 * k], s[8 * hf + 2 * k + 1]);
                    l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w[k]), ones, l, false);
                }
                const uint4 pw = make_uint4(w[0], w[1], w[2], w[3]);
                const __bf16 *const v16 = reinterpret_cast<const __bf16 *>(vt) + 16 * hf * D;
#pragma unroll
                for (int db = 0; db < ND; ++db) {
                    const s16x4 r1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(v16 + (voff[0] ^ (32 * db))));
                    const s16x4 r2 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(v16 + (voff[1] ^ (32 * db))));
                    const s16x8 av = {r1[0], r1[1], r1[2], r1[3], r2[0], r2[1], r2[2], r2[3]};
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, av),
                                                                    __builtin_bit_cast(bf16x8, pw), o[db], 0, 0, 0);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                l += s[j];
                const int r = grow(j, hh), sw = chunk_swz<BF16, D>(r);
#pragma unroll
                for (int db = 0; db < ND; ++db) {
                    const float vf = *reinterpret_cast<const float *>(vt + r * RB + 16 * ((8 * db + (l32 >> 2)) ^ sw) + 4 * (l32 & 3));
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf, s[j], o[db], 0, 0, 0);
                }
            }
        }
    }
};

// The near rows of positions k0 .. k0 + 31, one by one, for the queries (at qpos)
// that see them.
template <bool BF16, int D>
__device__ inline void late_rows(const CacheArgs &a, const Tile &x, int h, int k0, const QueryTile<BF16, D> &qt, int qpos,
                                 f32x16 (&o)[D / 32], float &m, float &l)
{
    const int end = k0 + 32 < x.pos + x.n ? k0 + 32 : x.pos + x.n;
    for (int pos = k0; pos < end; ++pos) {
        const char *k, *v;
        const int page = page_of(a, x.seq, pos / a.r);
        if (a.k && pos >= x.start) {
            const long long n = x.row0 + pos - x.start;
            k = static_cast<const char *>(elem<BF16>(a.k, n * a.kt + h * a.kh));
            v = static_cast<const char *>(elem<BF16>(a.v, n * a.vt + h * a.vh));
        } else if (page >= 0) {
            const long long off = page_row(a, page, h, pos % a.r);
            k = static_cast<const char *>(elem<BF16>(const_cast<const void *>(a.kp), off));
            v = static_cast<const char *>(elem<BF16>(const_cast<const void *>(a.vp), off));
        } else {
            continue;
        }
        float s = 0.f;
#pragma unroll
        for (int c = 0; c < qt.NC; ++c) {
            constexpr int W = BF16 ? 8 : 4;   // channels of a 16-byte chunk
            const uint4 w = qt.qo[c];
            const uint32_t qw[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int j = 0; j < W; ++j) {
                const int ch = (2 * c + qt.hh) * W + j;
                if constexpr (BF16)
                    s = fmaf(__uint_as_float(j & 1 ? qw[j / 2] & 0xffff0000u : qw[j / 2] << 16),
                             static_cast<float>(reinterpret_cast<const __bf16 *>(k)[ch]), s);
                else
                    s = fmaf(__uint_as_float(qw[j]), reinterpret_cast<const float *>(k)[ch], s);
            }
        }
        s = pair_sum(s) * qt.scale;
        if (pos > qpos) continue;
        const float top = fmaxf(m, s), ref = top == -INFINITY ? 0.f : top;
        const float corr = __builtin_amdgcn_exp2f(m - ref), p = __builtin_amdgcn_exp2f(s - ref);
        m = top;
        l = l * corr + (qt.hh ? 0.f : p);   // (a lane's part)
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int ch = 32 * db + grow(j, qt.hh);
                float y;
                if constexpr (BF16) y = static_cast<float>(reinterpret_cast<const __bf16 *>(v)[ch]);
                else y = reinterpret_cast<const float *>(v)[ch];
                o[db][j] = fmaf(p, y, o[db][j] * corr);
            }
        }
    }
}

}  // namespace

}  // namespace fma_dev

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
// fp32 weights meet bf16 rows exactly: each weight is split into three bf16
// terms (8 + 8 + 8 bits), so that the sums keep fp32 accuracy.
//
// What bounds it: bytes.  The rows are read once and written once; the weights
// (r floats per set) come from L2.
#include "cache_device.hpp"
#include "lds_rows.hpp"

namespace fma_dev {

namespace {

constexpr int kThreads = 256;

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));   // the caller's weights

template <bool BF16, int D>
__global__ __launch_bounds__(kThreads) void cache_append_kernel(CacheArgs a, Tiling t)
{
    __shared__ SumSmem<D, kThreads> sm;
    Tile x;
    if (!find_tile(a, t, blockIdx.x, x)) return;
    const int h = blockIdx.y, b = x.pos / a.r;
    const int page = page_of(a, x.seq, b);
    copy_rows<BF16, D, kThreads>(a, x, h, page);
    if (a.sets && (x.pos + x.n) % a.r == 0) summarize<BF16, D, kThreads>(a, x, h, b, page, sm);
}

// Pass 1.  Workgroup: a block and two key heads (waves 0, 1: keys, values of the
// first, ..).  32 rows at a time; the next tile's rows are on their way while
// one is multiplied.
template <bool BF16, int D>
__global__ __launch_bounds__(kThreads) void cache_blocks_kernel(CacheArgs a, Tiling t)
{
    constexpr int LPR = D / 8, RPL = 64 / LPR, NL = 32 / RPL, ND = D / 32;   // rows of a load, loads of a tile
    constexpr int RB = D * (BF16 ? 2 : 4);
    __shared__ __attribute__((aligned(16))) char lds[kThreads / 64][32 * RB];
    Tile x;
    if (!find_tile(a, t, blockIdx.x, x)) return;
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = 2 * blockIdx.y + (wave >> 1), kv = wave & 1;
    if (h >= a.kv_heads) return;
    const int b = x.pos / a.r, pos_b = b * a.r, page = page_of(a, x.seq, b);
    const bool done = a.sets && x.pos + x.n == pos_b + a.r;
    const int dst = done ? summary_of(a, x.seq, b) : -1;
    const char *const in = static_cast<const char *>(elem<BF16>(kv ? a.v : a.k, h * (kv ? a.vh : a.kh)));
    const long long in_t = (kv ? a.vt : a.kt) * (BF16 ? 2 : 4);
    char *const pg = static_cast<char *>(elem<BF16>(kv ? a.vp : a.kp, page_row(a, page, h, 0)));
    char *const tile = lds[wave];
    const int lr = lane / LPR, lc = lane % LPR;

    Raw8<BF16> raw[NL];
    // rows row0 .. row0 + 31 of the block; new ones go on to the page
    auto fetch = [&](int row0) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int row = row0 + i * RPL + lr, pos = pos_b + row;
            raw[i] = Raw8<BF16>();
            if (row >= a.r) continue;   // (r = 16: half a tile)
            if (pos >= x.start) {
                if (pos < x.pos + x.n) raw[i] = load_raw<BF16>(in + (long long)(x.row0 + pos - x.start) * in_t + RB / LPR * lc);
            } else if (page >= 0 && dst >= 0) {
                raw[i] = load_raw<BF16>(pg + row * RB + RB / LPR * lc);
            }
        }
    };
    auto keep = [&](int row0) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int row = row0 + i * RPL + lr, pos = pos_b + row;
            if (row < a.r && pos >= x.pos && pos < x.pos + x.n && page >= 0)
                store_raw<BF16>(pg + row * RB + RB / LPR * lc, raw[i]);
            if (dst < 0) continue;
            const int tr = i * RPL + lr;
            if constexpr (BF16) {
                *reinterpret_cast<uint4 *>(tile + tr * RB + 16 * (lc ^ swzd<D>(tr))) =
                    make_uint4(raw[i].w[0], raw[i].w[1], raw[i].w[2], raw[i].w[3]);
            } else {
                float f[8];
                floats<BF16>(raw[i], f);
                f32x4 *to = reinterpret_cast<f32x4 *>(tile + tr * RB + 32 * lc);
                to[0] = f32x4{f[0], f[1], f[2], f[3]};
                to[1] = f32x4{f[4], f[5], f[6], f[7]};
            }
        }
    };

    // set s0 + l32 is this lane's column
    for (int s0 = 0; s0 == 0 || s0 < a.sets; s0 += 32) {
        const int e = s0 + l32;
        const bool col = dst >= 0 && e < a.sets;
        const float *w = kv ? a.wv : a.wk;
        if (col) {
            const int l = e / a.rank, s = e - l * a.rank;
            const long long size = (long long)a.r << l;
            w += h * a.w_stride + a.rank * (size - a.r) + s * size + (long long)(b & ((1 << l) - 1)) * a.r;
        }
        f32x16 o[ND];
#pragma unroll
        for (int db = 0; db < ND; ++db) o[db] = f32x16{0};
        fetch(0);
        for (int row0 = 0; row0 < a.r; row0 += 32) {
            keep(row0);
            if (row0 + 32 < a.r) fetch(row0 + 32);
            if (dst < 0) continue;
            // rows 4 hh + .. of every eight in this lane's half
            float wf[16];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f32x4u x4 = {0.f, 0.f, 0.f, 0.f};
                if (col && row0 + 8 * i < a.r) x4 = *reinterpret_cast<const f32x4u *>(w + row0 + 8 * i + 4 * hh);
#pragma unroll
                for (int j = 0; j < 4; ++j) wf[4 * i + j] = x4[j];
            }
            if constexpr (BF16) {
                const int gq = lane >> 4, s4 = lane & 15, jr = s4 >> 2, qq = s4 & 3;
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    // the weights as three bf16 terms, each the rounding of what is left
                    bf16x8 ws[3];
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
                    for (int db = 0; db < ND; ++db) {
                        s16x4 r[2];
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const int row = 16 * hf + 8 * k + 4 * (gq >> 1) + jr;
                            const int off = row * D + ((8 * ((2 * (gq & 1) + (qq >> 1)) ^ swzd<D>(row)) + 4 * (qq & 1)) ^ (32 * db));
                            r[k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(reinterpret_cast<__bf16 *>(tile) + off));
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
                    const float *xr = reinterpret_cast<const float *>(tile) + grow(j, hh) * D + l32;
#pragma unroll
                    for (int db = 0; db < ND; ++db)
                        o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(xr[32 * db], wf[j], o[db], 0, 0, 0);
                }
            }
        }
        if (col) {
            float *const to = a.sum + ((((long long)dst * a.kv_heads + h) * 2 + kv) * a.sets + e) * D;
#pragma unroll
            for (int db = 0; db < ND; ++db)
#pragma unroll
                for (int j = 0; j < 16; j += 4)
                    *reinterpret_cast<f32x4 *>(to + 32 * db + grow(j, hh)) = f32x4{o[db][j], o[db][j + 1], o[db][j + 2], o[db][j + 3]};
        }
    }
}

// Pass 2: thread (sequence, head, four channels of a set) walks the blocks that
// the call completed, kScan of them on their way at a time.
constexpr int kScan = 16;

__global__ __launch_bounds__(64) void cache_scan_kernel(CacheArgs a)
{
    const int seq = blockIdx.x, h = blockIdx.y;
    const int col = 4 * (blockIdx.z * 64 + threadIdx.x), cols = 2 * a.sets * a.head_dim;
    if (col >= cols) return;
    const int c0 = a.cu[seq], c1 = a.cu[seq + 1], s = a.start[seq];
    if (!sequence_fits(a, c0, c1, s)) return;
    const int l = col / a.head_dim % a.sets / a.rank;
    if (l == 0) return;   // a group of level 1 is one block
    const int b0 = s / a.r, b1 = (s + c1 - c0) / a.r;
    if (b0 == b1) return;
    auto at = [&](int b) -> f32x4 * {
        const int p = b >= 0 && b < b1 ? summary_of(a, seq, b) : -1;
        return p < 0 ? nullptr : reinterpret_cast<f32x4 *>(a.sum + ((long long)p * a.kv_heads + h) * cols + col);
    };
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    const f32x4 *const prev = at(b0 - 1);
    f32x4 acc = prev ? *prev : zero;
    for (int b = b0; b < b1; b += kScan) {
        f32x4 *p[kScan], own[kScan];
#pragma unroll
        for (int i = 0; i < kScan; ++i) p[i] = at(b + i);
#pragma unroll
        for (int i = 0; i < kScan; ++i) own[i] = p[i] ? *p[i] : zero;
#pragma unroll
        for (int i = 0; i < kScan; ++i) {
            acc = (b + i) & ((1 << l) - 1) ? acc + own[i] : own[i];
            if (p[i])
                *p[i] = acc;
            else
                acc = zero;   // the sums of a missing page count as zero
        }
    }
}

template <bool BF16, int D>
hipError_t append_d(const CacheArgs &a, hipStream_t st)
{
    const Tiling t = make_tiling(a, a.r);
    if (a.max_chunk <= a.r) {
        hipLaunchKernelGGL((cache_append_kernel<BF16, D>), dim3((unsigned)t.units, a.kv_heads), dim3(kThreads), 0, st, a, t);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((cache_blocks_kernel<BF16, D>), dim3((unsigned)t.units, (a.kv_heads + 1) / 2), dim3(kThreads), 0, st,
                       a, t);
    if (a.levels > 1)
        hipLaunchKernelGGL(cache_scan_kernel, dim3(a.S, a.kv_heads, (2 * a.sets * D / 4 + 63) / 64), dim3(64), 0, st, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_append(const CacheArgs &a, hipStream_t st)
{
    if (a.S == 0 || a.rows == 0 || a.max_chunk == 0) return hipSuccess;
    switch (a.head_dim) {
    case 32: return a.bf16 ? append_d<true, 32>(a, st) : append_d<false, 32>(a, st);
    case 64: return a.bf16 ? append_d<true, 64>(a, st) : append_d<false, 64>(a, st);
    case 128: return a.bf16 ? append_d<true, 128>(a, st) : append_d<false, 128>(a, st);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace fma_dev

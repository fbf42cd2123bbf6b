// cache_token.hip -- FMA attention of at most four query rows per key head over
// the paged cache: single tokens, with shared key heads or a short draft, and in
// the same launch their way into the cache.
//
// What bounds it: the 2 r rows in sight, 48 KB per (sequence, key head) at r =
// 128 and d = 64 on average, are read once and meet four rows at most, so the
// matrix cores would idle; the arithmetic is on the vector ALU, in fp32, and
// the loads are whole rows.  d / 8 lanes hold a row of keys and of values; every
// row slot of the workgroup (64 / (d / 8) in each of 8 waves) keeps its own
// running maximum, sum and output, and nothing is exchanged until the end.
#include "cache_device.hpp"

namespace fma_dev {

namespace {

constexpr int kWaves = 8, kThreads = 64 * kWaves;

template <int D, int R>
struct TokenSmem {
    union {
        float o[kWaves][R][D];
        SumSmem<D, kThreads> sum;
    };
    float m[kWaves][R], l[kWaves][R];
};

template <bool BF16, int D, int R>
__global__ __launch_bounds__(kThreads) void cache_token_kernel(CacheArgs a, Tiling t)
{
    constexpr int LPR = D / 8, RPG = 64 / LPR, U = 4;   // rows of a wave's load
    __shared__ TokenSmem<D, R> sm;
    Tile x;
    if (!find_tile(a, t, blockIdx.x, x)) return;
    const int tid = threadIdx.x, lane = tid & 63, slot = lane / LPR, ch = 8 * (lane % LPR);
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = blockIdx.y, b = x.pos / a.r, pos_b = b * a.r;
    const int page = page_of(a, x.seq, b), page0 = b > 0 ? page_of(a, x.seq, b - 1) : -1;
    const int nrow = x.n * a.group;

    // far rows: level by level, one group or (odd q) two, each with all bases
    const int lq = b >= 2 ? 31 - __builtin_clz((unsigned)b) : 0, nlev = lq < a.levels ? lq : a.levels;
    const int nfar = a.rank * (nlev + __popc(b & ((1 << nlev) - 1)));
    auto far_row = [&](int i) -> const float * {   // key row of far source i, NULL if missing
        if (i >= nfar) return nullptr;
        int lv = 0, c = a.rank << (b & 1);
        while (i >= c) {
            i -= c;
            ++lv;
            c = a.rank << (b >> lv & 1);
        }
        const int two = i >= a.rank, g = (b >> lv) - 2 - two;
        const int sp = summary_of(a, x.seq, ((g + 1) << lv) - 1);
        return sp < 0 ? nullptr : a.sum + (((long long)sp * a.kv_heads + h) * 2 * a.sets + lv * a.rank + i - two * a.rank) * D + ch;
    };
    // (the waves take their far rows from the last one down: the near ones start at the first)
    const int fgroups = (nfar + RPG - 1) / RPG, fg0 = kWaves - 1 - wave;
    const float *far = fg0 < fgroups ? far_row(fg0 * RPG + slot) : nullptr;

    float q[R][8];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int qi = i < nrow ? i / a.group : 0, gi = i < nrow ? i - qi * a.group : 0;
        load8f<BF16>(elem<BF16>(a.q, (long long)(x.row + qi) * a.qt + (h * a.group + gi) * a.qh + ch), q[i]);
#pragma unroll
        for (int c = 0; c < 8; ++c) q[i][c] *= a.scale_log2;
    }

    float m[R], l[R], o[R][8];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        m[i] = -INFINITY;
        l[i] = 0.f;
#pragma unroll
        for (int c = 0; c < 8; ++c) o[i][c] = 0.f;
    }
    // one row of keys and values, at position pos, against the queries
    auto meet = [&](const float (&k)[8], const float (&v)[8], bool valid, int pos) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            float s = 0.f;
#pragma unroll
            for (int c = 0; c < 8; ++c) s = fmaf(q[i][c], k[c], s);
            s = row_sum<LPR>(s);
            const bool seen = valid && (R == 1 || pos <= x.pos + i / a.group);
            s = seen ? s : -INFINITY;
            const float mn = fmaxf(m[i], s), ref = mn == -INFINITY ? 0.f : mn;
            const float corr = __builtin_amdgcn_exp2f(m[i] - ref), p = __builtin_amdgcn_exp2f(s - ref);
            m[i] = mn;
            l[i] = fmaf(l[i], corr, p);
#pragma unroll
            for (int c = 0; c < 8; ++c) o[i][c] = fmaf(o[i][c], corr, p * v[c]);
        }
    };

    const int klo = b > 0 ? pos_b - a.r : 0, kend = x.pos + x.n;
    const int ngroups = (kend - klo + RPG - 1) / RPG;
    for (int g0 = wave; g0 < ngroups; g0 += kWaves * U) {
        Raw8<BF16> kk[U], vv[U];
        bool valid[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int pos = klo + (g0 + u * kWaves) * RPG + slot;
            const bool fresh = a.k && pos >= x.start;
            const int pg = pos >= pos_b ? page : page0;
            valid[u] = pos < kend && (fresh || pg >= 0);
            kk[u] = Raw8<BF16>();
            vv[u] = Raw8<BF16>();
            if (!valid[u]) continue;
            if (fresh) {
                const long long row = x.row0 + pos - x.start;
                kk[u] = load_raw<BF16>(elem<BF16>(a.k, row * a.kt + h * a.kh + ch));
                vv[u] = load_raw<BF16>(elem<BF16>(a.v, row * a.vt + h * a.vh + ch));
            } else {
                const long long off = page_row(a, pg, h, pos >= pos_b ? pos - pos_b : pos - klo) + ch;
                kk[u] = load_raw<BF16>(elem<BF16>(const_cast<const void *>(a.kp), off));
                vv[u] = load_raw<BF16>(elem<BF16>(const_cast<const void *>(a.vp), off));
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (g0 + u * kWaves >= ngroups) continue;
            float k[8], v[8];
            floats<BF16>(kk[u], k);
            floats<BF16>(vv[u], v);
            meet(k, v, valid[u], klo + (g0 + u * kWaves) * RPG + slot);
        }
    }
    for (int g = fg0; g < fgroups; g += kWaves) {
        if (g != fg0) far = far_row(g * RPG + slot);
        float k[8], v[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) k[c] = v[c] = 0.f;
        if (far) {
            load8f<false>(far, k);
            load8f<false>(far + (long long)a.sets * D, v);
        }
        meet(k, v, far != nullptr, 0);
    }
    if (a.write) copy_rows<BF16, D, kThreads>(a, x, h, page);

    // the slots of the wave, then the waves
#pragma unroll
    for (int i = 0; i < R; ++i) {
        float top = m[i];
#pragma unroll
        for (int k = LPR; k < 64; k *= 2) top = fmaxf(top, __shfl_xor(top, k));
        // (a slot without a score adds its zeros, or a NaN score's NaN)
        const float f = m[i] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[i] - top);
        l[i] *= f;
#pragma unroll
        for (int c = 0; c < 8; ++c) o[i][c] *= f;
#pragma unroll
        for (int k = LPR; k < 64; k *= 2) {
            l[i] += __shfl_xor(l[i], k);
#pragma unroll
            for (int c = 0; c < 8; ++c) o[i][c] += __shfl_xor(o[i][c], k);
        }
        if (lane < LPR) {
#pragma unroll
            for (int c = 0; c < 8; ++c) sm.o[wave][i][ch + c] = o[i][c];
            if (lane == 0) {
                sm.m[wave][i] = top;
                sm.l[wave][i] = l[i];
            }
        }
    }
    __syncthreads();
    for (int i = tid; i < nrow * D; i += kThreads) {
        const int row = i / D, c = i % D, qi = row / a.group;
        float top = -INFINITY, num = 0.f, den = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sm.m[w][row]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = sm.m[w][row] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(sm.m[w][row] - top);
            num = fmaf(sm.o[w][row][c], f, num);
            den = fmaf(sm.l[w][row], f, den);
        }
        const float y = den == 0.f ? 0.f : num / den;   // a row that sees nothing is zero
        const long long off = (long long)(x.row + qi) * a.ot + (h * a.group + row - qi * a.group) * a.oh + c;
        if constexpr (BF16)
            static_cast<__bf16 *>(a.out)[off] = static_cast<__bf16>(y);
        else
            static_cast<float *>(a.out)[off] = y;
    }
    if (a.write && a.sets && kend % a.r == 0) {
        __syncthreads();
        summarize<BF16, D, kThreads>(a, x, h, b, page, sm.sum);
    }
}

template <bool BF16, int D>
hipError_t token_d(const CacheArgs &a, hipStream_t st)
{
    const int most = a.max_chunk < a.rows ? a.max_chunk : a.rows;
    const Tiling t = make_tiling(a, most);
    const dim3 grid((unsigned)t.units, a.kv_heads);
    switch (most * a.group) {
    case 1: hipLaunchKernelGGL((cache_token_kernel<BF16, D, 1>), grid, dim3(kThreads), 0, st, a, t); break;
    case 2: hipLaunchKernelGGL((cache_token_kernel<BF16, D, 2>), grid, dim3(kThreads), 0, st, a, t); break;
    default: hipLaunchKernelGGL((cache_token_kernel<BF16, D, 4>), grid, dim3(kThreads), 0, st, a, t); break;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_token(const CacheArgs &a, hipStream_t st)
{
    switch (a.head_dim) {
    case 32: return a.bf16 ? token_d<true, 32>(a, st) : token_d<false, 32>(a, st);
    case 64: return a.bf16 ? token_d<true, 64>(a, st) : token_d<false, 64>(a, st);
    case 128: return a.bf16 ? token_d<true, 128>(a, st) : token_d<false, 128>(a, st);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace fma_dev

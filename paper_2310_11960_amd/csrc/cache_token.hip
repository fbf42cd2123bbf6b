// cache_token.hip -- FMA attention of at most four query rows per key head over
// the paged cache: single tokens, with shared key heads or a short draft, and in
// the same launch their way into the cache.
//
// What bounds it: the 2 r rows in sight, 48 KB per (sequence, key head) at r =
// 128 and d = 64 on average, are read once and meet four rows at most, so the
// matrix cores would idle; the arithmetic is on the vector ALU, in fp32, and
// the loads are whole rows.  d / 8 lanes hold a row of keys and of values; every
// row slot of the workgroup (64 / (d / 8) in each of 4 waves) keeps its own
// running maximum, sum and output, and nothing is exchanged until the end.
#include <type_traits>

#include "cache_device.hpp"

namespace fma_dev {

namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;

template <bool BF16, int D, int R>
struct TokenSmem {
    union {
        float o[kWaves][R][D];
        __attribute__((aligned(16))) char sum[kWaves][kSumTile<BF16>];
    };
    float m[kWaves][R], l[kWaves][R];
};

// A query's channels as this lane holds them; bf16 pairs meet the key's in two-term
// products with an fp32 sum.
template <bool BF16>
struct Query {
    Raw8<BF16> raw;
    __device__ float dot(const Raw8<BF16> &k) const
    {
        float s = 0.f;
#pragma unroll
        for (int c = 0; c < Raw8<BF16>::W; ++c) {
            if constexpr (BF16) {
                typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
                s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, raw.w[c]),
                                                    __builtin_bit_cast(bf16x2, k.w[c]), s, false);
            } else {
                s = fmaf(__uint_as_float(raw.w[c]), __uint_as_float(k.w[c]), s);
            }
        }
        return s;
    }
};

struct Source {
    int lo, hi, page, fresh;   // positions [lo, hi)
};

template <bool BF16, int D, int R>
__global__ __launch_bounds__(kThreads) void cache_token_kernel(CacheArgs a, Tiling t)
{
    constexpr int LPR = D / 8, RPG = 64 / LPR, U = 4;   // rows of a wave's load
    __shared__ TokenSmem<BF16, D, R> sm;
    Tile x;
    const CacheGroup cg = cache_group(a.kv_heads);
    if (!find_tile(a, t, cg.unit, x)) return;
    const int tid = threadIdx.x, lane = tid & 63, slot = lane / LPR, ch = 8 * (lane % LPR);
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = cg.head, b = x.pos / a.r, pos_b = b * a.r;
    const int page = page_of(a, x.seq, b), page0 = b > 0 ? page_of(a, x.seq, b - 1) : -1;
    const int nrow = x.n * a.group;

    const bool completes = a.write && a.sets && (x.pos + x.n) % a.r == 0;
    const int dst = completes ? summary_of(a, x.seq, b) : -1, before = completes && b > 0 ? summary_of(a, x.seq, b - 1) : -1;

    // (the waves take their far rows from the last one down: the near ones start at the first)
    const FarList list(a, b);
    const int fgroups = (list.n + RPG - 1) / RPG, fg0 = kWaves - 1 - wave;
    const float *far = fg0 < fgroups ? list.row(a, x.seq, h, fg0 * RPG + slot) : nullptr;

    Query<BF16> q[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int qi = i < nrow ? i / a.group : 0, gi = i < nrow ? i - qi * a.group : 0;
        q[i].raw = load_raw<BF16>(elem<BF16>(a.q, (long long)(x.row + qi) * a.qt + (h * a.group + gi) * a.qh + ch));
    }

    float m[R], l[R], o[R][8];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        m[i] = -INFINITY;
        l[i] = 0.f;
#pragma unroll
        for (int c = 0; c < 8; ++c) o[i][c] = 0.f;
    }
    // N rows of keys and values against the queries: one rescaling for all
    auto meet = [&](auto n, const Raw8<BF16> *k, const Raw8<BF16> *v, const bool *valid, const int *pos)
                    __attribute__((always_inline)) {
        constexpr int N = decltype(n)::value;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            float s[N], top = m[i];
#pragma unroll
            for (int u = 0; u < N; ++u) {
                s[u] = row_sum<LPR>(q[i].dot(k[u])) * a.scale_log2;
                s[u] = valid[u] && (R == 1 || pos[u] <= x.pos + i / a.group) ? s[u] : -INFINITY;
                top = fmaxf(top, s[u]);
            }
            const float ref = top == -INFINITY ? 0.f : top;   // nothing seen yet
            const float corr = __builtin_amdgcn_exp2f(m[i] - ref);
            m[i] = top;
            l[i] *= corr;
#pragma unroll
            for (int c = 0; c < 8; ++c) o[i][c] *= corr;
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const float p = __builtin_amdgcn_exp2f(s[u] - ref);
                float f[8];
                floats<BF16>(v[u], f);
                l[i] += p;
                if (R > 1 && s[u] == -INFINITY) continue;   // (0 times a later row's infinity is no number)
#pragma unroll
                for (int c = 0; c < 8; ++c) o[i][c] = fmaf(p, f[c], o[i][c]);
            }
        }
    };

    // near rows in groups of RPG that share a source: the previous block's page,
    // the own block's, the caller's tensors
    const int split = a.k ? (x.start < pos_b ? pos_b : x.start) : x.pos + x.n;   // own block's first fresh position
    const int old = a.k && x.start < pos_b ? x.start : pos_b;                    // previous block's: fresh from there
    const int klo = b > 0 ? pos_b - a.r : 0, kend = x.pos + x.n;
    const Source src[4] = {{klo, old, page0, 0}, {old, pos_b, -1, 1}, {pos_b, split, page, 0}, {split, kend, -1, 1}};
    int gn[4], total = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        gn[i] = (src[i].hi - src[i].lo + RPG - 1) / RPG;
        if (!src[i].fresh && src[i].page < 0) gn[i] = 0;
        total += gn[i];
    }
    for (int g0 = wave; g0 < total; g0 += kWaves * U) {
        Raw8<BF16> kk[U], vv[U];
        bool valid[U];
        int pos[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            int g = g0 + u * kWaves;   // uniform: group g of source i
            kk[u] = Raw8<BF16>();
            vv[u] = Raw8<BF16>();
            valid[u] = false;
            pos[u] = 0;
            if (g >= total) continue;
            int i = 0;
            if (g >= gn[0]) {
                g -= gn[0], i = 1;
                if (g >= gn[1]) {
                    g -= gn[1], i = 2;
                    if (g >= gn[2]) g -= gn[2], i = 3;
                }
            }
            const int lo = i == 0 ? klo : i == 1 ? old : i == 2 ? pos_b : split;
            const int hi = i == 0 ? old : i == 1 ? pos_b : i == 2 ? split : kend;
            pos[u] = lo + g * RPG + slot;
            valid[u] = pos[u] < hi;
            const int row = g * RPG + (valid[u] ? slot : 0);   // of the source (a group has a first row)
            const char *kb, *vb;
            int step_k, step_v;
            if (i & 1) {
                const long long r0 = x.row0 + lo - x.start;
                kb = static_cast<const char *>(elem<BF16>(a.k, r0 * a.kt + h * a.kh));
                vb = static_cast<const char *>(elem<BF16>(a.v, r0 * a.vt + h * a.vh));
                kb += row * a.kt * (BF16 ? 2 : 4);
                vb += row * a.vt * (BF16 ? 2 : 4);
                step_k = step_v = 0;
            } else {
                const long long off = page_row(a, i ? page : page0, h, 0);
                kb = static_cast<const char *>(elem<BF16>(const_cast<const void *>(a.kp), off));
                vb = static_cast<const char *>(elem<BF16>(const_cast<const void *>(a.vp), off));
                step_k = step_v = row * D * (BF16 ? 2 : 4);
            }
            const int c0 = ch * (BF16 ? 2 : 4);
            kk[u] = load_raw<BF16>(kb + (step_k + c0));
            vv[u] = load_raw<BF16>(vb + (step_v + c0));
        }
        meet(std::integral_constant<int, U>(), kk, vv, valid, pos);
    }
    for (int g = fg0; g < fgroups; g += kWaves) {
        if (g != fg0) far = list.row(a, x.seq, h, g * RPG + slot);
        Raw8<BF16> kf = Raw8<BF16>(), vf = Raw8<BF16>();
        if (far) {
            // fp32 rows, rounded to the cache's type as the dense path keeps them
            float f[8];
            load8f<false>(far + ch, f);
            kf = rounded<BF16>(f);
            load8f<false>(far + (long long)a.sets * D + ch, f);
            vf = rounded<BF16>(f);
        }
        const bool valid = far != nullptr;
        const int pos = 0;
        meet(std::integral_constant<int, 1>(), &kf, &vf, &valid, &pos);
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
    if (dst >= 0) {
        __syncthreads();
        summarize<BF16, D, kWaves>(a, x, h, b, page, dst, before, sm.sum[wave]);
    }
}

template <bool BF16, int D>
hipError_t token_d(const CacheArgs &a, hipStream_t st)
{
    const Tiling t = make_tiling(a, token_tile(a));
    const dim3 grid((unsigned)(t.units * a.kv_heads));
    switch (token_tile(a) * a.group) {
    case 1: hipLaunchKernelGGL((cache_token_kernel<BF16, D, 1>), grid, dim3(kThreads), 0, st, a, t); break;
    case 2: hipLaunchKernelGGL((cache_token_kernel<BF16, D, 2>), grid, dim3(kThreads), 0, st, a, t); break;
    default:   // (token_rows)
        if constexpr (!BF16 || D > 64) hipLaunchKernelGGL((cache_token_kernel<BF16, D, 4>), grid, dim3(kThreads), 0, st, a, t);
        else return hipErrorInvalidValue;
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

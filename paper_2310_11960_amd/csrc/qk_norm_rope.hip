// qk_norm_rope.hip -- per-head RMS norm and rotation of queries and keys, the
// values' copy, and the backward pass, from any strides to any strides.
//
//   forward   z = gamma x rs, rs = 1 / sqrt(mean x^2 + eps);  y = z c + z~ s
//   backward  z = g c - g~ s, u = gamma z, x^ = x rs:
//             dx = rs (u - x^ mean(u x^)),  dgamma = sum over rows of z x^
// where ~ is the pair's other channel, c the cosine and s the sine with the
// sign of the channel's side (c = 1, s = 0 beyond the rotated channels).
//
// d / 8 lanes hold a row, eight adjacent channels (16 bytes of bf16, 32 of
// fp32) each, and keep their token while they walk its heads, so the angles
// and gammas are formed once for all of them.  An angle is position x rate in
// fp64 turns, reduced to half a turn before it is rounded to fp32.  A pair
// that lies in two lanes is exchanged between them, raw in the forward.
//
// What bounds it: bytes; nothing is read twice.
#include "qk_norm_rope.hpp"

#include <type_traits>

#include "row_lanes.hpp"

namespace fma_dev {

namespace {

constexpr int kThreads = 256;

template <bool BF16>
__device__ inline Raw8<BF16> load8(const QkView &x, long long off)
{
    return load_raw<BF16>(static_cast<const char *>(x.p) + off * (BF16 ? 2 : 4));
}

template <bool BF16>
__device__ inline void store8(const QkView &x, long long off, const Raw8<BF16> &r)
{
    store_raw<BF16>(static_cast<char *>(x.p) + off * (BF16 ? 2 : 4), r);
}

// What a lane keeps of its token: cosine and signed sine of its channels.
struct Turn {
    float c[8], s[8];
    int peer;       // lane of the pairs' other channels (halves); -1: none of them rotated elsewhere
};

template <int D, bool IL>
__device__ inline Turn token_turn(const QkArgs &a, long long row, int t, int lane)
{
    constexpr int LPR = D / 8;
    Turn r;
    const int ch = 8 * (lane % LPR), sec = a.rotary / a.axes, half = sec / 2;
    r.peer = lane;
#pragma unroll
    for (int i = 0; i < 8; ++i) r.c[i] = 1.f, r.s[i] = 0.f;
    if (ch >= a.rotary) return r;
    const int axis = ch >= sec ? 1 : 0, in = ch - axis * sec;   // sec is a multiple of 16
    int p;
    if (a.pos)
        p = a.pos[row * a.axes + axis];
    else
        p = a.axes == 1 ? t : axis ? t % a.side : t / a.side;
    constexpr int NP = IL ? 4 : 8;
    const bool low = IL || in < half;
    const int pair = IL ? in / 2 : low ? in : in - half;
    if (!IL) r.peer = low ? lane + half / 8 : lane - half / 8;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const double turns = (double)p * a.turns[pair + i];
        float sn, cs;
        sincospif(2.f * (float)(turns - rint(turns)), &sn, &cs);
        if constexpr (IL) {
            r.c[2 * i] = r.c[2 * i + 1] = cs;
            r.s[2 * i] = -sn;
            r.s[2 * i + 1] = sn;
        } else {
            r.c[i] = cs;
            r.s[i] = low ? -sn : sn;
        }
    }
    return r;
}

template <int D>
__device__ inline void load_gamma(const float *g, int ch, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = g ? g[ch + i] : 1.f;
}

__device__ inline long long at(const QkView &x, int b, int h, int t)
{
    return b * x.bs + h * x.hs + t * x.ts;
}

// Forward.  Workgroup (x, y): tokens x * TPB .. of all, tasks [y * per, ..) of
// heads + 2 kv_heads: query heads, key heads, value heads.
template <bool BF16, int D, bool IL>
__global__ __launch_bounds__(kThreads) void qk_forward_kernel(QkArgs a, int per)
{
    constexpr int LPR = D / 8, TPB = kThreads / LPR, U = 4, W = Raw8<BF16>::W;
    const int tid = threadIdx.x, lane = tid & 63;
    const long long row = (long long)blockIdx.x * TPB + tid / LPR;
    const bool live = row < a.rows;   // the others repeat row 0 and store nothing
    const int b = live ? (int)row / a.tokens : 0, t = live ? (int)row - b * a.tokens : 0;
    const int ch = 8 * (lane % LPR);
    const int lo = blockIdx.y * per, all = a.heads + (a.has_v ? 2 : 1) * a.kv_heads;
    const int hi = lo + per < all ? lo + per : all, nqk = a.heads + a.kv_heads;
    Turn tu;
    float gq[8], gk[8], pq[8], pk[8];   // gammas of the own and the pair's channels
    if (lo < nqk) {
        tu = token_turn<D, IL>(a, live ? row : 0, t, lane);
        const int pch = IL ? ch : 8 * (tu.peer % LPR);
        load_gamma<D>(a.gamma_q, ch, gq);
        load_gamma<D>(a.gamma_k, ch, gk);
        if constexpr (!IL) {
            load_gamma<D>(a.gamma_q, pch, pq);
            load_gamma<D>(a.gamma_k, pch, pk);
        }
    }
    for (int i0 = lo; i0 < hi; i0 += U) {
        Raw8<BF16> x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u;
            if (i >= hi) continue;
            if (i < a.heads)
                x[u] = load8<BF16>(a.q, at(a.q, b, i, t) + ch);
            else if (i < nqk)
                x[u] = load8<BF16>(a.k, at(a.k, b, i - a.heads, t) + ch);
            else
                x[u] = load8<BF16>(a.v, at(a.v, b, i - nqk, t) + ch);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u;
            if (i >= hi) continue;
            Raw8<BF16> y = x[u];
            if (i < nqk) {
                float f[8], z[8];
                floats<BF16>(x[u], f);
                float ss = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) ss = fmaf(f[j], f[j], ss);
                const float rs = rsqrtf(row_sum<LPR>(ss) * (1.f / D) + a.eps);
                const bool isq = i < a.heads;
#pragma unroll
                for (int j = 0; j < 8; ++j) z[j] = f[j] * rs * (isq ? gq[j] : gk[j]);
                float o[8];
                if constexpr (IL) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) o[j] = fmaf(z[j ^ 1], tu.s[j], z[j] * tu.c[j]);
                } else {
                    Raw8<BF16> other;
#pragma unroll
                    for (int j = 0; j < W; ++j) other.w[j] = __shfl((int)x[u].w[j], tu.peer);
                    floats<BF16>(other, f);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        o[j] = fmaf(f[j] * rs * (isq ? pq[j] : pk[j]), tu.s[j], z[j] * tu.c[j]);
                }
                y = rounded<BF16>(o);
            }
            if (!live) continue;
            if (i < a.heads) {
                store8<BF16>(a.qo, at(a.qo, b, i, t) + ch, y);
            } else {
                const QkView &dst = i < nqk ? a.ko : a.vo;
                const int h = (i < nqk ? i - a.heads : i - nqk) * a.rep;
                for (int m = 0; m < a.rep; ++m) store8<BF16>(dst, at(dst, b, h + m, t) + ch, y);
            }
        }
    }
}

// Backward.  Workgroup w walks token tiles w, w + groups, .. with all heads; its
// sums of the gammas' gradients go to part[w].
template <bool BF16, int D, bool IL, bool SHARED>
__global__ __launch_bounds__(kThreads) void qk_backward_kernel(QkArgs a, int tiles, int ny, int per)
{
    constexpr int LPR = D / 8, TPB = kThreads / LPR;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int ch = 8 * (lane % LPR);
    const int nqk = a.heads + a.kv_heads, all = nqk + (a.has_v ? a.kv_heads : 0);
    const int gy = blockIdx.x % ny, gx = blockIdx.x / ny, gcount = gridDim.x / ny;
    const int lo = gy * per, hi = lo + per < all ? lo + per : all;
    float gq[8], gk[8], sq[8], sk[8];
    load_gamma<D>(a.gamma_q, ch, gq);
    load_gamma<D>(a.gamma_k, ch, gk);
#pragma unroll
    for (int j = 0; j < 8; ++j) sq[j] = sk[j] = 0.f;
    for (int tile = gx; tile < tiles; tile += gcount) {
        const long long row = (long long)tile * TPB + tid / LPR;
        const bool live = row < a.rows;   // the others repeat row 0 and add and store nothing
        const int b = live ? (int)row / a.tokens : 0, t = live ? (int)row - b * a.tokens : 0;
        const Turn tu = token_turn<D, IL>(a, live ? row : 0, t, lane);
        auto head = [&](int i) { return i < a.heads ? i : i < nqk ? i - a.heads : i - nqk; };
        auto input = [&](int i) {   // (values have none: their gradient goes through)
            const QkView &xv = i < a.heads ? a.q : a.k;
            return i < nqk ? load8<BF16>(xv, at(xv, b, head(i), t) + ch) : Raw8<BF16>();
        };
        auto upstream = [&](int i, int m) {   // of copy m of the head
            const QkView &gv = i < a.heads ? a.qo : i < nqk ? a.ko : a.vo;
            return load8<BF16>(gv, at(gv, b, head(i) * (i < a.heads ? 1 : a.rep) + m, t) + ch);
        };
        // one row: its gradient g in, the input's out
        auto finish = [&](int i, const Raw8<BF16> &raw, float (&g)[8]) __attribute__((always_inline)) {
            const bool isq = i < a.heads;
            if (i < nqk) {
                float x[8], z[8], ss = 0.f, ux = 0.f;
                floats<BF16>(raw, x);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float other = IL ? g[j ^ 1] : __shfl(g[j], tu.peer);
                    z[j] = fmaf(-other, tu.s[j], g[j] * tu.c[j]);
                    ss = fmaf(x[j], x[j], ss);
                }
                const float rs = rsqrtf(row_sum<LPR>(ss) * (1.f / D) + a.eps);
                float u[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    x[j] *= rs;
                    u[j] = z[j] * (isq ? gq[j] : gk[j]);
                    ux = fmaf(u[j], x[j], ux);
                    if (live) {
                        if (isq)
                            sq[j] = fmaf(z[j], x[j], sq[j]);
                        else
                            sk[j] = fmaf(z[j], x[j], sk[j]);
                    }
                }
                const float m = row_sum<LPR>(ux) * (1.f / D);
#pragma unroll
                for (int j = 0; j < 8; ++j) g[j] = rs * fmaf(-x[j], m, u[j]);
            }
            const QkView &dv = isq ? a.dq : i < nqk ? a.dk : a.dv;
            if (live) store8<BF16>(dv, at(dv, b, head(i), t) + ch, rounded<BF16>(g));
        };
        // heads of their own, two at a time: 4 KB per wave on the way
        const int one = SHARED && hi > a.heads ? (lo > a.heads ? lo : a.heads) : hi;
        for (int i0 = lo; i0 < one; i0 += 2) {
            Raw8<BF16> x[2], g[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int i = i0 + u < one ? i0 + u : i0;
                x[u] = input(i);
                g[u] = upstream(i, 0);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (i0 + u >= one) continue;
                float f[8];
                floats<BF16>(g[u], f);
                finish(i0 + u, x[u], f);
            }
        }
        if constexpr (SHARED) {   // shared heads: their copies' gradients, four at a time
            for (int i = one; i < hi; ++i) {
                const Raw8<BF16> x = input(i);
                float g[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) g[j] = 0.f;
                for (int m0 = 0; m0 < a.rep; m0 += 4) {
                    Raw8<BF16> more[4];
#pragma unroll
                    for (int m = 0; m < 4; ++m) more[m] = upstream(i, m0 + m < a.rep ? m0 + m : m0);
#pragma unroll
                    for (int m = 0; m < 4; ++m) {
                        if (m0 + m >= a.rep) continue;
                        float f[8];
                        floats<BF16>(more[m], f);
#pragma unroll
                        for (int j = 0; j < 8; ++j) g[j] += f[j];
                    }
                }
                finish(i, x, g);
            }
        }
    }
    // the lanes of a channel across the wave, then the four waves
    __shared__ float sum[kThreads / 64][2][D];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
#pragma unroll
        for (int m = LPR; m < 64; m *= 2) {
            sq[j] += __shfl_xor(sq[j], m);
            sk[j] += __shfl_xor(sk[j], m);
        }
    }
    if (lane < LPR) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            sum[wave][0][ch + j] = sq[j];
            sum[wave][1][ch + j] = sk[j];
        }
    }
    __syncthreads();
    for (int i = tid; i < 2 * D; i += kThreads) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < kThreads / 64; ++w) s += sum[w][i / D][i % D];
        a.part[(long long)blockIdx.x * 2 * D + i] = s;
    }
}

// dgamma from the workgroups' sums: workgroup c adds columns 16 c .. of the 2 d.
__global__ __launch_bounds__(1024) void qk_gamma_kernel(QkArgs a, int groups)
{
    const int col = 16 * blockIdx.x + (threadIdx.x & 15), d = a.head_dim;
    float s = 0.f;
#pragma unroll 8
    for (int g = threadIdx.x >> 4; g < groups; g += 64) s += a.part[(long long)g * 2 * d + col];
    __shared__ float part[64][17];
    part[threadIdx.x >> 4][threadIdx.x & 15] = s;
    __syncthreads();
    if (threadIdx.x < 16) {
        float x = 0.f;
        for (int i = 0; i < 64; ++i) x += part[i][threadIdx.x];
        float *dst = col < d ? a.dgamma_q : a.dgamma_k;
        if (dst) dst[col % d] = x;
    }
}

// Tasks (heads) of a workgroup: all of a token's, so that its angles are formed
// once, unless that leaves fewer than `want` workgroups.
int tasks_per_group(long long tiles, int tasks, long long want)
{
    long long split = (want + tiles - 1) / tiles;
    if (split > tasks) split = tasks;
    return (int)((tasks + split - 1) / split);
}

constexpr long long kForwardGroups = 1024, kBackwardGroups = 1024;

long long token_tiles(long long rows, int d) { return (rows + kThreads / (d / 8) - 1) / (kThreads / (d / 8)); }

struct BackwardGrid {
    int ny, per;
    long long groups;
};

BackwardGrid backward_grid(long long rows, int tasks, int d)
{
    const long long tiles = token_tiles(rows, d);
    BackwardGrid g;
    g.per = tasks_per_group(tiles, tasks, kForwardGroups);
    g.ny = (tasks + g.per - 1) / g.per;
    long long x = kBackwardGroups / g.ny;
    if (x < 1) x = 1;
    if (x > tiles) x = tiles;
    g.groups = x * g.ny;
    return g;
}

template <bool BF16, int D>
hipError_t forward_d(const QkArgs &a, hipStream_t st)
{
    const long long tiles = token_tiles(a.rows, D);
    const int tasks = a.heads + (a.has_v ? 2 : 1) * a.kv_heads;
    const int per = tasks_per_group(tiles, tasks, kForwardGroups);
    const dim3 grid((unsigned)tiles, (unsigned)((tasks + per - 1) / per));
    if (a.interleaved)
        hipLaunchKernelGGL((qk_forward_kernel<BF16, D, true>), grid, dim3(kThreads), 0, st, a, per);
    else
        hipLaunchKernelGGL((qk_forward_kernel<BF16, D, false>), grid, dim3(kThreads), 0, st, a, per);
    return hipGetLastError();
}

template <bool BF16, int D>
hipError_t backward_d(const QkArgs &a, hipStream_t st)
{
    const int tasks = a.heads + (a.has_v ? 2 : 1) * a.kv_heads;
    BackwardGrid g = {0, 0, 0};   // no rows: the gammas' gradients are sums of nothing
    if (a.rows) g = backward_grid(a.rows, tasks, D);
    const int tiles = (int)token_tiles(a.rows, D);
    auto launch = [&](auto il, auto shared) {
        hipLaunchKernelGGL((qk_backward_kernel<BF16, D, decltype(il)::value, decltype(shared)::value>), dim3((unsigned)g.groups),
                           dim3(kThreads), 0, st, a, tiles, g.ny, g.per);
    };
    typedef std::true_type Yes;
    typedef std::false_type No;
    if (g.groups && a.interleaved) a.rep > 1 ? launch(Yes(), Yes()) : launch(Yes(), No());
    if (g.groups && !a.interleaved) a.rep > 1 ? launch(No(), Yes()) : launch(No(), No());
    if (a.dgamma_q || a.dgamma_k)
        hipLaunchKernelGGL(qk_gamma_kernel, dim3(2 * D / 16), dim3(1024), 0, st, a, (int)g.groups);
    return hipGetLastError();
}

}  // namespace

long long qk_backward_groups(long long rows, int tasks, int head_dim)
{
    return backward_grid(rows, tasks, head_dim).groups;
}

hipError_t launch_qk(const QkArgs &a, hipStream_t st)
{
    switch (a.head_dim) {
    case 32: return a.dtype_bf16 ? forward_d<true, 32>(a, st) : forward_d<false, 32>(a, st);
    case 64: return a.dtype_bf16 ? forward_d<true, 64>(a, st) : forward_d<false, 64>(a, st);
    case 128: return a.dtype_bf16 ? forward_d<true, 128>(a, st) : forward_d<false, 128>(a, st);
    default: return hipErrorInvalidValue;
    }
}

hipError_t launch_qk_backward(const QkArgs &a, hipStream_t st)
{
    switch (a.head_dim) {
    case 32: return a.dtype_bf16 ? backward_d<true, 32>(a, st) : backward_d<false, 32>(a, st);
    case 64: return a.dtype_bf16 ? backward_d<true, 64>(a, st) : backward_d<false, 64>(a, st);
    case 128: return a.dtype_bf16 ? backward_d<true, 128>(a, st) : backward_d<false, 128>(a, st);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace fma_dev

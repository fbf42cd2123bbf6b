// row_lanes.hpp -- rows of d channels held by d / 8 adjacent lanes, eight
// channels each.
#pragma once

#include "fma_device.hpp"

namespace fma_dev {

namespace {

template <bool BF16>
struct Raw8 {                              // eight channels as they lie in memory
    static constexpr int W = BF16 ? 4 : 8;
    uint32_t w[W];
};

template <bool BF16>
__device__ inline Raw8<BF16> load_raw(const void *p)
{
    Raw8<BF16> r;
    const uint4 a = static_cast<const uint4 *>(p)[0];
    r.w[0] = a.x, r.w[1] = a.y, r.w[2] = a.z, r.w[3] = a.w;
    if constexpr (!BF16) {
        const uint4 b = static_cast<const uint4 *>(p)[1];
        r.w[4] = b.x, r.w[5] = b.y, r.w[6] = b.z, r.w[7] = b.w;
    }
    return r;
}

template <bool BF16>
__device__ inline void store_raw(void *p, const Raw8<BF16> &r)
{
    static_cast<uint4 *>(p)[0] = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
    if constexpr (!BF16) static_cast<uint4 *>(p)[1] = make_uint4(r.w[4], r.w[5], r.w[6], r.w[7]);
}

template <bool BF16>
__device__ inline void floats(const Raw8<BF16> &r, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (BF16)
            x[i] = i & 1 ? bf16hi_to_f32(r.w[i / 2]) : bf16lo_to_f32(r.w[i / 2]);
        else
            x[i] = __uint_as_float(r.w[i]);
    }
}

// the one rounding of a result: to the nearest of its type
template <bool BF16>
__device__ inline Raw8<BF16> rounded(const float (&x)[8])
{
    Raw8<BF16> r;
#pragma unroll
    for (int i = 0; i < Raw8<BF16>::W; ++i) {
        if constexpr (BF16) {
            typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
            const bf16x2 p = {static_cast<__bf16>(x[2 * i]), static_cast<__bf16>(x[2 * i + 1])};
            r.w[i] = __builtin_bit_cast(uint32_t, p);
        } else {
            r.w[i] = __float_as_uint(x[i]);
        }
    }
    return r;
}

template <int CTRL>
__device__ inline float dpp_add(float x)
{
    const int y = __builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true);
    return x + __int_as_float(y);
}

// sum over the N = 4, 8 or 16 adjacent lanes of a row (quad permutes, then
// mirrors of the half row and the row: VALU exchanges)
template <int N>
__device__ inline float row_sum(float x)
{
    x = dpp_add<0xB1>(x);                       // lane ^ 1
    x = dpp_add<0x4E>(x);                       // lane ^ 2
    if constexpr (N >= 8) x = dpp_add<0x141>(x);
    if constexpr (N >= 16) x = dpp_add<0x140>(x);
    return x;
}

}  // namespace

}  // namespace fma_dev

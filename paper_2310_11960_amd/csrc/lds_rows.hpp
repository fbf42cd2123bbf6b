// lds_rows.hpp -- bf16 rows in LDS as the 32x32 matrix operands read them:
// swizzled 16-byte chunks, and the transposing reads.
#pragma once

#include "fma_device.hpp"

namespace fma_dev {

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// The swizzle keeps both the row reads of a 32x32 operand (lane = row) and the
// transposing reads (four rows of two chunks per 16 lanes) on distinct banks;
// rows are 64, 128 or 256 bytes.
template <int D>
__device__ inline int swzd(int row)
{
    const int s64 = (2 * (row & 3)) ^ ((row >> 2) & 1) ^ (2 * ((row >> 3) & 1));
    if constexpr (D == 32) return (2 * ((row >> 1) & 1)) ^ ((row >> 2) & 1);
    else if constexpr (D == 64) return s64;
    else return s64 ^ (8 * (row & 1));
}

__device__ inline int grow(int i, int hh) { return 8 * (i >> 2) + 4 * hh + (i & 3); }   // accumulator row

}  // namespace

}  // namespace fma_dev

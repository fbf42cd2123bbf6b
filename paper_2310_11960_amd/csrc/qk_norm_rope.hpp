// qk_norm_rope.hpp -- arguments and launchers of the norm and rotation of
// queries and keys (internal to the library).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fma_dev {

// [batch][heads][tokens][d], element strides
struct QkView {
    void *p;
    long long bs, hs, ts;
};

constexpr int kMaxPairs = 64;

struct QkArgs {
    QkView q, k, v;                  // inputs (backward: q and k alone)
    QkView qo, ko, vo;               // outputs (backward: their gradients, inputs)
    QkView dq, dk, dv;               // backward: gradients of the inputs
    const float *gamma_q, *gamma_k;  // NULL: ones
    const int32_t *pos;              // [batch][tokens][axes]; NULL: the token's index
    float *part;                     // backward: [workgroups][2][d] partial gradients of the gammas
    float *dgamma_q, *dgamma_k;      // NULL: not wanted
    long long rows;                  // batch * tokens < 2^28 (threads of a launch stay below 2^32)
    int tokens;
    int heads, kv_heads, rep;        // rep: copies of a key / value head that leave
    int has_v;
    int side, axes, rotary, interleaved;
    int dtype_bf16, head_dim;
    float eps;
    double turns[kMaxPairs];         // rates of an axis' pairs, turns per position
};

// Workgroups of the backward pass (its partial sums' rows).
long long qk_backward_groups(long long rows, int tasks, int head_dim);
hipError_t launch_qk(const QkArgs &a, hipStream_t st);
hipError_t launch_qk_backward(const QkArgs &a, hipStream_t st);

}  // namespace fma_dev

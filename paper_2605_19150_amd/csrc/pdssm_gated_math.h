// pdssm_gated_math.h -- the gates of the gated linear recurrence for one
// entry, shared by its forward, backward and single-step kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pdssm_gated.h"
#include "pdssm_rows.h"

namespace pdssm {

// A gate logit at or under this one holds the state: a = 1, no input and no
// gradient, whatever the other rows hold (padding: the type's lowest value or
// -inf).  sigmoid(-64) is 1.6e-28, so s = rate * r stays a normal number for
// every gate that is not held and every rate from 1e-10 on; where it does not,
// a = 1 and beta = 0, and the gradients are those of a held row.
constexpr float kGateHold = -64.f;

__device__ __forceinline__ float sigmoid_f(float v) {
    // 1 / (1 + 2^(-v log2 e)); the power overflows to inf for v < -88 and the
    // reciprocal of that is the 0 it should be
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * -1.44269504088896340736f));
}

constexpr float kLog2e = 1.44269504088896340736f;

// A channel's rate.  One that is not positive and finite is no rate of this
// recurrence: as a NaN it makes s, a and beta of every row NaN, also where r is
// 0.  (Left as it is, 0 would hold the state, infinity give y = i x, and a
// negative one a beta^2 below 0, which the backward pass takes for a held row.)
__device__ __forceinline__ float rate_of(float rate) {
    return rate > 0.f && rate < INFINITY ? rate : __uint_as_float(0x7fc00000u);
}

// a = e^(-s) and beta^2 = 1 - a^2 of one entry, s = rate * r.  Long memories
// have s of 1e-3 and less, where two things need care: the difference 1 - a^2
// keeps only its last bits, and the hardware's exponential is off by 6e-9 to
// one side, which a recurrence adds up over the 1 / s rows that it remembers.
// So up to s = 0.15 drop = 1 - a comes from a polynomial (4e-8 of it off, to
// both sides), a = 1 - drop is the nearest number but for the rounding of drop,
// and beta^2 = drop (1 + a) is off by 2e-7 of itself at most; from there on 1 - a
// is exact to 3e-7.
struct Decay {
    float s, a;
    float beta2;   // 1 - a^2, beta squared
};

__device__ __forceinline__ Decay decay_of(float r, float rate) {
    Decay d;
    d.s = rate * r;
    const float e = __builtin_amdgcn_exp2f(d.s * -kLog2e);
    const bool near = d.s < 0.15f;
    float p = fmaf(d.s, -3.9347485e-2f, 0.16646752f);
    p = fmaf(d.s, p, -0.49999511f);
    p = fmaf(d.s, p, 1.f);
    const float drop = near ? d.s * p : 1.f - e;
    d.a = near ? 1.f - drop : e;
    d.beta2 = fmaf(drop, d.a, drop);
    return d;
}

}  // namespace pdssm

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
// every gate that is not held.
constexpr float kGateHold = -64.f;

__device__ __forceinline__ float sigmoid_f(float v) {
    // 1 / (1 + 2^(-v log2 e)); the power overflows to inf for v < -88 and the
    // reciprocal of that is the 0 it should be
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * -1.44269504088896340736f));
}

// e^(-s) - 1 for s >= 0, to about 3e-7 of its value.  Near 0 the difference
// of e^(-s) and 1 would keep only its last bits (s is rate * r, often 1e-3 and
// less), so there the Taylor series takes over: up to s = 0.2 its first
// omitted term is under 2e-8 of the sum.
__device__ __forceinline__ float expm1_neg(float s) {
    float p = fmaf(s, -1.f / 720.f, 1.f / 120.f);
    p = fmaf(-s, p, 1.f / 24.f);
    p = fmaf(-s, p, 1.f / 6.f);
    p = fmaf(-s, p, 0.5f);
    p = fmaf(-s, p, 1.f);
    const float far = __builtin_amdgcn_exp2f(s * -1.44269504088896340736f) - 1.f;
    return s < 0.2f ? -s * p : far;
}

struct Gate {
    float r, i;   // sigmoid of the two gate logits; r = 0 where the state is held
    float em;     // a - 1
    float beta;   // sqrt(1 - a^2) = sqrt(-em (2 + em))
    bool hold;
};

__device__ __forceinline__ Gate gate_of(float ga, float gi, float rate) {
    Gate g;
    g.hold = ga <= kGateHold;
    g.r = g.hold ? 0.f : sigmoid_f(ga);
    g.i = sigmoid_f(gi);
    g.em = expm1_neg(rate * g.r);
    g.beta = __builtin_amdgcn_sqrtf(-g.em * (2.f + g.em));
    return g;
}

}  // namespace pdssm

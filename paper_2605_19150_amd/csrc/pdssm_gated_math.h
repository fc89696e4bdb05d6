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

// a = e^(-s) and beta^2 = 1 - a^2 of one entry.  The latter needs care near
// a = 1, where the difference keeps only its last bits (s is rate * r, often
// 1e-3 and less): 1 - e^(-2s) = 2 e^(-s) sinh(s), and sinh's series converges
// fast.  Up to s = 0.3 its first omitted term is 1.5e-7 of the sum; from there
// on 1 - a^2 is off by 4e-7 of itself.  With v = s log2 e the powers of ln 2
// sit in the coefficients.
struct Decay {
    float a;
    float beta2;   // 1 - a^2, beta squared
};

__device__ __forceinline__ Decay decay_of(float r, float rate2) {  // rate2 = rate * log2 e
    Decay d;
    const float v = rate2 * r, u = v * v;
    d.a = __builtin_amdgcn_exp2f(-v);
    // 2 ln2 (1 + (ln2 v)^2 / 6 + (ln2 v)^4 / 120)
    const float p = fmaf(u, fmaf(u, 2.6667116e-3f, 0.11100822f), 1.3862944f);
    d.beta2 = v < 0.43280851f ? d.a * v * p : fmaf(-d.a, d.a, 1.f);
    return d;
}

constexpr float kLog2e = 1.44269504088896340736f;

}  // namespace pdssm

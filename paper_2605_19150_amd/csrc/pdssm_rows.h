// pdssm_rows.h -- entries of row tensors in registers: fp32, bf16 and the
// 8-bit form that activations are kept in between forward and backward.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pdssm_kept.h"

namespace pdssm {

// The 8-bit form: kKeptRows rows of a channel share an exponent e, the
// smallest one (at least -126) with 127 * 2^e >= the largest magnitude; an
// entry is the whole number q in [-127, 127] next to v * 2^-e, ties to even.
// Powers of two keep both ways free of any other rounding: v * 2^-e is exact,
// and q * 2^e, seven bits and a sign, is exact in bf16.  A value is off by at
// most 2^(e-1), 1/127 of the block's largest magnitude.
constexpr int kKeptPoison = -128;  // exponent of a block that held a NaN or an infinity: its values read NaN
constexpr int kKeptLow = -128;     // code of a held gate logit and of a shut input gate: reads -inf

// Exponent for the largest magnitude of a block, given as its bits (which
// order as the magnitudes do, NaN above infinity).
__device__ __forceinline__ int kept_exponent(uint32_t top) {
    if (top >= 0x7f800000u) return kKeptPoison;
    // top = (1 + m / 2^23) * 2^k with 127 * 2^(k-6) >= top up to m = 0x7e0000
    return max((int)(top >> 23) - 133 + ((top & 0x7fffffu) > 0x7e0000u ? 1 : 0), -126);
}
__device__ __forceinline__ float kept_scale(int e) {  // 2^e
    return e == kKeptPoison ? __uint_as_float(0x7fc00000u) : __uint_as_float((uint32_t)(e + 127) << 23);
}
__device__ __forceinline__ float kept_inverse(int e) {  // 2^-e, 0 for a poisoned block (whose codes say nothing)
    return e == kKeptPoison ? 0.f : __uint_as_float((uint32_t)(127 - e) << 23);
}
// Largest code of a block.  At the top exponent 122 the code 64 would stand for
// 2^128, which fp32 does not have: there codes end at 63.
__device__ __forceinline__ float kept_limit(int e) { return e == 122 ? 63.f : 127.f; }
// v * inverse to the nearest whole number (in a poisoned block any number but kKeptLow).
__device__ __forceinline__ int kept_code(float v, float inverse, float limit) {
    return (int)__builtin_rintf(__builtin_amdgcn_fmed3f(v * inverse, -limit, limit));
}
// The same where some entries have no part in the block's exponent: they may
// come to kKeptLow, which no other does.
__device__ __forceinline__ float kept_low(int e) { return e == kKeptPoison ? -127.f : (float)kKeptLow; }
__device__ __forceinline__ int kept_code_or_low(float v, float inverse, float low, float limit) {
    return (int)__builtin_rintf(__builtin_amdgcn_fmed3f(v * inverse, low, limit));
}

template <int IO>
struct Entry;
template <>
struct Entry<kRowF32> {
    using T = float;  // in memory
    static __device__ __forceinline__ float get(T v) { return v; }
    static __device__ __forceinline__ T put(float v) { return v; }
};
template <>
struct Entry<kRowBf16> {
    using T = uint16_t;
    static __device__ __forceinline__ float get(uint32_t v) { return __uint_as_float(v << 16); }
    // to nearest, ties to even: off by at most 2^-8 of the value, the one
    // rounding of an output
    static __device__ __forceinline__ T put(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
};

template <>
struct Entry<kRowKept> {
    using T = int8_t;
    // with the code of a held gate logit
    static __device__ __forceinline__ float get(int v, float scale) { return v == kKeptLow ? -INFINITY : (float)v * scale; }
};

}  // namespace pdssm

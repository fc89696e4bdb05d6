// pdssm_kept.h -- row tensors and their 8-bit form: formats and host-side
// launch interface (pdssm_kept.hip, pdssm_wgrad.hip).  Not installed; not part
// of the ABI.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace pdssm {

constexpr int kKeptRows = 32;     // rows that share an exponent in the 8-bit form

// Formats of a row tensor's entries.
constexpr int kRowF32 = 0;
constexpr int kRowBf16 = 1;
constexpr int kRowKept = 2;  // whole numbers of 8 bits and an exponent for kKeptRows rows of a channel

// A tensor of rows [T, C]: entry (t, c) at p + t * ld + c (ld in entries).
struct RowsIn {
    const void* p;
    int64_t ld;
    const int8_t* e;  // kRowKept: exponents [ceil(T / kKeptRows), C]
};

// The 8-bit form of u [T, C] (rows of ld entries, fp32 or bf16), and back.
hipError_t launch_pack8(int T, int C, int io, RowsIn u, int8_t* q, int8_t* e, hipStream_t s);
hipError_t launch_unpack8(int T, int C, int io, const int8_t* q, const int8_t* e, void* out, hipStream_t s);

// dW[m, d] = sum_t dP[t, m] u[t, d], u in the 8-bit form.
struct WgradArgs {
    int T, M, Dm;
    const uint16_t* dP;  // [T, M] bf16
    const int8_t* q;     // [T, Dm]
    const int8_t* e;     // [ceil(T / kKeptRows), Dm]
    float* dW;           // [M, Dm]
    void* ws;
};
size_t wgrad_workspace(int T, int M, int Dm);
hipError_t launch_wgrad(const WgradArgs& a, hipStream_t s);

}  // namespace pdssm

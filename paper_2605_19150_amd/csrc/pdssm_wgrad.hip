// pdssm_wgrad.hip -- weight gradient of a token projection, dW = dP^T u, from
// the 8-bit form of u, on the matrix cores (bf16 operands, fp32 sums).
#include "pdssm_device.h"
#include "pdssm_rows.h"

namespace pdssm {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// A workgroup of four waves sums a 64 x 64 block of dW; 32 tokens a step.
__global__ __launch_bounds__(256) void k_wgrad(WgradArgs a) {
    __shared__ uint16_t P[32][64], U[32][64];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int m0 = blockIdx.y * 64, d0 = blockIdx.x * 64;
    f32x16 acc;
    for (int r = 0; r < 16; ++r) acc[r] = 0.f;
    for (int t0 = 0; t0 < a.T; t0 += 32) {
        __syncthreads();
        for (int i = tid; i < 32 * 64; i += 256) {
            const int t = t0 + (i >> 6), c = i & 63;
            P[i >> 6][c] = t < a.T && m0 + c < a.M ? a.dP[(size_t)t * a.M + m0 + c] : 0;
            float v = 0.f;
            if (t < a.T && d0 + c < a.Dm)
                v = a.q[(size_t)t * a.Dm + d0 + c] * kept_scale(a.e[(size_t)(t0 / 32) * a.Dm + d0 + c]);
            U[i >> 6][c] = Entry<kRowBf16>::put(v);
        }
        __syncthreads();
        for (int k = 0; k < 32; k += 16) {
            bf16x8 A, B;
            for (int j = 0; j < 8; ++j) {
                A[j] = __builtin_bit_cast(__bf16, P[k + 8 * (lane >> 5) + j][(wv >> 1) * 32 + (lane & 31)]);
                B[j] = __builtin_bit_cast(__bf16, U[k + 8 * (lane >> 5) + j][(wv & 1) * 32 + (lane & 31)]);
            }
            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(A, B, acc, 0, 0, 0);
        }
    }
    for (int r = 0; r < 16; ++r) {
        const int m = m0 + (wv >> 1) * 32 + 8 * (r / 4) + 4 * (lane >> 5) + r % 4, d = d0 + (wv & 1) * 32 + (lane & 31);
        if (m < a.M && d < a.Dm) a.dW[(size_t)m * a.Dm + d] = acc[r];
    }
}

}  // namespace

size_t wgrad_workspace(int, int, int) { return 0; }

hipError_t launch_wgrad(const WgradArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(k_wgrad, dim3((a.Dm + 63) / 64, (a.M + 63) / 64), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace pdssm

// pdssm_kept.hip -- activations to the 8-bit form and back (pdssm_rows.h has
// the form).
#include "pdssm_device.h"
#include "pdssm_rows.h"

namespace pdssm {
namespace {

template <int IO>
__global__ void k_pack8(int T, int C, RowsIn u, int8_t* q, int8_t* e) {
    using En = Entry<IO>;
    const int c = blockIdx.x * 64 + threadIdx.x;
    if (c >= C) return;
    const int t0 = blockIdx.y * kKeptRows, t1 = min(t0 + kKeptRows, T);
    const auto* p = static_cast<const typename En::T*>(u.p);
    uint32_t top = 0;
    for (int t = t0; t < t1; ++t) top = max(top, __float_as_uint(En::get(p[(size_t)t * u.ld + c])) & 0x7fffffffu);
    const int ex = kept_exponent(top);
    e[(size_t)blockIdx.y * C + c] = (int8_t)ex;
    const float inv = kept_inverse(ex);
    for (int t = t0; t < t1; ++t) q[(size_t)t * C + c] = (int8_t)kept_code(En::get(p[(size_t)t * u.ld + c]), inv, kept_limit(ex));
}

template <int IO>
__global__ void k_unpack8(int T, int C, const int8_t* q, const int8_t* e, typename Entry<IO>::T* out) {
    const int c = blockIdx.x * 64 + threadIdx.x;
    if (c >= C) return;
    const int t0 = blockIdx.y * kKeptRows, t1 = min(t0 + kKeptRows, T);
    const float scale = kept_scale(e[(size_t)blockIdx.y * C + c]);
    for (int t = t0; t < t1; ++t) {
        const int v = q[(size_t)t * C + c];
        out[(size_t)t * C + c] = Entry<IO>::put(v == kKeptLow ? -INFINITY : v * scale);
    }
}

}  // namespace

hipError_t launch_pack8(int T, int C, int io, RowsIn u, int8_t* q, int8_t* e, hipStream_t s) {
    const dim3 g((C + 63) / 64, (T + kKeptRows - 1) / kKeptRows);
    if (io == kRowBf16) hipLaunchKernelGGL(k_pack8<kRowBf16>, g, dim3(64), 0, s, T, C, u, q, e);
    else hipLaunchKernelGGL(k_pack8<kRowF32>, g, dim3(64), 0, s, T, C, u, q, e);
    return hipGetLastError();
}
hipError_t launch_unpack8(int T, int C, int io, const int8_t* q, const int8_t* e, void* out, hipStream_t s) {
    const dim3 g((C + 63) / 64, (T + kKeptRows - 1) / kKeptRows);
    if (io == kRowBf16) hipLaunchKernelGGL(k_unpack8<kRowBf16>, g, dim3(64), 0, s, T, C, q, e, static_cast<uint16_t*>(out));
    else hipLaunchKernelGGL(k_unpack8<kRowF32>, g, dim3(64), 0, s, T, C, q, e, static_cast<float*>(out));
    return hipGetLastError();
}

}  // namespace pdssm

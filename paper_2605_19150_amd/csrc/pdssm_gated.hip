// pdssm_gated.hip -- the gated linear recurrence, forward, backward and single
// step.  For every channel c of a sequence, with r = sigmoid(ga), i =
// sigmoid(gi), s = rate[c] * r, a = e^(-s):
//
//   h_t = a_t h_{t-1} + sqrt(1 - a_t^2) i_t x_t,      y_t = h_t.
//
// Backward, with g_t the gradient reaching h_t (g_t = dy_t + a_{t+1} g_{t+1},
// dh_final added at a sequence's last row) and beta = sqrt(1 - a^2):
//
//   dx_t = g_t beta_t i_t              dgi_t = g_t beta_t x_t i_t (1 - i_t)
//   s ds_t = g_t s_t (i_t x_t a_t^2 / beta_t - a_t h_{t-1})
//   dga_t = s ds_t (1 - r_t)           drate = sum_t s ds_t / rate
//   dh0 = a_0 g_0
#include "pdssm_gated.h"

#include "pdssm_device.h"
#include "pdssm_gated_math.h"

namespace pdssm {
namespace {

__device__ __forceinline__ float row_get(const RowsIn& r, int io, int kept, int C, int t, int c, bool gate = false) {
    const size_t o = (size_t)t * r.ld + c;
    if (kept) {
        const int q = static_cast<const int8_t*>(r.p)[o];
        if (gate && q == kKeptLow) return -INFINITY;
        return (float)q * kept_scale(r.e[(size_t)(t / kKeptRows) * C + c]);
    }
    return io == kRowBf16 ? Entry<kRowBf16>::get(static_cast<const uint16_t*>(r.p)[o]) : static_cast<const float*>(r.p)[o];
}
__device__ __forceinline__ void row_put(void* p, size_t o, int io, float v) {
    if (io == kRowBf16) static_cast<uint16_t*>(p)[o] = Entry<kRowBf16>::put(v);
    else static_cast<float*>(p)[o] = v;
}

__device__ __forceinline__ void seq_rows(const GatedArgs& a, int s, int& t0, int& t1) {
    if (!a.cu) {
        t0 = s * a.L;
        t1 = t0 + a.L;
        return;
    }
    t0 = a.cu[s];
    t1 = a.cu[s + 1];
    bool bad = t0 < 0 || t1 < t0 || t1 > a.T || (s == 0 && t0 != 0);
    t0 = min(max(t0, 0), a.T);
    t1 = min(max(t1, t0), a.T);
    if (bad) report_index_error(a.status);
}

__global__ void k_gated_fwd(GatedArgs a) {
    const int c = blockIdx.x * blockDim.x + threadIdx.x, s = blockIdx.y;
    if (c >= a.C) return;
    int t0, t1;
    seq_rows(a, s, t0, t1);
    const float rate = a.rate[c];
    float h = a.h0 ? a.h0[(size_t)s * a.C + c] : 0.f;
    for (int t = t0; t < t1; ++t) {
        if (a.saved && t % kGatedChunk == 0) a.saved[(size_t)(t / kGatedChunk) * a.C + c] = t == t0 ? 0.f : h;
        const Gate g = gate_of(row_get(a.ga, a.io, 0, a.C, t, c), row_get(a.gi, a.io, 0, a.C, t, c), rate);
        const float b = g.hold ? 0.f : g.beta * g.i * row_get(a.x, a.io, 0, a.C, t, c);
        h = fmaf(1.f + g.em, h, b);
        row_put(a.y, (size_t)t * a.C + c, a.io, h);
    }
    if (a.h_final) a.h_final[(size_t)s * a.C + c] = h;
}

// The 8-bit form of x, ga and gi: rows of one block that lie in a sequence.
__global__ void k_gated_keep(GatedArgs a) {
    const int c = blockIdx.x * blockDim.x + threadIdx.x, k = blockIdx.y;
    if (c >= a.C) return;
    const int end = a.cu ? min(a.T, max(0, a.cu[a.S])) : a.T;
    const int t0 = k * kKeptRows, t1 = min(t0 + kKeptRows, end);
    if (t0 >= t1) return;
    for (int n = 0; n < 3; ++n) {
        const RowsIn& r = n == 0 ? a.x : n == 1 ? a.ga : a.gi;
        uint32_t top = 0;
        for (int t = t0; t < t1; ++t) {
            if (row_get(a.ga, a.io, 0, a.C, t, c) <= kGateHold) continue;
            top = max(top, __float_as_uint(row_get(r, a.io, 0, a.C, t, c)) & 0x7fffffffu);
        }
        const int e = kept_exponent(top);
        a.e[n][(size_t)k * a.C + c] = (int8_t)e;
        for (int t = t0; t < t1; ++t) {
            const bool hold = row_get(a.ga, a.io, 0, a.C, t, c) <= kGateHold;
            a.q[n][(size_t)t * a.C + c] =
                hold ? (n == 1 ? kKeptLow : 0) : (int8_t)kept_code(row_get(r, a.io, 0, a.C, t, c), kept_inverse(e), kept_limit(e));
        }
    }
}

__global__ void k_gated_bwd(GatedArgs a, float* part) {
    const int c = blockIdx.x * blockDim.x + threadIdx.x, s = blockIdx.y;
    if (c >= a.C) return;
    int t0, t1;
    seq_rows(a, s, t0, t1);
    const float rate = a.rate[c];
    float g = a.dhf ? a.dhf[(size_t)s * a.C + c] : 0.f, sum = 0.f;
    float before[kGatedChunk];
    for (int hi = t1; hi > t0;) {
        const int lo = max(t0, (hi - 1) / kGatedChunk * kGatedChunk);
        float h = lo > t0 ? a.saved[(size_t)(lo / kGatedChunk) * a.C + c] : a.h0 ? a.h0[(size_t)s * a.C + c] : 0.f;
        for (int t = lo; t < hi; ++t) {
            before[t - lo] = h;
            const Gate k = gate_of(row_get(a.ga, a.io, a.kept, a.C, t, c, true), row_get(a.gi, a.io, a.kept, a.C, t, c), rate);
            h = fmaf(1.f + k.em, h, k.hold ? 0.f : k.beta * k.i * row_get(a.x, a.io, a.kept, a.C, t, c));
        }
        for (int t = hi - 1; t >= lo; --t) {
            const Gate k = gate_of(row_get(a.ga, a.io, a.kept, a.C, t, c, true), row_get(a.gi, a.io, a.kept, a.C, t, c), rate);
            const float x = k.hold ? 0.f : row_get(a.x, a.io, a.kept, a.C, t, c);
            const float ac = 1.f + k.em, gi = k.hold ? 0.f : k.i, sr = rate * k.r;
            g += row_get(a.dy, a.io, 0, a.C, t, c);
            const float dx = g * k.beta * gi;
            const float ds = k.hold ? 0.f : g * sr * (gi * x * ac * ac / k.beta - ac * before[t - lo]);
            const size_t o = (size_t)t * a.ldd + c;
            row_put(a.d[0], o, a.io, k.hold ? 0.f : dx);
            row_put(a.d[1], o, a.io, ds * (1.f - k.r));
            row_put(a.d[2], o, a.io, k.hold ? 0.f : dx * x * (1.f - gi));
            sum += ds;
            g *= ac;
        }
        hi = lo;
    }
    if (a.dh0) a.dh0[(size_t)s * a.C + c] = g;
    part[(size_t)s * a.C + c] = sum;
}
__global__ void k_gated_rate(const float* part, const float* rate, float* drate, int n, int C) {
    const int c = blockIdx.x * blockDim.x + threadIdx.x;
    if (c >= C) return;
    float s = 0.f;
    for (int k = 0; k < n; ++k) s += part[(size_t)k * C + c];
    drate[c] = s / rate[c];
}

__global__ __launch_bounds__(256) void k_gated_step(GatedStepArgs a) {
    const int c = blockIdx.x * 256 + threadIdx.x, b = blockIdx.y;
    int slot = b;
    if (a.slots) {
        slot = a.slots[b];
        if (slot < 0 || slot >= a.pool) {
            if (slot >= a.pool) report_index_error(a.status);
            return;
        }
    }
    // the first row that names a slot has it; others of the same batch are refused
    bool again = false;
    if (a.slots)
        for (int k = threadIdx.x; k < b; k += 256) again |= a.slots[k] == slot;
    if (__syncthreads_or(again)) {
        report_index_error(a.status);
        return;
    }
    if (c >= a.C) return;
    const Gate g = gate_of(row_get(a.ga, a.io, 0, a.C, b, c), row_get(a.gi, a.io, 0, a.C, b, c), a.rate[c]);
    const size_t o = (size_t)slot * a.C + c;
    const float in = g.hold ? 0.f : g.beta * g.i * row_get(a.x, a.io, 0, a.C, b, c);
    const float h = fmaf(1.f + g.em, a.h_in[o], in);
    a.h_out[o] = h;
    row_put(a.y, (size_t)b * a.C + c, a.io, h);
}

}  // namespace

size_t gated_workspace(int T, int C, int S, bool bwd) { return bwd ? (size_t)S * C * 4 : 0; }

hipError_t launch_gated_fwd(const GatedArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(k_gated_fwd, dim3((a.C + 63) / 64, a.S), dim3(64), 0, s, a);
    if (a.q[0] && a.T)
        hipLaunchKernelGGL(k_gated_keep, dim3((a.C + 63) / 64, (a.T + kKeptRows - 1) / kKeptRows), dim3(64), 0, s, a);
    return hipGetLastError();
}
hipError_t launch_gated_bwd(const GatedArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(k_gated_bwd, dim3((a.C + 63) / 64, a.S), dim3(64), 0, s, a, static_cast<float*>(a.ws));
    if (a.drate)
        hipLaunchKernelGGL(k_gated_rate, dim3((a.C + 63) / 64), dim3(64), 0, s, static_cast<const float*>(a.ws), a.rate,
                           a.drate, a.S, a.C);
    return hipGetLastError();
}
hipError_t launch_gated_step(const GatedStepArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(k_gated_step, dim3((a.C + 255) / 256, a.B), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace pdssm

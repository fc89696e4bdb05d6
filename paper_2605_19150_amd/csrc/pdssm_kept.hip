// pdssm_kept.hip -- activations to the 8-bit form and back (pdssm_rows.h has
// the form).  Bound by HBM: one read, one write.  A wave has a block of 32 rows:
// where rows allow 16-byte accesses, 16 lanes side by side and four groups of 8
// rows, which agree on the largest magnitudes by two lane exchanges; else 64
// channels side by side, all 32 rows in each lane.  The rows stay in registers
// between the magnitude and the codes.  T32768 C4096 bf16 takes 89 to 99 us to
// the form and 63 to 65 back (407 MB: 4.1 to 4.6 and 6.3 to 6.5 TB/s; a large copy
// reaches 5.2), fp32 138 to 151 and 107 to 109 (675 MB).
#include "pdssm_device.h"
#include "pdssm_rows.h"

#include <initializer_list>

namespace pdssm {
namespace {

// How a wave covers a block with V entries a lane.
template <int V>
struct Cover {
    static constexpr int LANES = V > 1 ? 16 : 64;         // lanes side by side
    static constexpr int GROUPS = 64 / LANES;             // groups of rows
    static constexpr int ROWS = kKeptRows / GROUPS;       // rows of a lane
    static constexpr int WIDTH = LANES * V;               // channels of a wave
};

template <class T, int V>
struct __align__(V * sizeof(T)) Pack {
    T v[V];
};

struct Place {
    int k, c, row0;  // block, first channel, first row of the lane
    bool live;
};
template <int V>
__device__ __forceinline__ Place place_of(int T, int C) {
    using G = Cover<V>;
    const int lane = lane_id(), across = (C + G::WIDTH - 1) / G::WIDTH;
    const int64_t w = (int64_t)blockIdx.x * 4 + wave_id();
    Place p;
    p.k = (int)(w / across);
    p.c = (int)(w - (int64_t)p.k * across) * G::WIDTH + lane % G::LANES * V;
    p.row0 = p.k * kKeptRows + lane / G::LANES * G::ROWS;
    p.live = p.c < C && p.k < (T + kKeptRows - 1) / kKeptRows;
    return p;
}

template <int IO, int V>
__global__ __launch_bounds__(256) void k_pack8(int T, int C, RowsIn u, int8_t* q, int8_t* e) {
    using En = Entry<IO>;
    using G = Cover<V>;
    const Place at = place_of<V>(T, C);
    const auto* p = static_cast<const typename En::T*>(u.p);
    Pack<typename En::T, V> v[G::ROWS];
    uint32_t top[V] = {};
#pragma unroll
    for (int i = 0; i < G::ROWS; ++i)
        if (at.live && at.row0 + i < T)
            v[i] = *reinterpret_cast<const Pack<typename En::T, V>*>(p + (int64_t)(at.row0 + i) * u.ld + at.c);
        else
            v[i] = {};
#pragma unroll
    for (int i = 0; i < G::ROWS; ++i)
#pragma unroll
        for (int n = 0; n < V; ++n) top[n] = max(top[n], __float_as_uint(En::get(v[i].v[n])) & 0x7fffffffu);
    float inv[V], lim[V];
    Pack<int8_t, V> ex;
#pragma unroll
    for (int n = 0; n < V; ++n) {
#pragma unroll
        for (int m = G::LANES; m < 64; m *= 2) top[n] = max(top[n], (uint32_t)__shfl_xor((int)top[n], m));
        const int x = kept_exponent(top[n]);
        inv[n] = kept_inverse(x);
        lim[n] = kept_limit(x);
        ex.v[n] = (int8_t)x;
    }
    if (at.live && at.row0 == at.k * kKeptRows) *reinterpret_cast<Pack<int8_t, V>*>(e + (size_t)at.k * C + at.c) = ex;
#pragma unroll
    for (int i = 0; i < G::ROWS; ++i) {
        Pack<int8_t, V> w;
#pragma unroll
        for (int n = 0; n < V; ++n) w.v[n] = (int8_t)kept_code(En::get(v[i].v[n]), inv[n], lim[n]);
        if (at.live && at.row0 + i < T) *reinterpret_cast<Pack<int8_t, V>*>(q + (size_t)(at.row0 + i) * C + at.c) = w;
    }
}

template <int IO, int V>
__global__ __launch_bounds__(256) void k_unpack8(int T, int C, const int8_t* q, const int8_t* e, typename Entry<IO>::T* out) {
    using G = Cover<V>;
    const Place at = place_of<V>(T, C);
    if (!at.live) return;
    Pack<int8_t, V> v[G::ROWS];
    const Pack<int8_t, V> ex = *reinterpret_cast<const Pack<int8_t, V>*>(e + (size_t)at.k * C + at.c);
#pragma unroll
    for (int i = 0; i < G::ROWS; ++i)
        if (at.row0 + i < T) v[i] = *reinterpret_cast<const Pack<int8_t, V>*>(q + (size_t)(at.row0 + i) * C + at.c);
        else v[i] = {};
    float scale[V];
#pragma unroll
    for (int n = 0; n < V; ++n) scale[n] = kept_scale(ex.v[n]);
#pragma unroll
    for (int i = 0; i < G::ROWS; ++i) {
        Pack<typename Entry<IO>::T, V> w;
#pragma unroll
        for (int n = 0; n < V; ++n) w.v[n] = Entry<IO>::put(Entry<kRowKept>::get(v[i].v[n], scale[n]));
        if (at.row0 + i < T)
            *reinterpret_cast<Pack<typename Entry<IO>::T, V>*>(out + (size_t)(at.row0 + i) * C + at.c) = w;
    }
}

template <int V>
dim3 grid_of(int T, int C) {
    const int64_t waves = (int64_t)((T + kKeptRows - 1) / kKeptRows) * ((C + Cover<V>::WIDTH - 1) / Cover<V>::WIDTH);
    return dim3((unsigned)((waves + 3) / 4));
}

// Entries of a lane that fill 16 bytes, if every row begins at a multiple of them; else 1.
bool wide_ok(int io, int C, std::initializer_list<const void*> rows, std::initializer_list<const void*> bytes, int64_t ld) {
    const int V = io == kRowBf16 ? 8 : 4;
    if (C % V != 0 || ld % V != 0) return false;
    for (const void* p : rows)
        if (reinterpret_cast<uintptr_t>(p) % 16 != 0) return false;
    for (const void* p : bytes)
        if (reinterpret_cast<uintptr_t>(p) % V != 0) return false;
    return true;
}

}  // namespace

hipError_t launch_pack8(int T, int C, int io, RowsIn u, int8_t* q, int8_t* e, hipStream_t s) {
    const bool wide = wide_ok(io, C, {u.p}, {q, e}, u.ld);
    auto go = [&](auto* f, dim3 g) { hipLaunchKernelGGL(f, g, dim3(256), 0, s, T, C, u, q, e); };
    if (io == kRowBf16 && wide) go(k_pack8<kRowBf16, 8>, grid_of<8>(T, C));
    else if (io == kRowBf16) go(k_pack8<kRowBf16, 1>, grid_of<1>(T, C));
    else if (wide) go(k_pack8<kRowF32, 4>, grid_of<4>(T, C));
    else go(k_pack8<kRowF32, 1>, grid_of<1>(T, C));
    return hipGetLastError();
}

hipError_t launch_unpack8(int T, int C, int io, const int8_t* q, const int8_t* e, void* out, hipStream_t s) {
    const bool wide = wide_ok(io, C, {out}, {q, e}, C);
    if (io == kRowBf16) {
        auto* o = static_cast<uint16_t*>(out);
        if (wide) hipLaunchKernelGGL((k_unpack8<kRowBf16, 8>), grid_of<8>(T, C), dim3(256), 0, s, T, C, q, e, o);
        else hipLaunchKernelGGL((k_unpack8<kRowBf16, 1>), grid_of<1>(T, C), dim3(256), 0, s, T, C, q, e, o);
    } else {
        auto* o = static_cast<float*>(out);
        if (wide) hipLaunchKernelGGL((k_unpack8<kRowF32, 4>), grid_of<4>(T, C), dim3(256), 0, s, T, C, q, e, o);
        else hipLaunchKernelGGL((k_unpack8<kRowF32, 1>), grid_of<1>(T, C), dim3(256), 0, s, T, C, q, e, o);
    }
    return hipGetLastError();
}

}  // namespace pdssm

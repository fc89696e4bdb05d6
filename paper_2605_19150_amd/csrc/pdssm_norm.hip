// pdssm_norm.hip -- group norm of rows, channels last, with an activation or a
// gate behind it, forward and backward.
//
// For each row and group of c = C / G neighbouring channels
//   n = (x - mean) / sqrt(var + eps),   u = n w + b,
//   y = f(u), or u f(gate),             f(z) = z or z sigmoid(z).
// With du = dy f'(u), or dy f(gate):
//   db = sum du,  dw = sum du n (over the rows),  dgate = dy u f'(gate),
//   dn = du w,    dx = (dn - mean(dn) - n mean(dn n)) / sqrt(var + eps).
//
// Bound by memory: x, dy and gate are read once, y, dx and dgate written once.  A
// team of 1 to 64 neighbouring lanes has a group's row in registers, takes mean and
// variance of it in two passes over them, and goes from row to row with the same
// channels, so w, b and the sums over the rows stay in registers too; the sums of
// the blocks of rows are added in one order by a second kernel.  Groups that do not fit
// a wave's registers are read once for each pass by a workgroup.
#include <math.h>

#include <algorithm>

#include "pdssm_norm.h"
#include "pdssm_rows.h"

namespace pdssm {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlocks = 512;      // blocks of rows that a call of any width may have
constexpr int kNormWaves = 4096;  // waves that fill the card
// Bytes of a row tensor from which on rows go past the caches, which they would only sweep, if what a wave has of a
// row and the row are whole pieces of kPiece bytes.  At 32768 rows, bf16 with a gate: 4096 channels in 32 groups 167 ->
// 161 us forward, 298 -> 290 us backward, in 512 groups 164 -> 150 and 287 -> 275; 4080 channels, whose rows are not, in
// 170 groups 218 -> 224 and 376 -> 398, in 102 groups 222 -> 234 and 418 -> 416.
constexpr int64_t kPast = 64 << 20;
constexpr int kPiece = 64;

template <int IO, int V, bool PAST>
__device__ __forceinline__ void load(const void* p, size_t i, float* x) {
    using T = typename Entry<IO>::T;
    const T* q = static_cast<const T*>(p) + i;
    if constexpr (V * sizeof(T) == 16) {
        union {
            u32x4 u;
            T v[V];
        } t;
        t.u = PAST ? __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(q)) : *reinterpret_cast<const u32x4*>(q);
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] = Entry<IO>::get(t.v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] = Entry<IO>::get(q[e]);
    }
}
template <int IO, int V, bool PAST>
__device__ __forceinline__ void store(void* p, size_t i, const float* x) {
    using T = typename Entry<IO>::T;
    T* q = static_cast<T*>(p) + i;
    if constexpr (V * sizeof(T) == 16) {
        union {
            u32x4 u;
            T v[V];
        } t;
#pragma unroll
        for (int e = 0; e < V; ++e) t.v[e] = Entry<IO>::put(x[e]);
        if constexpr (PAST) __builtin_nontemporal_store(t.u, reinterpret_cast<u32x4*>(q));
        else *reinterpret_cast<u32x4*>(q) = t.u;
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) q[e] = Entry<IO>::put(x[e]);
    }
}

// f(z) and f'(z).  exp(-z) = 2^t (1 + r ln 2) with t + r = -z log2(e) to twice
// the digits: off by 2 units of the last place, at any z.  Below -88, where they are
// under 1e-36, silu and its slope count as 0, at -inf and the type's lowest value too;
// at +inf the slope is 1.
struct Act {
    float f, df;
};
template <bool SLOPE>
__device__ __forceinline__ Act act(float z, int silu) {
    if (!silu) return {z, 1.f};
    constexpr float kLog2e = 1.44269502f, kRest = 1.92596303e-8f;
    const float c = fminf(fmaxf(z, -88.f), 88.f);
    const float t = -c * kLog2e, r = fmaf(-c, kLog2e, -t) - c * kRest;
    const float e = __builtin_amdgcn_exp2f(t);
    const float s = __builtin_amdgcn_rcpf(1.f + fmaf(e, r * 0.693147182f, e));
    Act a;
    a.f = z < -88.f ? 0.f : z * s;
    if constexpr (SLOPE) {
        const float o = 1.f - s;
        a.df = z < -88.f ? 0.f : s * (1.f + (z > 88.f ? 0.f : z * o));
    }
    return a;
}

// The sum over a team's lanes, in each of them.
__device__ __forceinline__ float team_sum(float x, int team) {
    for (int m = team >> 1; m; m >>= 1) x += __shfl_xor(x, m);
    return x;
}

// What a lane has: vectors lane, lane + team, .. of a group's row.
template <int V, int NV>
struct Lane {
    int group, first, block;  // first: channel of the lane's first vector
    bool live;                // the group exists
    int left;                 // entries of the group from the lane's first one on
    __device__ __forceinline__ Lane(const NormArgs& a) {
        const int c = a.C / a.G, per = 64 / a.team, sets = (a.G + per - 1) / per;
        const int wave = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
        group = wave % sets * per + lane / a.team;
        block = wave / sets;
        const int at = lane % a.team * V;
        live = group < a.G;
        first = group * c + at;
        left = live ? c - at : 0;
    }
    __device__ __forceinline__ bool has(int k, int team) const { return k * team * V < left; }
};

template <int IO, int V, int NV, bool PAST>
__global__ __launch_bounds__(256) void k_norm_fwd(NormArgs a) {
    const Lane<V, NV> l(a);
    if (l.block >= a.blocks) return;
    float w[NV][V], b[NV][V];
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int c = l.first + k * a.team * V + e;
            const bool has = l.has(k, a.team);
            w[k][e] = has && a.w ? a.w[c] : 1.f;
            b[k][e] = has && a.b ? a.b[c] : 0.f;
        }
    const float inv = 1.f / (float)(a.C / a.G);
    for (int t = l.block; t < a.T; t += a.blocks) {
        float x[NV][V] = {}, z[NV][V] = {};
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (l.has(k, a.team)) {
                const size_t c = l.first + k * a.team * V;
                load<IO, V, PAST>(a.x.p, (size_t)t * a.x.ld + c, x[k]);
                if (a.gate.p) load<IO, V, PAST>(a.gate.p, (size_t)t * a.gate.ld + c, z[k]);
            }
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) sum += x[k][e];
        const float mean = team_sum(sum, a.team) * inv;
        sum = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                x[k][e] = l.has(k, a.team) ? x[k][e] - mean : 0.f;
                sum = fmaf(x[k][e], x[k][e], sum);
            }
        const float rstd = 1.f / sqrtf(fmaf(team_sum(sum, a.team), inv, a.eps));
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (l.has(k, a.team)) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float u = fmaf(x[k][e] * rstd, w[k][e], b[k][e]);
                    x[k][e] = a.gate.p ? u * act<false>(z[k][e], a.silu).f : act<false>(u, a.silu).f;
                }
                store<IO, V, PAST>(a.y, (size_t)t * a.C + l.first + k * a.team * V, x[k]);
            }
    }
}

template <int IO, int V, int NV, bool PAST>
__global__ __launch_bounds__(256) void k_norm_bwd(NormArgs a) {
    const Lane<V, NV> l(a);
    if (l.block >= a.blocks) return;
    float w[NV][V], b[NV][V], dw[NV][V] = {}, db[NV][V] = {};
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int c = l.first + k * a.team * V + e;
            const bool has = l.has(k, a.team);
            w[k][e] = has && a.w ? a.w[c] : 1.f;
            b[k][e] = has && a.b ? a.b[c] : 0.f;
        }
    const float inv = 1.f / (float)(a.C / a.G);
    for (int t = l.block; t < a.T; t += a.blocks) {
        float x[NV][V] = {}, z[NV][V] = {}, d[NV][V] = {};
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (l.has(k, a.team)) {
                const size_t c = l.first + k * a.team * V;
                load<IO, V, PAST>(a.x.p, (size_t)t * a.x.ld + c, x[k]);
                load<IO, V, PAST>(a.dy.p, (size_t)t * a.dy.ld + c, d[k]);
                if (a.gate.p) load<IO, V, PAST>(a.gate.p, (size_t)t * a.gate.ld + c, z[k]);
            }
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) sum += x[k][e];
        const float mean = team_sum(sum, a.team) * inv;
        sum = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                x[k][e] = l.has(k, a.team) ? x[k][e] - mean : 0.f;
                sum = fmaf(x[k][e], x[k][e], sum);
            }
        const float rstd = 1.f / sqrtf(fmaf(team_sum(sum, a.team), inv, a.eps));
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (l.has(k, a.team)) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float n = x[k][e] * rstd, u = fmaf(n, w[k][e], b[k][e]);
                    float du;
                    if (a.gate.p) {
                        const Act g = act<true>(z[k][e], a.silu);
                        du = d[k][e] * g.f;
                        z[k][e] = d[k][e] * u * g.df;
                    } else {
                        du = d[k][e] * act<true>(u, a.silu).df;
                    }
                    db[k][e] += du;
                    dw[k][e] = fmaf(du, n, dw[k][e]);
                    x[k][e] = n;
                    d[k][e] = du * w[k][e];
                    s1 += d[k][e];
                    s2 = fmaf(d[k][e], n, s2);
                }
                if (a.gate.p) store<IO, V, PAST>(a.dgate, (size_t)t * a.C + l.first + k * a.team * V, z[k]);
            }
        s1 = team_sum(s1, a.team) * inv;
        s2 = team_sum(s2, a.team) * inv;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (l.has(k, a.team)) {
#pragma unroll
                for (int e = 0; e < V; ++e) x[k][e] = rstd * (d[k][e] - s1 - x[k][e] * s2);
                store<IO, V, PAST>(a.dx, (size_t)t * a.C + l.first + k * a.team * V, x[k]);
            }
    }
    if (!a.part) return;
    float* p = a.part + (size_t)l.block * 2 * a.C;
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (l.has(k, a.team))
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const int c = l.first + k * a.team * V + e;
                p[c] = dw[k][e];
                p[a.C + c] = db[k][e];
            }
}

// The sum over a workgroup's threads, in each of them.
__device__ __forceinline__ float all_sum(float x, float* lds) {
    x = team_sum(x, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    return lds[0] + lds[1] + lds[2] + lds[3];
}

// Groups of any size, a workgroup for each: entries are read again for each pass.
template <int IO, bool BWD>
__global__ __launch_bounds__(256) void k_norm_large(NormArgs a) {
    using En = Entry<IO>;
    using T = typename En::T;
    __shared__ float lds[4];
    const int group = blockIdx.x % a.G, block = blockIdx.x / a.G, n = a.C / a.G, c0 = group * n;
    const float inv = 1.f / (float)n;
    float* pw = BWD && a.part ? a.part + (size_t)block * 2 * a.C + c0 : nullptr;
    float* pb = pw ? pw + a.C : nullptr;
    for (int t = block; t < a.T; t += a.blocks) {
        auto row = [&](const RowsIn& r) { return static_cast<const T*>(r.p) + (size_t)t * r.ld + c0; };
        auto out = [&](void* p) { return static_cast<T*>(p) + (size_t)t * a.C + c0; };
        const T* x = row(a.x);
        const T* g = a.gate.p ? row(a.gate) : nullptr;
        float sum = 0.f;
        for (int c = threadIdx.x; c < n; c += 256) sum += En::get(x[c]);
        const float mean = all_sum(sum, lds) * inv;
        sum = 0.f;
        for (int c = threadIdx.x; c < n; c += 256) {
            const float d = En::get(x[c]) - mean;
            sum = fmaf(d, d, sum);
        }
        const float rstd = 1.f / sqrtf(fmaf(all_sum(sum, lds), inv, a.eps));
        auto norm = [&](int c) { return (En::get(x[c]) - mean) * rstd; };
        auto weight = [&](int c) { return a.w ? a.w[c0 + c] : 1.f; };
        auto after = [&](int c) { return fmaf(norm(c), weight(c), a.b ? a.b[c0 + c] : 0.f); };
        if constexpr (!BWD) {
            T* y = out(a.y);
            for (int c = threadIdx.x; c < n; c += 256)
                y[c] = En::put(g ? after(c) * act<false>(En::get(g[c]), a.silu).f : act<false>(after(c), a.silu).f);
        } else {
            const T* dy = row(a.dy);
            auto slope = [&](int c) { return En::get(dy[c]) * (g ? act<false>(En::get(g[c]), a.silu).f : act<true>(after(c), a.silu).df); };
            float s1 = 0.f, s2 = 0.f;
            for (int c = threadIdx.x; c < n; c += 256) {
                const float du = slope(c), k = norm(c), dn = du * weight(c);
                s1 += dn;
                s2 = fmaf(dn, k, s2);
                if (pw) {
                    pw[c] = fmaf(du, k, t == block ? 0.f : pw[c]);
                    pb[c] = du + (t == block ? 0.f : pb[c]);
                }
                if (g) out(a.dgate)[c] = En::put(En::get(dy[c]) * after(c) * act<true>(En::get(g[c]), a.silu).df);
            }
            s1 = all_sum(s1, lds) * inv;
            s2 = all_sum(s2, lds) * inv;
            T* dx = out(a.dx);
            for (int c = threadIdx.x; c < n; c += 256) dx[c] = En::put(rstd * (slope(c) * weight(c) - s1 - norm(c) * s2));
        }
    }
}

// dw and db from the blocks' sums: 16 threads share a column's blocks, and add theirs up in one order.
__global__ __launch_bounds__(256) void k_norm_sum(const float* part, int blocks, int C, float* dw, float* db) {
    __shared__ float lds[16][17];
    const int c = blockIdx.x * 16 + (threadIdx.x & 15), k = threadIdx.x >> 4;  // columns of dw, then those of db
    float sum = 0.f;
    if (c < 2 * C) {
        for (int b = k; b < blocks; b += 16 * 8) {  // eight loads are under way at a time
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = b + e * 16 < blocks ? part[(size_t)(b + e * 16) * 2 * C + c] : 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += x[e];
        }
    }
    lds[k][threadIdx.x & 15] = sum;
    __syncthreads();
    if (k == 0 && c < 2 * C) {
        for (int r = 1; r < 16; ++r) sum += lds[r][threadIdx.x];
        float* to = c < C ? dw : db;
        if (to) to[c < C ? c : c - C] = sum;
    }
}

bool quick(const RowsIn& r, int V) { return !r.p || (reinterpret_cast<uintptr_t>(r.p) % 16 == 0 && r.ld % V == 0); }
bool quick(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

struct Shape {
    int vec;   // entries of a vector: 16 bytes of them, or 1
    int num;   // vectors a lane, 1, 2, 4 or 8; 0: the group does not fit a wave
    int team;
};
Shape shape(const NormArgs& a) {
    const int c = a.C / a.G, v = a.io == kRowBf16 ? 8 : 4;
    Shape s;
    s.vec = c % v == 0 && a.C % v == 0 && quick(a.x, v) && quick(a.gate, v) && quick(a.dy, v) && quick(a.y) && quick(a.dx) && quick(a.dgate) ? v : 1;
    const int n = (c + s.vec - 1) / s.vec;
    for (s.team = 1; s.team < 64 && s.team < n; s.team *= 2) {}
    const int num = (n + s.team - 1) / s.team;
    s.num = num <= 1 ? 1 : num <= 2 ? 2 : num <= 4 ? 4 : num <= 8 ? 8 : 0;
    return s;
}

// Blocks of rows, each of which is one wave's for some of the groups.  Enough waves to fill the
// card; backward four rows or more in a block, whose sums take as much room as four bf16 rows.
int row_blocks(int T, int C, bool bwd) {
    const int waves = (C + 511) / 512;
    int most = std::max(kBlocks, kNormWaves / waves);
    if (bwd) most = std::min(most, std::max(64, (1 << 23) / C));  // the sums of very wide rows: 64 MB, or 64 blocks
    return std::min(bwd ? (T + 3) / 4 : T, most);
}

}  // namespace

size_t norm_workspace(int T, int C) { return ((size_t)row_blocks(T, C, true) * 2 * C * 4 + 255) / 256 * 256; }

bool norm_fits(int T, int C, int G) { return (int64_t)row_blocks(T, C, false) * G < (1 << 24); }

namespace {

template <int IO, int V, bool PAST>
void (*pick(int num, bool bwd))(NormArgs) {
    switch (num) {
        case 1: return bwd ? k_norm_bwd<IO, V, 1, PAST> : k_norm_fwd<IO, V, 1, PAST>;
        case 2: return bwd ? k_norm_bwd<IO, V, 2, PAST> : k_norm_fwd<IO, V, 2, PAST>;
        case 4: return bwd ? k_norm_bwd<IO, V, 4, PAST> : k_norm_fwd<IO, V, 4, PAST>;
        default: return bwd ? k_norm_bwd<IO, V, 8, PAST> : k_norm_fwd<IO, V, 8, PAST>;
    }
}

hipError_t rows(NormArgs& a, bool bwd, hipStream_t s) {
    const Shape sh = shape(a);
    const bool b = a.io == kRowBf16;
    a.team = sh.team;
    a.blocks = row_blocks(a.T, a.C, bwd);
    if (a.T == 0) return hipSuccess;
    void (*f)(NormArgs);
    unsigned grid;
    if (sh.num) {
        const int size = b ? 2 : 4, wave = 64 / sh.team * (a.C / a.G) * size;
        const bool past = (int64_t)a.T * a.C * size >= kPast && a.C * size % kPiece == 0 && wave % kPiece == 0;
        if (sh.vec == 1) f = b ? pick<kRowBf16, 1, false>(sh.num, bwd) : pick<kRowF32, 1, false>(sh.num, bwd);
        else if (past) f = b ? pick<kRowBf16, 8, true>(sh.num, bwd) : pick<kRowF32, 4, true>(sh.num, bwd);
        else f = b ? pick<kRowBf16, 8, false>(sh.num, bwd) : pick<kRowF32, 4, false>(sh.num, bwd);
        const int per = 64 / sh.team, sets = (a.G + per - 1) / per;
        grid = (unsigned)(((int64_t)sets * a.blocks + 3) / 4);
    } else {
        f = bwd ? (b ? k_norm_large<kRowBf16, true> : k_norm_large<kRowF32, true>)
                : (b ? k_norm_large<kRowBf16, false> : k_norm_large<kRowF32, false>);
        grid = (unsigned)a.G * a.blocks;
    }
    hipLaunchKernelGGL(f, dim3(grid), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_fwd(NormArgs a, hipStream_t s) { return rows(a, false, s); }

hipError_t launch_norm_bwd(NormArgs a, hipStream_t s) {
    if (!a.dw && !a.db) a.part = nullptr;
    const hipError_t e = rows(a, true, s);
    if (e != hipSuccess || (!a.dw && !a.db)) return e;
    hipLaunchKernelGGL(k_norm_sum, dim3((2 * a.C + 15) / 16), dim3(256), 0, s, a.part, a.blocks, a.C, a.dw, a.db);
    return hipGetLastError();
}

}  // namespace pdssm

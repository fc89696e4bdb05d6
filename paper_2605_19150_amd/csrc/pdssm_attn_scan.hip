// pdssm_attn_scan.hip -- the scan of linear attention with a decay for each
// head, forward and in reverse, for rows of up to DC entries (PDSSM_DC).
//
// With a = exp(-rate) and S_t = a S_{t-1} + k_t v_t^T, a chunk of n rows that
// begins with the state S has, i and j counted from its first row,
//
//   out_i = sa (sum_{j<=i} a^(i-j) (q_i . k_j) v_j + a^(i+1) S^T q_i)
//   S'    = a^n S + sum_j a^(n-1-j) k_j v_j^T,
//
// four matrix products.  A workgroup of four waves takes the chunks of a segment
// of a sequence one after the other, for one head; a wave owns 16 NT columns of v
// and holds these columns of the state in its accumulators, so q, k, v are read
// once and out is written once, and no state goes through memory.  The registers
// hold S with its columns across the lanes and four rows a lane: what an operand of
// S^T q has to be, when q is read in the same order.  Weighted by powers of a are v
// (for S') and results; where a product's operand has more bits than bf16 (S, the
// weighted v, the weighted scores) it is taken as the sum of two bf16 numbers, off
// by 2^-17 at most.  fp32 rows go through the fp32 matrix instructions.
//
// A chunk that holds a NaN or an infinity would give it to rows before it (0 times
// infinity): from there on the segment is computed row by row.
#include <math.h>

#include "pdssm_attn.h"
#include "pdssm_rows.h"

namespace pdssm {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int kWaves = 4;

// Operands of a matrix instruction over 16 x 16 results.  Lane l has row (or
// column) l % 16 and, of each 16 places of the summed axis, the four from 4 (l / 16) on.
template <int IO>
struct Mat;
template <>
struct Mat<kRowBf16> {
    using T = uint16_t;
    using Frag = bf16x8;                // two times 16 places
    static constexpr int kDepth = 32;
    static constexpr int kChunk = 64;   // rows of a chunk
    static constexpr bool kSplit = true;
    // p: the lane's four entries of a row in LDS, the other 16 places on
    static __device__ __forceinline__ Frag row(const T* p) {
        const u32x2 lo = *reinterpret_cast<const u32x2*>(p), hi = *reinterpret_cast<const u32x2*>(p + 16);
        return __builtin_bit_cast(Frag, u32x4{lo.x, lo.y, hi.x, hi.y});
    }
    // the same of columns: 16 lanes hand each other the four entries of their four rows
    static __device__ __forceinline__ Frag col(const T* tile, int pitch, int lane) {
        const T* p = tile + ((lane >> 4) * 4 + ((lane & 15) >> 2)) * pitch + (lane & 3) * 4;
        union {
            s16x4 h[2];
            Frag f;
        } u;
        u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
        u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 16 * pitch));
        return u.f;
    }
    static __device__ __forceinline__ f32x4 mul(Frag a, Frag b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ float get(Frag f, int e) { return (float)f[e]; }
};
template <>
struct Mat<kRowF32> {
    using T = float;
    using Frag = f32x4;
    static constexpr int kDepth = 16;
    static constexpr int kChunk = 32;
    static constexpr bool kSplit = false;
    static __device__ __forceinline__ Frag row(const T* p) { return *reinterpret_cast<const Frag*>(p); }
    static __device__ __forceinline__ Frag col(const T* tile, int pitch, int lane) {
        const T* p = tile + (lane >> 4) * 4 * pitch + (lane & 15);
        return Frag{p[0], p[pitch], p[2 * pitch], p[3 * pitch]};
    }
    static __device__ __forceinline__ f32x4 mul(Frag a, Frag b, f32x4 c) {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
    static __device__ __forceinline__ float get(Frag f, int e) { return f[e]; }
};

// 16 bytes of a row: those behind the row's n entries are zero.  quick: the row
// is 16-byte aligned and n a multiple of what 16 bytes hold.
template <int IO>
__device__ __forceinline__ u32x4 load16(const typename Mat<IO>::T* row, int c, int n, bool quick) {
    using T = typename Mat<IO>::T;
    constexpr int V = 16 / sizeof(T);
    u32x4 x = {};
    if (quick) {
        if (c < n) x = *reinterpret_cast<const u32x4*>(row + c);
    } else {
        union {
            T v[V];
            u32x4 x;
        } u;
#pragma unroll
        for (int e = 0; e < V; ++e) u.v[e] = c + e < n ? row[c + e] : T(0);
        x = u.x;
    }
    return x;
}

// Not zero if one of the entries is an infinity or a NaN.
template <int IO>
__device__ __forceinline__ uint32_t wild(u32x4 x) {
    uint32_t r = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        r |= IO == kRowBf16 ? ((x[e] & 0x7f807f80u) + 0x00800080u) & 0x80008000u : ((x[e] & 0x7f800000u) + 0x00800000u) & 0x80000000u;
    return r;
}

// The rows of a chunk on their way to LDS, which a thread has in registers.
template <int IO, int W>  // W entries of a row, with those that fill it up
struct Stage {
    using T = typename Mat<IO>::T;
    static constexpr int C = Mat<IO>::kChunk, V = 16 / sizeof(T), N = C * W / V, U = (N + 255) / 256;
    u32x4 x[U];
    // rows first, first + step, ..: n of them, entries c0 .. of rows of `wide` ones
    __device__ __forceinline__ void load(const T* p, int64_t ld, int64_t first, int step, int n, int c0, int wide, bool quick) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = threadIdx.x + u * 256, r = k / (W / V), c = c0 + k % (W / V) * V;
            x[u] = u32x4{};
            if (r < n) x[u] = load16<IO>(p + (first + (int64_t)r * step) * ld, c, wide, quick);
        }
    }
    __device__ __forceinline__ uint32_t store(T* tile, int pitch) {
        uint32_t bad = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = threadIdx.x + u * 256, r = k / (W / V), c = k % (W / V) * V;
            bad |= wild<IO>(x[u]);
            if (N % 256 == 0 || k < N) *reinterpret_cast<u32x4*>(tile + r * pitch + c) = x[u];
        }
        return bad;
    }
};

// x as the sum of two numbers of the operands' type.
template <int IO>
__device__ __forceinline__ void split(const float* x, typename Mat<IO>::Frag& hi, typename Mat<IO>::Frag& lo) {
    if constexpr (Mat<IO>::kSplit) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            hi[e] = (__bf16)x[e];
            lo[e] = (__bf16)(x[e] - (float)hi[e]);
        }
    } else {
        hi = typename Mat<IO>::Frag{x[0], x[1], x[2], x[3]};
        lo = hi;
    }
}

template <int IO>
__device__ __forceinline__ bool quick_rows(const HeadsIn& r, int n) {
    constexpr int V = 16 / sizeof(typename Mat<IO>::T);
    return ((reinterpret_cast<uintptr_t>(r.p) | 0) % 16 == 0) && r.ld % V == 0 && r.hs % V == 0 && n % V == 0;
}

// DC: entries of q and k rows, filled up; NT: 16-column blocks of v that a wave owns.
template <int IO, int DC, int NT, bool FULL>
__global__ __launch_bounds__(256, DC > 128 ? 1 : 2) void k_attn_scan(AttnScan a) {
    using M = Mat<IO>;
    using T = typename M::T;
    using Frag = typename M::Frag;
    constexpr int C = M::kChunk, KB = M::kDepth, W = kWaves * NT * 16, PAD = 16 / sizeof(T);
    constexpr int PK = DC + PAD, PV = W + PAD, PA = C + PAD, NI = C / 16, ND = DC / 16, E = KB / 4;
    __shared__ __align__(16) T ks[C * PK];
    __shared__ __align__(16) T vs[C * PV];
    __shared__ __align__(16) T qs[FULL ? C * PK : 8];
    __shared__ __align__(16) T as[FULL ? (M::kSplit ? 2 : 1) * C * PA : 8];  // weighted scores, and what bf16 leaves of them
    __shared__ float pw[C + 2];      // powers of a
    __shared__ float wu[2 * C + 4];  // weights of a chunk's rows in the state behind it, zeros behind them
    __shared__ int bad;

    // the workgroups of one segment of a head are neighbours on one of the 8 XCDs,
    // so that rows which several of them read come from its L2
    const int xcd = blockIdx.x & 7, y = blockIdx.x >> 3;
    const int64_t group = (int64_t)(y / a.members) * 8 + xcd;
    if (group >= a.groups) return;
    int member = y % a.members;
    int ri = 0;
    while (ri + 1 < a.roles && member >= a.role[ri].slices) member -= a.role[ri++].slices;
    const AttnRole& R = a.role[ri];
    const int item = (int)(group / a.H), h = (int)(group % a.H), col0 = member * W;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, lr = lane & 15;

    // The segment: sequence s has the items from cu[s] / seg_rows + s on, more than it can need.
    int s, seg;
    int64_t begin, end, slot;
    if (a.cu) {
        int lo = 0, n = a.S;
        while (n > 1) {  // the last sequence that begins at or before this item
            const int step = (n + 255) / 256, at = lo + tid * step;
            const bool in = tid * step < n && (int64_t)(min(max(a.cu[at], 0), a.T) / a.seg_rows) + at <= item;
            const int k = max(__syncthreads_count(in) - 1, 0);
            n = min(step, n - k * step);
            lo += k * step;
        }
        s = lo;
        begin = min(max(a.cu[s], 0), a.T);
        end = min(max(a.cu[s + 1], (int)begin), a.T);
        seg = max(item - (int)(begin / a.seg_rows) - s, 0);
        // rows behind the last sequence come back as zeros
        if constexpr (FULL) {
            const int64_t rest = min(max(a.cu[a.S], 0), a.T), wide = (int64_t)a.H * R.Do;
            const int64_t n = (a.T - rest) * wide, share = (n + a.items * (int64_t)a.H - 1) / (a.items * (int64_t)a.H);
            if (member == 0 && n > 0 && !R.out32)
                for (int64_t e = group * share + tid; e < min((group + 1) * share, n); e += 256)
                    static_cast<T*>(R.out)[rest * wide + e] = T(0);
        }
    } else {
        const int per = max((a.L + a.seg_rows - 1) / a.seg_rows, 1);
        s = item / per;
        seg = item % per;
        begin = (int64_t)s * a.L;
        end = begin + a.L;
    }
    slot = begin / a.seg_rows + seg;
    const int64_t len = end - begin, p0 = (int64_t)seg * a.seg_rows;
    const size_t at_seq = ((size_t)s * a.H + h) * a.state;
    if (p0 >= len) {
        if (FULL && len == 0 && seg == 0 && R.fin)  // a sequence without rows hands its state on
            for (int e = tid; e < R.Dc * W; e += 256) {
                const int c = e / W, o = col0 + e % W;
                const size_t i = at_seq + (size_t)c * R.rs + (size_t)o * R.cs;
                if (o < R.Do) R.fin[i] = R.keep ? R.keep[i] : 0.f;
            }
        return;
    }
    const bool last_seg = p0 + a.seg_rows >= len;
    if (!FULL && last_seg) return;
    const int rows = (int)(min(len, p0 + a.seg_rows) - p0);

    const int late = R.late;
    const float s_in = late ? 1.f : a.scale, s_up = late ? a.scale : 1.f;
    const float rate = a.rate[h];
    const bool fine = rate >= 0.f && rate < INFINITY;
    for (int d = tid; d < C + 2; d += 256) pw[d] = fine ? (float)exp(-(double)rate * d) : NAN;
    for (int j = tid; j < 2 * C + 4; j += 256) wu[j] = j < C ? (fine ? s_up * (float)exp(-(double)rate * (C - 1 - j + late)) : NAN) : 0.f;
    if (tid == 0) bad = 0;
    if constexpr (FULL)  // the scores of later rows stay zero
        for (int e = tid; e < (M::kSplit ? 2 : 1) * C * PA; e += 256) as[e] = T(0);

    const T* qp = static_cast<const T*>(R.q.p) + (int64_t)(h / R.q.share) * R.q.hs;
    const T* kp = static_cast<const T*>(R.k.p) + (int64_t)(h / R.k.share) * R.k.hs;
    const T* vp = static_cast<const T*>(R.v.p) + (int64_t)(h / R.v.share) * R.v.hs;
    const bool qq = quick_rows<IO>(R.q, R.Dc), kq = quick_rows<IO>(R.k, R.Dc), vq = quick_rows<IO>(R.v, R.Do);
    const int step = late ? -1 : 1;
    const int64_t first = late ? end - 1 - p0 : begin + p0;  // row of position p: first + step * p
    const bool o_quick = R.Do % 4 == 0 && reinterpret_cast<uintptr_t>(R.out) % 16 == 0;

    Stage<IO, DC> sq, sk;
    Stage<IO, W> sv;
    auto load = [&](int p) {
        const int n = min(C, rows - p);
        const int64_t r = first + (int64_t)step * p;
        if constexpr (FULL) sq.load(qp, R.q.ld, r, step, n, 0, R.Dc, qq);
        sk.load(kp, R.k.ld, r, step, n, 0, R.Dc, kq);
        sv.load(vp, R.v.ld, r, step, n, col0, R.Do, vq);
    };
    load(0);

    // the state: rows 16 d + 4 g + r, column lr of the wave's block t
    const int wc = wave * NT * 16;
    f32x4 S[ND][NT];
    const float* x = nullptr;
    if (FULL && seg > 0) x = R.seg + ((size_t)slot * a.H + h) * a.state;
    else if (FULL && R.x0) x = R.x0 + at_seq;
    bool sick = false;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int c = d * 16 + g * 4 + r, o = col0 + wc + t * 16 + lr;
                float e = 0.f;
                if (FULL && x && c < R.Dc && o < R.Do) e = x[(size_t)c * R.rs + (size_t)o * R.cs];
                sick |= !(fabsf(e) < INFINITY);
                S[d][t][r] = e;
            }
    __syncthreads();
    if (sick) bad = 1;

    auto out_at = [&](int p, int t) -> int64_t {  // entry of out of position p, column 4 g of block t
        return ((first + (int64_t)step * p) * a.H + h) * R.Do + col0 + wc + t * 16;
    };

    for (int p = 0; p < rows; p += C) {
        const int n = min(C, rows - p);
        uint32_t w = sk.store(ks, PK) | sv.store(vs, PV);
        if constexpr (FULL) w |= sq.store(qs, PK);
        if (w) bad = 1;
        __syncthreads();
        const bool slow = bad;
        if (p + C < rows) load(p + C);
        if (!slow) {
            if constexpr (FULL) {
                f32x4 acc[NI][NT] = {};
                // S^T q
#pragma unroll
                for (int kb = 0; kb < DC / KB; ++kb) {
                    Frag hi[NT], lo[NT];
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        float e[8];
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            e[r] = S[kb * (KB / 16)][t][r];
                            e[4 + r] = S[kb * (KB / 16) + KB / 16 - 1][t][r];
                        }
                        split<IO>(e, hi[t], lo[t]);
                    }
#pragma unroll
                    for (int i = 0; i < NI; ++i) {
                        const Frag f = M::row(qs + (i * 16 + lr) * PK + kb * KB + g * 4);
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            acc[i][t] = M::mul(hi[t], f, acc[i][t]);
                            if constexpr (M::kSplit) acc[i][t] = M::mul(lo[t], f, acc[i][t]);
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    const float f = s_in * pw[i * 16 + lr + 1 - late];
#pragma unroll
                    for (int t = 0; t < NT; ++t) acc[i][t] *= f;
                }
                // the scores at and below the diagonal, 16 x 16 of them at a time
                for (int b = wave; b < NI * (NI + 1) / 2; b += kWaves) {
                    int i = 0, j = b;
                    while (j > i) j -= ++i;
                    f32x4 sc = {};
#pragma unroll
                    for (int kb = 0; kb < DC / KB; ++kb)
                        sc = M::mul(M::row(ks + (j * 16 + lr) * PK + kb * KB + g * 4), M::row(qs + (i * 16 + lr) * PK + kb * KB + g * 4), sc);
                    float e[8] = {};
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int d = (i - j) * 16 + lr - g * 4 - r;
                        e[r] = d >= 0 ? sc[r] * a.scale * pw[max(d, 0)] : 0.f;
                    }
                    Frag hi, lo;
                    split<IO>(e, hi, lo);
                    T* to = as + (i * 16 + lr) * PA + j * 16 + g * 4;
                    if constexpr (M::kSplit) {
                        const u32x4 uh = __builtin_bit_cast(u32x4, hi), ul = __builtin_bit_cast(u32x4, lo);
                        *reinterpret_cast<u32x2*>(to) = u32x2{uh.x, uh.y};
                        *reinterpret_cast<u32x2*>(to + C * PA) = u32x2{ul.x, ul.y};
                    } else {
                        *reinterpret_cast<Frag*>(to) = hi;
                    }
                }
                __syncthreads();
#pragma unroll
                for (int kb = 0; kb < C / KB; ++kb) {
                    Frag vf[NT];
#pragma unroll
                    for (int t = 0; t < NT; ++t) vf[t] = M::col(vs + kb * KB * PV + wc + t * 16, PV, lane);
#pragma unroll
                    for (int i = kb * KB / 16; i < NI; ++i) {
                        const T* from = as + (i * 16 + lr) * PA + kb * KB + g * 4;
                        const Frag hi = M::row(from);
#pragma unroll
                        for (int t = 0; t < NT; ++t) acc[i][t] = M::mul(vf[t], hi, acc[i][t]);
                        if constexpr (M::kSplit) {
                            const Frag lo = M::row(from + C * PA);
#pragma unroll
                            for (int t = 0; t < NT; ++t) acc[i][t] = M::mul(vf[t], lo, acc[i][t]);
                        }
                    }
                }
                // lane: row i * 16 + lr, columns 4 g .. 4 g + 3
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    const int r = i * 16 + lr;
                    if (r >= n) continue;
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const int c = col0 + wc + t * 16 + g * 4;
                        const int64_t at = out_at(p + r, t) + g * 4;
                        if (R.out32 || IO == kRowF32) {
                            float* to = static_cast<float*>(R.out) + at;
                            if (o_quick) {
                                if (c < R.Do) *reinterpret_cast<f32x4*>(to) = acc[i][t];
                            } else {
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if (c + e < R.Do) to[e] = acc[i][t][e];
                            }
                        } else {
                            uint16_t* to = static_cast<uint16_t*>(R.out) + at;
                            uint32_t v[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) v[e] = Entry<kRowBf16>::put(acc[i][t][e]);
                            if (o_quick) {
                                if (c < R.Do) *reinterpret_cast<u32x2*>(to) = u32x2{v[0] | v[1] << 16, v[2] | v[3] << 16};
                            } else {
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if (c + e < R.Do) to[e] = (uint16_t)v[e];
                            }
                        }
                    }
                }
            }
            // the state behind the chunk
            const float keep = pw[n];
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int t = 0; t < NT; ++t) S[d][t] *= keep;
#pragma unroll
            for (int kb = 0; kb < C / KB; ++kb) {
                Frag hi[NT], lo[NT];
                const float* u = wu + kb * KB + g * 4 + C - n;
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const Frag vf = M::col(vs + kb * KB * PV + wc + t * 16, PV, lane);
                    float e[8];
#pragma unroll
                    for (int r = 0; r < E; ++r) e[r] = M::get(vf, r) * u[r + (r >= 4 ? 12 : 0)];
                    split<IO>(e, hi[t], lo[t]);
                }
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    const Frag kf = M::col(ks + kb * KB * PK + d * 16, PK, lane);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        S[d][t] = M::mul(kf, hi[t], S[d][t]);
                        if constexpr (M::kSplit) S[d][t] = M::mul(kf, lo[t], S[d][t]);
                    }
                }
            }
        } else {
            // row by row, as the recurrence is written
            const float decay = pw[1];
            for (int r = 0; r < n; ++r) {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const float v = s_up * Entry<IO>::get(vs[r * PV + wc + t * 16 + lr]);
                    float o = 0.f;
#pragma unroll
                    for (int d = 0; d < ND; ++d)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int c = d * 16 + g * 4 + e;
                            if (c >= R.Dc) continue;
                            if (!late) S[d][t][e] *= decay;
                            S[d][t][e] = fmaf(Entry<IO>::get(ks[r * PK + c]), v, S[d][t][e]);
                            if constexpr (FULL) o = fmaf(Entry<IO>::get(qs[r * PK + c]), S[d][t][e], o);
                            if (late) S[d][t][e] *= decay;
                        }
                    if constexpr (FULL) {
                        o += __shfl_xor(o, 16);
                        o += __shfl_xor(o, 32);
                        o *= s_in * pw[0];
                        const int64_t at = out_at(p + r, t) + lr;
                        if (g == 0 && col0 + wc + t * 16 + lr < R.Do) {
                            if (R.out32 || IO == kRowF32) static_cast<float*>(R.out)[at] = o;
                            else static_cast<uint16_t*>(R.out)[at] = Entry<kRowBf16>::put(o);
                        }
                    }
                }
            }
        }
        __syncthreads();
    }

    float* to = nullptr;
    if (!FULL) to = const_cast<float*>(R.seg) + ((size_t)(slot + 1) * a.H + h) * a.state;
    else if (last_seg && R.fin) to = R.fin + at_seq;
    if (to) {
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int c = d * 16 + g * 4 + r, o = col0 + wc + t * 16 + lr;
                    if (c < R.Dc && o < R.Do) to[(size_t)c * R.rs + (size_t)o * R.cs] = S[d][t][r];
                }
    }
}

}  // namespace

template <int DC>
hipError_t launch_attn_scan(const AttnScan& a, bool full, bool wide, hipStream_t s) {
    const int64_t n = (a.groups + 7) / 8 * 8 * a.members;
    const bool b = a.io == kRowBf16;
    void (*f)(AttnScan) = nullptr;
    // NT = 2 needs more registers than there are for rows past 128 entries
    constexpr int N2 = DC > 128 ? 1 : 2;
    if (full) {
        if (wide) f = b ? k_attn_scan<kRowBf16, DC, N2, true> : k_attn_scan<kRowF32, DC, N2, true>;
        else f = b ? k_attn_scan<kRowBf16, DC, 1, true> : k_attn_scan<kRowF32, DC, 1, true>;
    } else {
        if (wide) f = b ? k_attn_scan<kRowBf16, DC, N2, false> : k_attn_scan<kRowF32, DC, N2, false>;
        else f = b ? k_attn_scan<kRowBf16, DC, 1, false> : k_attn_scan<kRowF32, DC, 1, false>;
    }
    hipLaunchKernelGGL(f, dim3((unsigned)n), dim3(256), 0, s, a);
    return hipGetLastError();
}
template hipError_t launch_attn_scan<PDSSM_DC>(const AttnScan&, bool, bool, hipStream_t);

}  // namespace pdssm

// pdssm_attn_scan.hip -- the scan of linear attention with a decay for each
// head, forward and in reverse, for rows of up to DC entries (PDSSM_DC).
//
// With a = exp(-rate) and S_t = a S_{t-1} + k_t v_t^T, a chunk of n rows that
// begins with the state S has, i and j counted from its first row,
//
//   out_i = sa (sum_{j<=i} a^(i-j) (q_i . k_j) v_j + a^(i+1) S^T q_i)
//   S'    = a^n S + sum_j a^(n-1-j) k_j v_j^T,
//
// four matrix products.  A workgroup takes the chunks of a segment of a sequence one
// after the other, for one head; a wave owns 16 NT columns of v
// and holds these columns of the state in its accumulators, so q, k, v are read
// once and out is written once, and no state goes through memory.  The registers
// hold S with its columns across the lanes and four rows a lane: what an operand of
// S^T q has to be, when q is read in the same order.  Weighted by powers of a are v
// (for S') and results; where a product's operand has more bits than bf16 (S, the
// weighted v, the weighted scores) it is taken as the sum of two or three bf16 numbers.
// fp32 rows go through the fp32 matrix instructions.
//
// In reverse rows stand in LDS as they do in memory; scores above the diagonal
// count, and the two tables of weights change places.
//
// A chunk that holds a NaN or an infinity would give it to rows before it (0 times
// infinity): from there on the segment is computed row by row.
#include <math.h>

#include <algorithm>

#include "pdssm_attn.h"
#include "pdssm_device.h"
#include "pdssm_rows.h"

namespace pdssm {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// With bf16 rows, the bf16 numbers whose sum an operand of more bits is taken as.  The state where a row reads it and
// weighted scores: kTerms, off by 2^-16 of themselves, so that a row output is off by its own rounding alone, also where
// k or v stands ten deviations off centre and what it is multiplied by has no constant part.  With one number
// rows were 1.4 times as far off, and 9 times in that case, for 8 to 14 % less time (684 us in place of 800 backward
// at 8 x 4096 rows of 32 heads of 128, 89 in place of 97 forward at 16 x 2048 of 16 of 64).
// Weighted rows that go into a state: kRow, the 24 bits of what a sum in fp32 holds (with two a state is 2.4e-6 off in
// place of 1e-7 to 3e-7), or kInner in the scans of dq and dk, whose states rows alone are made of, by way of
// kTerms numbers (with three 837 us in place of 800).
constexpr int kTerms = 2, kRow = 3, kInner = 2;

// A tile of rows in LDS.  Its pitch is 8 banks past a multiple of 32 (bf16), and of
// rows 8 to 15 of each 16 the 16-byte pieces change places in pairs, so that 16 lanes with
// a row each do not meet in a bank.  Reads of columns do: 32 lanes have four entries of rows 0 to 3 and of rows 8 to 11,
// which begin in the same bank, two lanes a bank.  Such conflicts are two fifths of the cycles that LDS is
// active in (the counters of the backward and forward at heads of 64 and 128).
template <int IO>
struct Tile;
template <>
struct Tile<kRowBf16> {
    static constexpr int kPad = 16;
    static __device__ __forceinline__ int col(int row, int c) { return c ^ (row & 8); }
};
template <>
struct Tile<kRowF32> {
    static constexpr int kPad = 4;
    static __device__ __forceinline__ int col(int, int c) { return c; }
};

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
    // where a lane begins to read columns of eight neighbouring rows, and the read: 16 lanes hand each other the
    // four entries of their four rows
    static __device__ __forceinline__ int col_at(int lane, int pitch) {
        const int r = (lane >> 4) * 8 + ((lane & 15) >> 2);
        return r * pitch + Tile<kRowBf16>::col(r, (lane & 3) * 4);
    }
    static __device__ __forceinline__ Frag col(const T* p, int pitch) {
        union {
            s16x4 h[2];
            Frag f;
        } u;
        u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
        u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * pitch));
        return u.f;
    }
    // 16 bytes of a row: eight neighbours of the summed axis, where both operands are read so
    static constexpr int kNear = 8;
    static __device__ __forceinline__ Frag near(const T* p) { return *reinterpret_cast<const Frag*>(p); }
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
    static __device__ __forceinline__ int col_at(int lane, int pitch) { return (lane >> 4) * 4 * pitch + (lane & 15); }
    static __device__ __forceinline__ Frag col(const T* p, int pitch) { return Frag{p[0], p[pitch], p[2 * pitch], p[3 * pitch]}; }
    static constexpr int kNear = 4;
    static __device__ __forceinline__ Frag near(const T* p) { return *reinterpret_cast<const Frag*>(p); }
    static __device__ __forceinline__ f32x4 mul(Frag a, Frag b, f32x4 c) {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
    static __device__ __forceinline__ float get(Frag f, int e) { return f[e]; }
};

// The hardware does not hold back a reader of a matrix instruction's result: the compiler has to keep up to ten wait
// states between them.  Where the paths between them join behind a short branch it counts along one path only and
// may leave too few (scores of fp32 rows past 128 entries lost their last product that way).  So no branch stands behind
// the scores, and the ten states stand here behind products that a later block reads.
__device__ __forceinline__ void settle() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 9");
    __builtin_amdgcn_sched_barrier(0);
}

// Whether one of a wave's entries is an infinity or a NaN.
template <int IO>
struct Wild;
template <>
struct Wild<kRowBf16> {
    f32x4 sum = {};  // of the entries times zero: NaN then.  On the matrix cores, which have time; by their bits 8 operations more for each 16 bytes
    __device__ __forceinline__ void add(u32x4 x) {
        sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), bf16x8{}, sum, 0, 0, 0);
    }
    __device__ __forceinline__ bool any() const { return !(sum.x + sum.y + sum.z + sum.w == 0.f); }
};
template <>
struct Wild<kRowF32> {
    uint32_t top = 0;
    __device__ __forceinline__ void add(u32x4 x) {
#pragma unroll
        for (int e = 0; e < 4; ++e) top = max(top, x[e] & 0x7fffffffu);
    }
    __device__ __forceinline__ bool any() const { return top >= 0x7f800000u; }
};

// Cache policy of stores past the caches, which a large out would only sweep (176 -> 168 us backward at B16 L2048,
// 16 heads of 64; for pieces of 32 bytes, an accumulator's, it is ruinous).
constexpr int kPastCaches = 2;
constexpr uint32_t kOutside = 0x80000000u;  // an offset past every chunk: loads of zeros, stores that are dropped

// The rows of a chunk on their way to LDS, which a thread has in registers.
template <int IO, int W, int NTH>  // W entries of a row, with those that fill it up; NTH threads
struct Stage {
    using T = typename Mat<IO>::T;
    static constexpr int C = Mat<IO>::kChunk, V = 16 / sizeof(T), P = W + Tile<IO>::kPad;
    static constexpr int kRows = NTH * V / W;  // rows between a thread's vectors
    static constexpr int U = C / kRows;
    static_assert(NTH * V % W == 0 && C % kRows == 0, "whole rows a thread");
    u32x4 x[U];
    uint32_t voff;  // of the first vector from the chunk's first row on
    int row, c;
    // entries c0 .. of rows of `wide` ones
    __device__ __forceinline__ Stage(int ld, int c0, int wide) : row(threadIdx.x / (W / V)), c(c0 + threadIdx.x % (W / V) * V) {
        voff = c < wide ? ((uint32_t)row * ld + c) * (uint32_t)sizeof(T) : kOutside;
    }
    // n rows from `low` on, those behind them and entries behind a row's end as zeros.  BY: bytes of a
    // load, 16 if rows are aligned to them and `wide` fills whole ones.  Nothing branches, so the
    // loads are all under way at once (those of 2 bytes are waited for here: they would need too many registers).
    template <int BY>
    __device__ __forceinline__ void load(const T* low, int ld, int n, int wide) {
        const __amdgpu_buffer_rsrc_t rsrc = row_block(low, (uint32_t)((int64_t)(n - 1) * ld + wide) * (uint32_t)sizeof(T));
        const uint32_t step = (uint32_t)(kRows * ld) * (uint32_t)sizeof(T);
        if (BY == 16 && n == C) {
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, voff, u * step, 0);
            return;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t at = row + u * kRows < n && voff < kOutside ? voff + u * step : kOutside;
            if constexpr (BY == 16) {
                x[u] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, 0, 0);
            } else if constexpr (BY == 4) {
                constexpr int E = 4 / sizeof(T);  // entries of a load: all in the row, or none
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    x[u][e] = __builtin_amdgcn_raw_buffer_load_b32(rsrc, c + e * E < wide ? at + e * 4 : kOutside, 0, 0);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t lo = __builtin_amdgcn_raw_buffer_load_b16(rsrc, c + 2 * e < wide ? at + e * 4 : kOutside, 0, 0);
                    const uint32_t hi = __builtin_amdgcn_raw_buffer_load_b16(rsrc, c + 2 * e + 1 < wide ? at + e * 4 + 2 : kOutside, 0, 0);
                    x[u][e] = lo | hi << 16;
                }
            }
        }
    }
    // where u-th 16 bytes are in a tile
    __device__ __forceinline__ int at(int u, int c0) const {
        const int r = row + u * kRows;
        return r * P + Tile<IO>::col(r, c - c0);
    }
    __device__ __forceinline__ void store(T* tile, int c0, Wild<IO>& top) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            top.add(x[u]);
            *reinterpret_cast<u32x4*>(tile + at(u, c0)) = x[u];
        }
    }
};

// Two bf16 numbers, to nearest even, the first in the low half.
__device__ __forceinline__ uint32_t pair(float x, float y) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){x, y}, bf16x2));
}

// x as the sum of N numbers of the operands' type.
template <int IO, int N>
__device__ __forceinline__ void split(const float* x, typename Mat<IO>::Frag (&f)[N]) {
    if constexpr (Mat<IO>::kSplit) {
        u32x4 to[N];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f32x2 rest = {x[2 * e], x[2 * e + 1]};
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const uint32_t u = pair(rest.x, rest.y);
                to[n][e] = u;
                rest.x -= __uint_as_float(u << 16);
                rest.y -= __uint_as_float(u & 0xffff0000u);
            }
        }
#pragma unroll
        for (int n = 0; n < N; ++n) f[n] = __builtin_bit_cast(typename Mat<IO>::Frag, to[n]);
    } else {
        f[0] = typename Mat<IO>::Frag{x[0], x[1], x[2], x[3]};
    }
}

template <int IO, int DC, int W, bool FULL>
struct Shared {
    using T = typename Mat<IO>::T;
    static constexpr int C = Mat<IO>::kChunk, PK = DC + Tile<IO>::kPad, PV = W + Tile<IO>::kPad, PA = C + 16 / sizeof(T);
    static constexpr int NA = Mat<IO>::kSplit ? kTerms : 1;
    alignas(16) T ks[C * PK];
    alignas(16) T vs[C * PV];
    alignas(16) T qs[FULL ? C * PK : 8];
    alignas(16) T as[FULL ? NA * C * PA : 8];  // weighted scores, in their terms
    // weights of a chunk's rows: a^(r+1), and from C - n on a^(n-1-r) with zeros behind it; the ones of
    // the state in out, and of rows in the state (late: the other way round); and powers of a
    float up[C], down[2 * C], pw[C + 1];
    int bad;
};

// The scan of a segment of a head, for the W columns of out from W * member on.
template <int IO, int DC, int NW, int NT, bool FULL, int BY, bool LATE, int ROW>
__device__ __forceinline__ void scan_segment(const AttnScan& a, const AttnRole& R, int64_t group, int member,
                                             Shared<IO, DC, NW * NT * 16, FULL>& lds) {
    using M = Mat<IO>;
    using T = typename M::T;
    using Frag = typename M::Frag;
    constexpr int C = M::kChunk, KB = M::kDepth, W = NW * NT * 16, NTH = NW * 64, B = KB / 16;
    constexpr int PK = DC + Tile<IO>::kPad, PV = W + Tile<IO>::kPad, PA = C + 16 / sizeof(T), NI = C / 16, ND = DC / 16, E = KB / 4;
    constexpr int NS = M::kSplit ? kTerms : 1, NA = NS, NV = M::kSplit ? ROW : 1;
    T *const ks = lds.ks, *const vs = lds.vs, *const qs = lds.qs, *const as = lds.as;
    float *const up = lds.up, *const down = lds.down, *const pw = lds.pw;
    int& bad = lds.bad;
    const int item = (int)(group / a.H), h = (int)(group % a.H), col0 = member * W;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, lr = lane & 15;

    // The segment: sequence s has the items from cu[s] / seg_rows + s on, more than it can need.
    int s, seg;
    int64_t begin, end, slot;
    if (a.cu) {
        int lo = 0, n = a.S;
        while (n > 1) {  // the last sequence that begins at or before this item
            const int step = (n + NTH - 1) / NTH, at = lo + tid * step;
            const bool in = tid * step < n && (int64_t)(min(max(a.cu[at], 0), a.T) / a.seg_rows) + at <= item;
            const int k = max(__syncthreads_count(in) - 1, 0);
            n = min(step, n - k * step);
            lo += k * step;
        }
        s = __builtin_amdgcn_readfirstlane(lo);
        begin = min(max(a.cu[s], 0), a.T);
        end = min(max(a.cu[s + 1], (int)begin), a.T);
        seg = max(item - (int)(begin / a.seg_rows) - s, 0);
        // rows behind the last sequence come back as zeros
        if constexpr (FULL) {
            const int64_t rest = min(max(a.cu[a.S], 0), a.T), wide = (int64_t)a.H * R.Do;
            const int64_t n = (a.T - rest) * wide, share = (n + a.groups - 1) / a.groups;
            if (member == 0 && n > 0 && !R.out32)
                for (int64_t e = group * share + tid; e < min((group + 1) * share, n); e += NTH)
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
            for (int e = tid; e < R.Dc * W; e += NTH) {
                const int c = e / W, o = col0 + e % W;
                const size_t i = at_seq + (size_t)c * R.rs + (size_t)o * R.cs;
                if (o < R.Do) R.fin[i] = R.keep ? R.keep[i] : 0.f;
            }
        return;
    }
    const bool last_seg = p0 + a.seg_rows >= len;
    if (!FULL && last_seg) return;
    const int rows = (int)(min(len, p0 + a.seg_rows) - p0);

    const int64_t first = LATE ? end - 1 - p0 : begin + p0;  // row of position 0
    // the lowest row of n positions from p on
    auto low = [&](int p, int n) { return LATE ? first - p - (n - 1) : first + p; };
    const T* qp = static_cast<const T*>(R.q.p) + (int64_t)(h / R.q.share) * R.q.hs;
    const T* kp = static_cast<const T*>(R.k.p) + (int64_t)(h / R.k.share) * R.k.hs;
    const T* vp = static_cast<const T*>(R.v.p) + (int64_t)(h / R.v.share) * R.v.hs;
    Stage<IO, DC, NTH> sq((int)R.q.ld, 0, R.Dc), sk((int)R.k.ld, 0, R.Dc);
    Stage<IO, W, NTH> sv((int)R.v.ld, col0, R.Do);
    auto load = [&](int p) {
        const int n = min(C, rows - p);
        const int64_t r = low(p, n);
        sk.template load<BY>(kp + r * R.k.ld, (int)R.k.ld, n, R.Dc);
        if constexpr (FULL) sq.template load<BY>(qp + r * R.q.ld, (int)R.q.ld, n, R.Dc);
        sv.template load<BY>(vp + r * R.v.ld, (int)R.v.ld, n, R.Do);
    };
    load(0);

    // powers of a, NaN for a rate that is none
    {
        const float r = a.rate[h];
        const double rate = r >= 0.f && r < INFINITY ? (double)r : (double)NAN;
        if (tid <= C) pw[tid] = (float)exp(-rate * tid);
    }
    __syncthreads();
    const float s_in = LATE ? 1.f : a.scale, s_up = LATE ? a.scale : 1.f;
    const float s_one = LATE ? s_up : s_in, s_two = LATE ? s_in : s_up;  // of the two tables
    if (tid < C) {
        up[tid] = s_one * pw[tid + 1];
        down[tid] = s_two * pw[C - 1 - tid];
        down[C + tid] = 0.f;
    }
    // of the scores: in the tile on the diagonal a^d at and below it; in a tile D further on a^(16 D - 15) times a^(15 + d)
    float w0[4], w1[4];
    if constexpr (FULL)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int d = LATE ? g * 4 + r - lr : lr - g * 4 - r;
            w0[r] = d >= 0 ? a.scale * pw[max(d, 0)] : 0.f;
            w1[r] = a.scale * pw[15 + d];
        }
    const float one = pw[1], sixteen = pw[16];
    if (tid == 0) bad = 0;
    if constexpr (FULL)  // the scores of later rows stay zero
        for (int e = tid; e < NA * C * PA; e += NTH) as[e] = T(0);

    // the wave's columns of the state: rows 16 d + 4 g + r, column lr of block t
    const int wc = wave * NT * 16, col = col0 + wc + lr;
    f32x4 S[ND][NT];
    const float* x = nullptr;
    if (FULL && seg > 0) x = R.seg + ((size_t)slot * a.H + h) * a.state;
    else if (FULL && R.x0) x = R.x0 + at_seq;
    bool sick = false;
    // Entry (16 d + 4 g + r, column of block t) at a lane's offset and a uniform one.  The lane's part is
    // hidden from the compiler, which would keep the offsets of the loads for the stores at the end.
    auto state_offsets = [&]() {
        int c = g * 4, o = col;
        asm volatile("" : "+v"(c), "+v"(o));
        const uint32_t off = (uint32_t)(c * R.rs + o * R.cs) * 4;
        return [&R, c, o, off](int d, int t, int r) {
            return d * 16 + c + r < R.Dc && o + t * 16 < R.Do ? off + (uint32_t)((d * 16 + r) * R.rs + t * 16 * R.cs) * 4 : kOutside;
        };
    };
    const uint32_t s_bytes = (uint32_t)a.state * 4;
    {
        const __amdgpu_buffer_rsrc_t from = row_block(x, x ? s_bytes : 0);
        const auto state_at = state_offsets();
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    S[d][t][r] = FULL ? __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(from, state_at(d, t, r), 0, 0)) : 0.f;
                }
    }
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) sick |= !(fabsf(S[d][t][r]) < INFINITY);
    __syncthreads();
    if (sick) bad = 1;
    float* to_state = nullptr;
    if (!FULL) to_state = const_cast<float*>(R.seg) + ((size_t)(slot + 1) * a.H + h) * a.state;
    else if (last_seg && R.fin) to_state = R.fin + at_seq;

    const int64_t out_ld = (int64_t)a.H * R.Do;
    auto out_row = [&](int64_t row) { return row * out_ld + (int64_t)h * R.Do; };
    // where the lane reads: rows and columns of the tiles
    const T* qrow = qs + lr * PK + Tile<IO>::col(lr, g * 4);
    const T* knear = ks + lr * PK + Tile<IO>::col(lr, g * M::kNear);
    const T* qnear = qs + lr * PK + Tile<IO>::col(lr, g * M::kNear);
    const T* kcol = ks + M::col_at(lane, PK);
    const T* vcol = vs + M::col_at(lane, PV) + wc;
    auto block = [&](int i) { return LATE ? NI - 1 - i : i; };  // of 16 rows, the i-th on the way

    // Rows of out as whole lines: a chunk's are put into the place of its q, and the threads that stage the
    // next q there take them out first (each the 16 bytes that it will overwrite).  Stored as the
    // accumulators hold them, 32 bytes of a row at a time, they cost 7 % more at rows
    // of 64 entries (180 -> 168 us backward at B16 L2048, 16 heads), 2 % at 128.
    constexpr bool kWhole = FULL && BY == 16 && DC == W;
    const bool tile = kWhole && (IO == kRowF32 || !R.out32);
    int left = 0;  // rows of out that are there
    using Out = Stage<IO, DC, NTH>;
    auto take = [&](u32x4 (&y)[Out::U]) {
#pragma unroll
        for (int u = 0; u < Out::U; ++u) y[u] = *reinterpret_cast<const u32x4*>(qs + sq.at(u, 0));
    };
    auto put = [&](const u32x4 (&y)[Out::U], int64_t row, int n) {  // n rows from the first one on
        const __amdgpu_buffer_rsrc_t to = row_block(static_cast<T*>(R.out) + out_row(row) + col0, n > 0 ? (uint32_t)((n - 1) * out_ld + R.Do - col0) * (uint32_t)sizeof(T) : 0);
#pragma unroll
        for (int u = 0; u < Out::U; ++u) {
            const int r = sq.row + u * Out::kRows;
            const uint32_t off = ((uint32_t)r * (uint32_t)out_ld + sq.c) * (uint32_t)sizeof(T);
            const uint32_t at = r < n && col0 + sq.c < R.Do ? off : kOutside;
            if (R.past) __builtin_amdgcn_raw_buffer_store_b128(y[u], to, at, 0, kPastCaches);
            else __builtin_amdgcn_raw_buffer_store_b128(y[u], to, at, 0, 0);
        }
    };

    int p = 0;
    for (; p < rows; p += C) {
        const int n = min(C, rows - p);
        Wild<IO> top;
        u32x4 y[Out::U];
        if constexpr (kWhole) take(y);
        sk.store(ks, 0, top);
        if constexpr (FULL) sq.store(qs, 0, top);
        sv.store(vs, col0, top);
        if (top.any()) bad = 1;
        __syncthreads();
        if constexpr (kWhole) put(y, left > 0 ? low(p - C, left) : 0, left);
        left = 0;
        if (bad) break;
        if (p + C < rows) load(p + C);
        if constexpr (FULL) {
            // the scores that count, 16 x 16 of them at a time
            for (int b = wave; b < NI * (NI + 1) / 2; b += NW) {
                int i = 0, j = b;
                while (j > i) j -= ++i;
                const int bi = block(i) * 16, bj = block(j) * 16;
                // weights first: no branch may stand between the products and what reads them (settle)
                float far = one;
                for (int d = 1; d < i - j; ++d) far *= sixteen;
                float w[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) w[r] = i == j ? w0[r] : w1[r] * far;
                f32x4 sc = {};
#pragma unroll
                for (int kb = 0; kb < DC / KB; ++kb) sc = M::mul(M::near(knear + bj * PK + kb * KB), M::near(qnear + bi * PK + kb * KB), sc);
                float e[8] = {};
#pragma unroll
                for (int r = 0; r < 4; ++r) e[r] = w[r] != 0.f ? sc[r] * w[r] : 0.f;
                Frag f[NA];
                split<IO>(e, f);
                T* to = as + (bi + lr) * PA + bj + g * 4;
#pragma unroll
                for (int m = 0; m < NA; ++m)
                    if constexpr (M::kSplit) {
                        const u32x4 u = __builtin_bit_cast(u32x4, f[m]);
                        *reinterpret_cast<u32x2*>(to + m * C * PA) = u32x2{u.x, u.y};
                    } else {
                        *reinterpret_cast<Frag*>(to) = f[0];
                    }
            }
            // S^T q
            f32x4 acc[NI][NT] = {};
#pragma unroll
            for (int kb = 0; kb < DC / KB; ++kb) {
                Frag f[NT][NS];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    float e[8];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        e[r] = S[kb * B][t][r];
                        e[4 + r] = S[kb * B + B - 1][t][r];
                    }
                    split<IO>(e, f[t]);
                }
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    const Frag qf = M::row(qrow + block(i) * 16 * PK + kb * KB);
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int m = 0; m < NS; ++m) acc[i][t] = M::mul(f[t][m], qf, acc[i][t]);
                }
            }
            const float* in = LATE ? down + C - n : up;
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const float w = in[block(i) * 16 + lr];
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[i][t] *= w;
            }
            __syncthreads();
#pragma unroll
            for (int kb = 0; kb < C / KB; ++kb) {
                const int bj = LATE ? C - KB - kb * KB : kb * KB;
                Frag vf[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) vf[t] = M::col(vcol + bj * PV + t * 16, PV);
#pragma unroll
                for (int i = kb * B; i < NI; ++i)
#pragma unroll
                    for (int m = 0; m < NA; ++m) {
                        const Frag af = M::near(as + (m * C + block(i) * 16 + lr) * PA + bj + g * M::kNear);
#pragma unroll
                        for (int t = 0; t < NT; ++t) acc[i][t] = M::mul(vf[t], af, acc[i][t]);
                    }
            }
            // lane: row lr of a block of 16, columns 4 g .. 4 g + 3
            if (kWhole && tile) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 0; i < NI; ++i) {
                        T* to = qs + (block(i) * 16 + lr) * PK + Tile<IO>::col(lr, wc + t * 16 + g * 4);
                        const f32x4 x = acc[i][t];
                        if constexpr (IO == kRowBf16) *reinterpret_cast<u32x2*>(to) = u32x2{pair(x[0], x[1]), pair(x[2], x[3])};
                        else *reinterpret_cast<f32x4*>(to) = x;
                    }
                left = n;
            } else {
                const int64_t base = out_row(low(p, n));
                const bool f32 = IO == kRowF32 || R.out32;
                const uint32_t size = f32 ? 4 : 2;
                const __amdgpu_buffer_rsrc_t to = row_block(static_cast<char*>(R.out) + base * size, (uint32_t)((n - 1) * out_ld + R.Do) * size);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const int c = col0 + wc + t * 16 + g * 4;
                    const uint32_t off = ((uint32_t)lr * (uint32_t)out_ld + c) * size;
#pragma unroll
                    for (int i = 0; i < NI; ++i) {
                        const int bi = block(i) * 16;
                        const f32x4 x = acc[i][t];
                        if constexpr (BY == 16) {
                            const uint32_t at = bi + lr < n && c < R.Do ? off + (uint32_t)bi * (uint32_t)out_ld * size : kOutside;
                            if (f32) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), to, at, 0, 0);
                            else __builtin_amdgcn_raw_buffer_store_b64(u32x2{pair(x[0], x[1]), pair(x[2], x[3])}, to, at, 0, 0);
                        } else if (bi + lr < n) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int64_t o = base + (bi + lr) * out_ld + c + e;
                                if (c + e >= R.Do) continue;
                                if (f32) static_cast<float*>(R.out)[o] = x[e];
                                else static_cast<uint16_t*>(R.out)[o] = Entry<kRowBf16>::put(x[e]);
                            }
                        }
                    }
                }
            }
        }
        if (p + C < rows || to_state) {
            // the state behind the chunk
            const float keep = pw[n];
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int t = 0; t < NT; ++t) S[d][t] *= keep;
            const float* in = LATE ? up : down + C - n;
#pragma unroll
            for (int kb = 0; kb < C / KB; ++kb) {
                Frag f[NT][NV];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const Frag vf = M::col(vcol + kb * KB * PV + t * 16, PV);
                    float e[8];
#pragma unroll
                    for (int r = 0; r < E; ++r) e[r] = M::get(vf, r) * in[kb * KB + g * M::kNear + r];
                    split<IO>(e, f[t]);
                }
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    const Frag kf = M::col(kcol + kb * KB * PK + d * 16, PK);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
#pragma unroll
                        for (int m = 0; m < NV; ++m) S[d][t] = M::mul(kf, f[t][m], S[d][t]);
                    }
                }
            }
            settle();
        }
        __syncthreads();
    }
    if constexpr (kWhole) {
        u32x4 y[Out::U];
        take(y);
        put(y, left > 0 ? low((rows - 1) / C * C, left) : 0, left);
    }
    // row by row, as the recurrence is written
    for (; p < rows; p += C) {
        const int n = min(C, rows - p);
        __syncthreads();
        load(p);
        Wild<IO> top;
        sk.store(ks, 0, top);
        if constexpr (FULL) sq.store(qs, 0, top);
        sv.store(vs, col0, top);
        __syncthreads();
        for (int r = 0; r < n; ++r) {
            const int at = LATE ? n - 1 - r : r;
            const int64_t to = out_row(low(p, n) + at) + col;
            int g4 = g * 4;
            asm volatile("" : "+v"(g4));  // what depends on it is not kept in registers over the loops
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const float v = s_up * Entry<IO>::get(vs[at * PV + Tile<IO>::col(at, wc + t * 16 + lr)]);
                float o = 0.f;
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int c = d * 16 + g4 + e, i = at * PK + Tile<IO>::col(at, c);
                        const bool has = c < R.Dc;  // no branch: the state stays in registers
                        float x = LATE ? S[d][t][e] : S[d][t][e] * one;
                        x = fmaf(Entry<IO>::get(ks[i]), v, x);
                        if constexpr (FULL) o = has ? fmaf(Entry<IO>::get(qs[i]), x, o) : o;
                        S[d][t][e] = has ? (LATE ? x * one : x) : 0.f;
                    }
                if constexpr (FULL) {
                    o += __shfl_xor(o, 16);
                    o += __shfl_xor(o, 32);
                    o = one == one ? o * s_in : NAN;
                    if (g == 0 && col + t * 16 < R.Do) {
                        if (R.out32 || IO == kRowF32) static_cast<float*>(R.out)[to + t * 16] = o;
                        else static_cast<uint16_t*>(R.out)[to + t * 16] = Entry<kRowBf16>::put(o);
                    }
                }
            }
        }
    }

    if (to_state) {
        const __amdgpu_buffer_rsrc_t to = row_block(to_state, s_bytes);
        const auto state_at = state_offsets();
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(S[d][t][r]), to, state_at(d, t, r), 0, 0);
    }
}

// DC: entries of q and k rows, filled up; NW waves, each of which owns NT blocks of 16 columns of v.
template <int IO, int DC, int NW, int NT, bool FULL, int BY>
__global__ __launch_bounds__(NW * 64, DC > 128 ? NW / 4 : 2) void k_attn_scan(AttnScan a) {
    __shared__ Shared<IO, DC, NW * NT * 16, FULL> lds;
    // the workgroups of one segment of a head are neighbours on one of the 8 XCDs,
    // so that rows which several of them read come from its L2
    const int xcd = blockIdx.x & 7, y = blockIdx.x >> 3;
    const int64_t group = (int64_t)(y / a.members) * 8 + xcd;
    if (group >= a.groups) return;
    int member = y % a.members;
    int ri = 0;
    while (ri + 1 < a.roles && member >= a.role[ri].slices) member -= a.role[ri++].slices;
    const AttnRole& R = a.role[ri];
    // slower loads do without the variant that is faster
    if constexpr (FULL && IO == kRowBf16 && BY == 16) {
        if (R.inner) {
            if (R.late) scan_segment<IO, DC, NW, NT, FULL, BY, true, kInner>(a, R, group, member, lds);
            else scan_segment<IO, DC, NW, NT, FULL, BY, false, kInner>(a, R, group, member, lds);
            return;
        }
    }
    if (R.late) scan_segment<IO, DC, NW, NT, FULL, BY, true, kRow>(a, R, group, member, lds);
    else scan_segment<IO, DC, NW, NT, FULL, BY, false, kRow>(a, R, group, member, lds);
}

template <int IO, int DC, int NW, int NT, bool FULL>
void (*pick(int by))(AttnScan) {
    if (by == 16) return k_attn_scan<IO, DC, NW, NT, FULL, 16>;
    if (IO == kRowF32 || by == 4) return k_attn_scan<IO, DC, NW, NT, FULL, 4>;
    return k_attn_scan<IO, DC, NW, NT, FULL, IO == kRowF32 ? 4 : 2>;
}

// Bytes that all loads of a row may have, as long as they end with the row.
int load_bytes(const HeadsIn& r, int n, int size) {
    for (int by : {16, 4})
        if (reinterpret_cast<uintptr_t>(r.p) % by == 0 && r.ld * size % by == 0 && r.hs * size % by == 0 && n * size % by == 0) return by;
    return 2;
}

}  // namespace

template <int DC>
hipError_t launch_attn_scan(const AttnScan& a, bool full, bool wide, hipStream_t s) {
    const int64_t n = (a.groups + 7) / 8 * 8 * a.members;
    const bool b = a.io == kRowBf16;
    int by = 16;
    for (int r = 0; r < a.roles; ++r) {
        const AttnRole& R = a.role[r];
        by = std::min({by, load_bytes(R.q, R.Dc, b ? 2 : 4), load_bytes(R.k, R.Dc, b ? 2 : 4), load_bytes(R.v, R.Do, b ? 2 : 4)});
        // with 16 rows of out are stored four entries at a time, at offsets below kOutside within a chunk
        const int64_t chunk = (int64_t)(b ? Mat<kRowBf16>::kChunk : Mat<kRowF32>::kChunk) * a.H * R.Do * (b && !R.out32 ? 2 : 4);
        if (full && (R.Do % 4 != 0 || reinterpret_cast<uintptr_t>(R.out) % 16 != 0 || chunk > (int64_t)kOutside)) by = std::min(by, 4);
    }
    // 128 columns: two blocks a wave, or for rows past 128 entries, whose state needs the registers, one
    constexpr int NW = attn_threads(DC, true, true) / 64, NT = DC > 128 ? 1 : 2;
    static_assert(attn_threads(DC, false, true) == 512 && attn_threads(DC, true, false) == 256 && attn_threads(DC, false, false) == 256, "waves below");
    void (*f)(AttnScan);
    if (b) f = full ? (wide ? pick<kRowBf16, DC, NW, NT, true>(by) : pick<kRowBf16, DC, 4, 1, true>(by))
                    : (wide ? pick<kRowBf16, DC, 8, 1, false>(by) : pick<kRowBf16, DC, 4, 1, false>(by));
    else f = full ? (wide ? pick<kRowF32, DC, NW, NT, true>(by) : pick<kRowF32, DC, 4, 1, true>(by))
                  : (wide ? pick<kRowF32, DC, 8, 1, false>(by) : pick<kRowF32, DC, 4, 1, false>(by));
    hipLaunchKernelGGL(f, dim3((unsigned)n), dim3(attn_threads(DC, full, wide)), 0, s, a);
    return hipGetLastError();
}
template hipError_t launch_attn_scan<PDSSM_DC>(const AttnScan&, bool, bool, hipStream_t);

}  // namespace pdssm

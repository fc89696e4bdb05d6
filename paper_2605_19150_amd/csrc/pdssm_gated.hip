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
//   w_t = g_t s_t (i_t x_t a_t^2 / beta_t - a_t h_{t-1})
//   dga_t = w_t (1 - r_t)              drate = sum_t w_t / rate
//   dh0 = a_0 g_0
//
// One read of the inputs.  The rows of all sequences are one axis, cut into
// chunks of kGatedChunk rows without regard to where sequences begin (a row
// that begins one drops what comes from its left), so packed sequences of any
// lengths make equal pieces of work.  A workgroup has one chunk of 64 channels:
// eight waves of 16 rows, a channel a lane.  A wave folds its rows into one
// step (A, B): h_out = A h_in + B; the wave steps are folded in LDS into the
// chunk's; and the state that enters the chunk comes from the chunks before
// it, whose workgroups publish their step as soon as they have it and the state
// behind them when they know it: a chunk takes the nearest known state and the
// steps from there on (chunk_entry).  Then the rows run again, from registers.
//
// Every fold goes in row order from left to right (the backward one from right
// to left), whatever was known when: results do not depend on timing.
#include "pdssm_gated.h"

#include <type_traits>

#include "pdssm_device.h"
#include "pdssm_gated_math.h"

namespace pdssm {
namespace {

// Rows of a wave in each direction, and how many of them the compiler may work
// on at once (more would cost registers, and with them a workgroup of the CU).
constexpr int kFwdRows = 16, kBwdRows = 16, kTogether = 4;

// ------------------------------------------------------------------ workspace
// A ticket counter for every 64 channels, kTicketStride bytes apart, then a
// word for every chunk and channel: empty, a chunk's step
// (A in the high half, which is never negative; B in the low half), or the
// state behind it (sign bit of the high half set).  Value and kind are one
// 8-byte word, so a reader needs no fence.
constexpr uint64_t kEmpty = ~0ull;
constexpr size_t kTicketStride = 256;  // bytes: counters on cache lines of their own

__host__ __device__ inline int chunks_of(int T) { return (T + kGatedChunk - 1) / kGatedChunk; }
__host__ __device__ inline int blocks_of(int C) { return (C + 63) / 64; }
inline size_t words_of(int T, int C) { return (size_t)chunks_of(T) * blocks_of(C) * 64; }
__host__ __device__ inline uint64_t* words_in(void* ws, int NB) {
    return reinterpret_cast<uint64_t*>(static_cast<char*>(ws) + NB * kTicketStride);
}

__device__ __forceinline__ uint64_t step_word(float A, float B) {
    return (uint64_t)(__float_as_uint(A) & 0x7fffffffu) << 32 | __float_as_uint(B);
}
__device__ __forceinline__ uint64_t state_word(float h) { return 0x8000000000000000ull | __float_as_uint(h); }
__device__ __forceinline__ void put_word(uint64_t* p, uint64_t w) {
    __hip_atomic_store(p, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__global__ __launch_bounds__(256) void k_gated_clear(void* ws, int NB, size_t n) {
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i < (size_t)NB) *reinterpret_cast<unsigned*>(static_cast<char*>(ws) + i * kTicketStride) = 0;
    if (i < n) words_in(ws, NB)[i] = kEmpty;
}

// The state (or gradient) that enters a chunk, for the 64 channels of a wave:
// near points at the words of the chunk it comes from, step is the distance to
// the next one further away, n their number.  Words are looked at in batches,
// the nearest first, until one has a state with no gap in front of it; then
// they are folded from there towards the chunk: a state sets the value, a step
// advances it.  Chunks are handed out in the order in which they depend on
// each other (chunk_ticket), so the chunks waited for are running or done, the
// first one waits for nobody, and every wait ends; a wait of kWaitLimit looks
// (over a second) ends all the same, reports PDSSM_ERR_HIP and gives NaN.
constexpr int kBatch = 8, kBatches = 8;
constexpr int kWaitLimit = 1 << 20;
constexpr int kErrWait = -4;  // PDSSM_ERR_HIP

// Folds words d * kBatch .. of the n into h; known: h is a value; gap: an empty word.
__device__ __forceinline__ void fold_batch(const uint64_t* near, ptrdiff_t step, int n, int d, float& h, bool& known,
                                           bool& gap) {
    uint64_t w[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
        const int i = d * kBatch + j;
        w[j] = i < n ? __hip_atomic_load(near + i * step + lane_id(), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : kEmpty;
    }
    gap = false;
#pragma unroll
    for (int j = kBatch - 1; j >= 0; --j) {
        const uint32_t hi = (uint32_t)(w[j] >> 32);
        const float lo = __uint_as_float((uint32_t)w[j]);
        const bool state = (int)hi < 0, empty = w[j] == kEmpty;
        h = state ? lo : fmaf(__uint_as_float(hi), h, lo);
        known = !empty && (state || known);
        gap |= empty;
    }
}

__device__ __forceinline__ float chunk_entry(const uint64_t* near, ptrdiff_t step, int n, int* status) {
    for (int looks = 0; looks < kWaitLimit; ++looks) {
        float h = 0.f;
        for (int d = 0; d < kBatches; ++d) {
            bool known = false, gap;
            fold_batch(near, step, n, d, h, known, gap);
            if (__all(known)) {
                // nearer words may have become states since: the same bits as the fold gives
                while (--d >= 0) fold_batch(near, step, n, d, h, known, gap);
                return h;
            }
            if (__any(gap && !known)) break;  // a chunk in front of the nearest state is not folded yet
        }
        __builtin_amdgcn_s_sleep(2);
    }
    if (status && lane_id() == 0) *status = kErrWait;
    return __uint_as_float(0x7fc00000u);
}

// ------------------------------------------------------------------ sequences
// Sequence of row t, or -1 outside all of them: the last s with cu[s] <= t.
__device__ __forceinline__ int sequence_of(const GatedArgs& a, int t) {
    if (t < 0 || t >= a.T) return -1;
    if (!a.cu) return t / a.L;
    int lo = 0, hi = a.S + 1;  // cu[lo - 1] <= t < cu[hi], as far as cu is in order
    while (lo < hi) {
        const int m = (lo + hi) >> 1;
        if (a.cu[m] <= t) lo = m + 1;
        else hi = m;
    }
    return lo == a.S + 1 ? -1 : lo - 1;
}

// What a wave's rows are: bit i of each mask is row i.
struct RowKinds {
    uint32_t used, first, last;
    int id;  // lane i + 1: sequence of row i
    uint32_t all;
    // rows that begin or end a sequence or are in none; most waves have no such row
    __device__ __forceinline__ uint32_t special() const { return (all & ~used) | first | last; }
    __device__ __forceinline__ int seq(int i) const { return readlane_i(id, i + 1); }
};

template <int ROWS>
__device__ __forceinline__ RowKinds row_kinds(const GatedArgs& a, int row0) {
    RowKinds k;
    constexpr uint32_t kAll = (1u << ROWS) - 1;
    const int lane = lane_id();
    k.id = lane < ROWS + 2 ? sequence_of(a, row0 - 1 + lane) : -1;
    const int before = __shfl_up(k.id, 1), after = __shfl_down(k.id, 1);
    k.all = kAll;
    k.used = (uint32_t)(__ballot(k.id >= 0) >> 1) & kAll;
    k.first = (uint32_t)(__ballot(k.id >= 0 && k.id != before) >> 1) & kAll;
    k.last = (uint32_t)(__ballot(k.id >= 0 && k.id != after) >> 1) & kAll;
    return k;
}

// cu is in order and in range, or the call is reported; out[s] = in[s] (0 if
// in is null) for the sequences without rows.  By one wave for 64 channels.
__device__ void empty_sequences(const GatedArgs& a, const float* in, float* out, int c, bool check) {
    if (!a.cu) return;
    const int lane = lane_id();
    for (int s0 = 0; s0 < a.S; s0 += 64) {
        const int s = s0 + lane;
        const int lo = s < a.S ? a.cu[s] : 0, hi = s < a.S ? a.cu[s + 1] : 0;
        if (check && s < a.S && (lo < 0 || hi < lo || hi > a.T || (s == 0 && lo != 0))) report_index_error(a.status);
        uint64_t none = __ballot(s < a.S && lo == hi);
        while (none) {
            const int k = s0 + __builtin_ctzll(none);
            none &= none - 1;
            if (out && c < a.C) out[(size_t)k * a.C + c] = in ? in[(size_t)k * a.C + c] : 0.f;
        }
    }
}

// ------------------------------------------------------------------ rows
// A wave's rows as a buffer: reads behind the last row give 0, stores there
// are dropped, and so are those of lanes past the last channel, whose offset
// lies past every buffer.
struct RowBlock {
    __amdgpu_buffer_rsrc_t r;
    uint32_t ld;    // bytes from row to row
    uint32_t last;  // offset of the last row (the scalar offset stays within the buffer)
    __device__ __forceinline__ uint32_t at(int i) const { return min((uint32_t)i * ld, last); }
};
constexpr uint32_t kPast = 0x80000000u;  // 16 rows of at most 2^26 bytes and an entry end below it

template <int ROWS>
__device__ __forceinline__ RowBlock row_block_of(const void* p, int64_t ld, int size, int T, int C, int row0) {
    RowBlock b;
    const int n = min(T - row0, ROWS);
    b.ld = (uint32_t)ld * size;
    b.last = n > 0 ? (uint32_t)(n - 1) * b.ld : 0;
    b.r = row_block(static_cast<const char*>(p) + (n > 0 ? (int64_t)row0 * ld * size : 0),
                    n > 0 ? b.last + (uint32_t)C * size : 0);
    return b;
}

template <class T>
__device__ __forceinline__ T load_entry(const RowBlock& b, int i, uint32_t voff) {
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(T, (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(b.r, voff, b.at(i), 0));
    else if constexpr (sizeof(T) == 2) return (T)__builtin_amdgcn_raw_buffer_load_b16(b.r, voff, b.at(i), 0);
    else return (T)__builtin_amdgcn_raw_buffer_load_b8(b.r, voff, b.at(i), 0);
}
// Nobody reads the outputs here again: stored past the caches (nontemporal),
// 147 -> 138 us for the backward at B16 L2048 C1024 bf16.
template <class T>
__device__ __forceinline__ void store_entry(const RowBlock& b, int i, uint32_t voff, T v) {
    if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v), b.r, voff, b.at(i), kLoadStream);
    else if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16(v, b.r, voff, b.at(i), kLoadStream);
    else __builtin_amdgcn_raw_buffer_store_b8((uint8_t)v, b.r, voff, b.at(i), kLoadStream);
}

// This lane's entries of the wave's rows (rows behind the last: 0).
template <int IO, int ROWS>
__device__ __forceinline__ void load_rows(typename Entry<IO>::R (&v)[ROWS], const RowsIn& r, int T, int C, int row0, int c) {
    using E = typename Entry<IO>::T;
    const RowBlock b = row_block_of<ROWS>(r.p, r.ld, sizeof(E), T, C, row0);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) v[i] = load_entry<E>(b, i, (uint32_t)c * sizeof(E));
}

// A barrier for LDS alone: __syncthreads would also wait for the stores of rows.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// The turn of this workgroup among those of its 64 channels (cb), in the order
// in which they begin.  One counter for all of them would hand out tickets
// 12.5 ns apart, 51 us at B16 L2048 C1024, as long as the data takes.
__device__ __forceinline__ int chunk_ticket(void* ws, int cb) {
    __shared__ int mine;
    if (threadIdx.x == 0) mine = (int)atomicAdd(reinterpret_cast<unsigned*>(static_cast<char*>(ws) + cb * kTicketStride), 1u);
    lds_barrier();
    return __builtin_amdgcn_readfirstlane(mine);
}

// A kernel argument that stays in a scalar register from here on: past the
// one-lane branch of the ticket the compiler has carried such values in vector
// registers, and then loops over the lanes for every buffer access.
__device__ __forceinline__ void keep_scalar(int& v) { asm volatile("" : "+s"(v)); }

// ------------------------------------------------------------------ forward
template <int IO, bool KEEP>
__global__ __launch_bounds__(kGatedChunk / kFwdRows * 64, 6) void k_gated_fwd(GatedArgs a) {
    using En = Entry<IO>;
    constexpr int kRows = kFwdRows, kWaves = kGatedChunk / kRows;
    __shared__ float2 fold[kWaves][64];
    __shared__ int cuts[kWaves];
    __shared__ float entry[64];
    __shared__ uint32_t tops[KEEP ? 3 : 1][kWaves][64];
    __shared__ int some[KEEP ? kWaves : 1];
    const int wv = wave_id(), lane = lane_id();
    const int NC = chunks_of(a.T), NB = blocks_of(a.C);
    const int cb = (blockIdx.x + blockIdx.x / NB) % NB;
    const int k = NC > 1 ? chunk_ticket(a.ws, cb) : 0;
    keep_scalar(a.T);
    keep_scalar(a.C);
    const int row0 = k * kGatedChunk + wv * kRows;
    const int c = cb * 64 + lane;
    const bool live = c < a.C;
    const int cc = live ? c : a.C - 1;

    typename En::R x[kRows], ga[kRows], gi[kRows];
    load_rows<IO>(ga, a.ga, a.T, a.C, row0, cc);
    load_rows<IO>(gi, a.gi, a.T, a.C, row0, cc);
    load_rows<IO>(x, a.x, a.T, a.C, row0, cc);
    const float rate2 = a.rate[cc] * kLog2e;
    const RowKinds rows = row_kinds<kRows>(a, row0);
    if (k == 0 && wv == kWaves - 1) empty_sequences(a, a.h0, a.h_final, c, cb == 0);

    if constexpr (KEEP) {
        // the 8-bit form of the rows in sequences; held rows keep only that
        uint32_t top[3] = {0, 0, 0};
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            if (!(rows.used >> i & 1)) continue;
            const float l = En::get(ga[i]);
            const bool hold = l <= kGateHold;
            const float v[3] = {En::get(x[i]), l, En::get(gi[i])};
#pragma unroll
            for (int n = 0; n < 3; ++n) top[n] = max(top[n], hold ? 0u : __float_as_uint(v[n]) & 0x7fffffffu);
        }
#pragma unroll
        for (int n = 0; n < 3; ++n) tops[n][wv][lane] = top[n];
        if (lane == 0) some[wv] = rows.used != 0;
        __syncthreads();
        float inv[3], lim[3];
#pragma unroll
        for (int n = 0; n < 3; ++n) {
            constexpr int kShare = kKeptRows / kRows;  // waves of a block
            uint32_t all = 0;
            bool any = false;
#pragma unroll
            for (int w = 0; w < kShare; ++w) {
                all = max(all, tops[n][(wv & -kShare) + w][lane]);
                any |= __builtin_amdgcn_readfirstlane(some[(wv & -kShare) + w]);
            }
            const int e = kept_exponent(all);
            inv[n] = kept_inverse(e);
            lim[n] = kept_limit(e);
            if (wv % kShare == 0 && any && live) a.e[n][(size_t)(row0 / kKeptRows) * a.C + c] = (int8_t)e;
        }
        const RowBlock q0 = row_block_of<kRows>(a.q[0], a.C, 1, a.T, a.C, row0);
        const RowBlock q1 = row_block_of<kRows>(a.q[1], a.C, 1, a.T, a.C, row0);
        const RowBlock q2 = row_block_of<kRows>(a.q[2], a.C, 1, a.T, a.C, row0);
        const uint32_t voff = live ? (uint32_t)c : kPast;
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            if (!(rows.used >> i & 1)) continue;
            const float l = En::get(ga[i]);
            const bool hold = l <= kGateHold;
            store_entry(q0, i, voff, (int8_t)(hold ? 0 : kept_code(En::get(x[i]), inv[0], lim[0])));
            store_entry(q1, i, voff, (int8_t)(hold ? kKeptLow : kept_code(l, inv[1], lim[1])));
            store_entry(q2, i, voff, (int8_t)(hold ? 0 : kept_code(En::get(gi[i]), inv[2], lim[2])));
        }
    }

    // what few rows need stands in branches that the others jump over
    const uint32_t special = rows.special();
    float av[kRows], bv[kRows];
    float A = 1.f, B = 0.f;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const float l = En::get(ga[i]);
        float r = sigmoid_f(l), in = sigmoid_f(En::get(gi[i])), xi = En::get(x[i]);
        const bool hold = l <= kGateHold;
        if (__builtin_expect(__any(hold), 0)) {
            r = hold ? 0.f : r;  // a = 1 and beta = 0
            in = hold ? 0.f : in;
            xi = hold ? 0.f : xi;
        }
        const Decay d = decay_of(r, rate2);
        av[i] = d.a;
        bv[i] = __builtin_amdgcn_sqrtf(d.beta2) * in * xi;
        float h = B;
        if (__builtin_expect(special >> i & 1, 0)) {
            if (!(rows.used >> i & 1)) av[i] = 1.f, bv[i] = 0.f;
            if (rows.first >> i & 1) {
                bv[i] = fmaf(av[i], a.h0 ? a.h0[(size_t)rows.seq(i) * a.C + cc] : 0.f, bv[i]);
                h = 0.f;
            }
        }
        B = fmaf(av[i], h, bv[i]);
        A *= av[i];
        if (i % kTogether == kTogether - 1) __builtin_amdgcn_sched_barrier(0);
    }
    fold[wv][lane] = make_float2(A, B);
    if (lane == 0) cuts[wv] = rows.first != 0;
    __syncthreads();
    if (wv == 0) {
        float At = 1.f, Bt = 0.f;
        bool cut = k == 0;  // nothing from the left reaches the last row
#pragma unroll 4
        for (int w = 0; w < kWaves; ++w) {
            const float2 f = fold[w][lane];
            const bool cw = __builtin_amdgcn_readfirstlane(cuts[w]);
            Bt = cw ? f.y : fmaf(f.x, Bt, f.y);
            At *= f.x;
            cut |= cw;
        }
        uint64_t* mine = words_in(a.ws, NB) + ((size_t)k * NB + cb) * 64;
        const bool more = k + 1 < NC;
        if (more) put_word(mine + lane, cut ? state_word(Bt) : step_word(At, Bt));
        float h = 0.f;
        if (k > 0 && !(rows.first & 1)) {
            h = chunk_entry(mine - (size_t)NB * 64, -(ptrdiff_t)NB * 64, k, a.status);
            if (more && !cut) put_word(mine + lane, state_word(fmaf(At, h, Bt)));
        }
        entry[lane] = h;
        if (a.saved && live && (rows.used & 1)) a.saved[(size_t)k * a.C + c] = h;
    }
    __syncthreads();
    float h = entry[lane];
    for (int w = 0; w < wv; ++w) {
        const float2 f = fold[w][lane];
        h = __builtin_amdgcn_readfirstlane(cuts[w]) ? f.y : fmaf(f.x, h, f.y);
    }
    const RowBlock y = row_block_of<kRows>(a.y, a.C, sizeof(typename En::T), a.T, a.C, row0);
    const uint32_t voff = live ? (uint32_t)c * sizeof(typename En::T) : kPast;
    auto emit = [&](auto plain_) {
        constexpr bool PLAIN = decltype(plain_)::value;
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            h = !PLAIN && (rows.first >> i & 1) ? bv[i] : fmaf(av[i], h, bv[i]);
            if (PLAIN || (rows.used >> i & 1)) store_entry(y, i, voff, En::put(h));
            if constexpr (!PLAIN)
                if ((rows.last >> i & 1) && live && a.h_final) a.h_final[(size_t)rows.seq(i) * a.C + c] = h;
        }
    };
    if (special == 0) emit(std::true_type{});
    else emit(std::false_type{});
}

// ------------------------------------------------------------------ backward
// IN: format of x, ga, gi (IO's, or the 8-bit form).
template <int IO, int IN>
__global__ __launch_bounds__(kGatedChunk / kBwdRows * 64, 4) void k_gated_bwd(GatedArgs a, float* part) {
    using En = Entry<IO>;
    constexpr int kRows = kBwdRows, kWaves = kGatedChunk / kRows;
    __shared__ float fold[3][kWaves][64];
    __shared__ int cuts[2][kWaves];
    __shared__ float entry[64];
    const int wv = wave_id(), lane = lane_id();
    const int NC = chunks_of(a.T), NB = blocks_of(a.C);
    const int cb = (blockIdx.x + blockIdx.x / NB) % NB;
    const int k = NC - 1 - (NC > 1 ? chunk_ticket(a.ws, cb) : 0);  // from the last chunk to the first
    keep_scalar(a.T);
    keep_scalar(a.C);
    const int row0 = k * kGatedChunk + wv * kRows;
    const int c = cb * 64 + lane;
    const bool live = c < a.C;
    const int cc = live ? c : a.C - 1;

    typename Entry<IN>::R xr[kRows], gar[kRows], gir[kRows];
    typename En::R dyr[kRows];
    load_rows<IN>(gar, a.ga, a.T, a.C, row0, cc);
    load_rows<IN>(gir, a.gi, a.T, a.C, row0, cc);
    load_rows<IN>(xr, a.x, a.T, a.C, row0, cc);
    load_rows<IO>(dyr, a.dy, a.T, a.C, row0, cc);
    float scale[3] = {1.f, 1.f, 1.f};
    if constexpr (IN == kRowKept) {
        const size_t o = (size_t)(min(row0, a.T - 1) / kKeptRows) * a.C + cc;
        scale[0] = kept_scale(a.x.e[o]);
        scale[1] = kept_scale(a.ga.e[o]);
        scale[2] = kept_scale(a.gi.e[o]);
    }
    const float rate = a.rate[cc], rate2 = rate * kLog2e;
    const float before_chunk = a.saved[(size_t)k * a.C + cc];
    const RowKinds rows = row_kinds<kRows>(a, row0);
    if (k == 0 && wv == kWaves - 1) empty_sequences(a, a.dhf, a.dh0, c, cb == 0);

    // gates, and the wave's two folds: states from the left, gradients from the
    // right.  hb: the row's input term, later the state before it.  a and beta
    // are computed anew from r wherever they are needed: with them kept, a
    // wave's 16 rows would not leave room for a second workgroup on the CU,
    // which is what hides this one's waits (203 us with rows halved and all
    // kept, one workgroup a CU, at B16 L2048 C1024 bf16)
    const uint32_t special = rows.special();

    float r[kRows], in[kRows], hb[kRows];
    float A = 1.f, B = 0.f, G = 0.f, Gend = 0.f;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const float l = Entry<IN>::gate(gar[i], scale[1]);
        r[i] = sigmoid_f(l);
        in[i] = sigmoid_f(Entry<IN>::get(gir[i], scale[2]));
        float ix = in[i] * Entry<IN>::get(xr[i], scale[0]);
        const bool hold = l <= kGateHold;

        r[i] = hold ? 0.f : r[i];
        ix = hold ? 0.f : ix;
        float h = B;
        if (__builtin_expect(special >> i & 1, 0)) {
            if (!(rows.used >> i & 1)) r[i] = 0.f;
            if (rows.first >> i & 1) h = a.h0 ? a.h0[(size_t)rows.seq(i) * a.C + cc] : 0.f;
        }
        const Decay d = decay_of(r[i], rate2);
        hb[i] = __builtin_amdgcn_sqrtf(d.beta2) * ix;
        B = fmaf(d.a, h, hb[i]);
        A *= d.a;
        // the gradient that leaves the first row: dy of each row times the a's up to it ...
        G = fmaf(A, En::get(dyr[i]), G);
        // ... as far as the first row that ends a sequence
        if (__builtin_expect((rows.last & ((2u << i) - 1)) == 1u << i, 0))
            Gend = fmaf(A, a.dhf ? a.dhf[(size_t)rows.seq(i) * a.C + cc] : 0.f, G);
        if (i % kTogether == kTogether - 1) __builtin_amdgcn_sched_barrier(0);
    }
    if (rows.last) G = Gend;
    fold[0][wv][lane] = A;
    fold[1][wv][lane] = B;
    fold[2][wv][lane] = G;
    if (lane == 0) {
        cuts[0][wv] = rows.first != 0;
        cuts[1][wv] = rows.last != 0;
    }
    __syncthreads();
    // the last wave's rows end the chunk: it finds what comes from the right
    if (wv == kWaves - 1) {
        float At = 1.f, Gt = 0.f;
        bool cut = k == NC - 1;
#pragma unroll 4
        for (int w = kWaves - 1; w >= 0; --w) {
            const bool cw = __builtin_amdgcn_readfirstlane(cuts[1][w]);
            Gt = cw ? fold[2][w][lane] : fmaf(fold[0][w][lane], Gt, fold[2][w][lane]);
            At *= fold[0][w][lane];
            cut |= cw;
        }
        uint64_t* mine = words_in(a.ws, NB) + ((size_t)k * NB + cb) * 64;
        if (k > 0) put_word(mine + lane, cut ? state_word(Gt) : step_word(At, Gt));
        float u = 0.f;
        if (k + 1 < NC && !(rows.last >> (kRows - 1) & 1)) {
            u = chunk_entry(mine + (size_t)NB * 64, (ptrdiff_t)NB * 64, NC - 1 - k, a.status);
            if (k > 0 && !cut) put_word(mine + lane, state_word(fmaf(At, u, Gt)));
        }
        entry[lane] = u;
    }
    // the states before the rows, while that wave may wait
    float h = before_chunk;
#pragma unroll 4
    for (int w = 0; w < wv; ++w)
        h = __builtin_amdgcn_readfirstlane(cuts[0][w]) ? fold[1][w][lane] : fmaf(fold[0][w][lane], h, fold[1][w][lane]);
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        if (__builtin_expect(rows.first >> i & 1, 0)) h = a.h0 ? a.h0[(size_t)rows.seq(i) * a.C + cc] : 0.f;
        const float b = hb[i];
        hb[i] = h;
        h = fmaf(__builtin_amdgcn_exp2f(-rate2 * r[i]), h, b);
        // what comes of these is computed again below, not kept
        asm volatile("" : "+v"(r[i]), "+v"(xr[i]), "+v"(dyr[i]));
    }
    __syncthreads();
    float u = entry[lane];
#pragma unroll 4
    for (int w = kWaves - 1; w > wv; --w)
        u = __builtin_amdgcn_readfirstlane(cuts[1][w]) ? fold[2][w][lane] : fmaf(fold[0][w][lane], u, fold[2][w][lane]);
    RowBlock out[3];
#pragma unroll
    for (int n = 0; n < 3; ++n) out[n] = row_block_of<kRows>(a.d[n], a.ldd, sizeof(typename En::T), a.T, a.C, row0);
    const uint32_t voff = live ? (uint32_t)c * sizeof(typename En::T) : kPast;
    float sum = 0.f;
#pragma unroll
    for (int i = kRows - 1; i >= 0; --i) {
        if (__builtin_expect(rows.last >> i & 1, 0)) u = a.dhf ? a.dhf[(size_t)rows.seq(i) * a.C + cc] : 0.f;
        const float g = En::get(dyr[i]) + u, x = Entry<IN>::get(xr[i], scale[0]);
        const Decay d = decay_of(r[i], rate2);
        const float t = in[i] * __builtin_amdgcn_rsqf(d.beta2);  // i / beta
        float dx = g * d.beta2 * t;
        u = g * d.a;
        float w = rate * r[i] * u * fmaf(x * d.a, t, -hb[i]);
        float dxx = dx * x;
        dxx = fmaf(-dxx, in[i], dxx);
        {
            const bool hold = r[i] == 0.f;
            dx = hold ? 0.f : dx;
            w = hold ? 0.f : w;
            dxx = hold ? 0.f : dxx;
        }
        sum += w;
        if (rows.used >> i & 1) {
            store_entry(out[0], i, voff, En::put(dx));
            store_entry(out[1], i, voff, En::put(fmaf(-w, r[i], w)));
            store_entry(out[2], i, voff, En::put(dxx));
        }
        if (__builtin_expect((rows.first >> i & 1) && live && a.dh0, 0)) a.dh0[(size_t)rows.seq(i) * a.C + c] = u;
        if (i % kTogether == 0) __builtin_amdgcn_sched_barrier(0);
    }
    if (!a.drate) return;
    __syncthreads();
    fold[0][wv][lane] = sum;
    __syncthreads();
    if (wv == 0 && live) {
        float all = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) all += fold[0][w][lane];
        if (NC > 1) part[(size_t)k * a.C + c] = all;
        else a.drate[c] = all / rate;
    }
}

// drate from the chunks' sums: 16 waves take every 16th chunk of 64 channels.
__global__ __launch_bounds__(1024) void k_gated_rate(const float* part, const float* rate, float* drate, int NC, int C) {
    __shared__ float sums[16][64];
    const int wv = wave_id(), lane = lane_id(), c = blockIdx.x * 64 + lane;
    float s = 0.f;
    if (c < C)
        for (int k = wv; k < NC; k += 16) s += part[(size_t)k * C + c];
    sums[wv][lane] = s;
    __syncthreads();
    if (wv != 0 || c >= C) return;
    s = 0.f;
    for (int w = 0; w < 16; ++w) s += sums[w][lane];
    drate[c] = s / rate[c];
}

// No rows at all: out = in for every sequence, and a zero rate gradient.
__global__ __launch_bounds__(64) void k_gated_none(GatedArgs a, const float* in, float* out) {
    const int c = blockIdx.x * 64 + threadIdx.x;
    if (a.cu) empty_sequences(a, in, out, c, blockIdx.x == 0);
    if (c >= a.C) return;
    if (!a.cu && out)
        for (int s = 0; s < a.S; ++s) out[(size_t)s * a.C + c] = in ? in[(size_t)s * a.C + c] : 0.f;
    if (a.drate) a.drate[c] = 0.f;
}

template <int IO>
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
    using En = Entry<IO>;
    auto at = [&](const RowsIn& r) { return En::get(static_cast<const typename En::T*>(r.p)[(size_t)b * r.ld + c]); };
    const float l = at(a.ga);
    const bool hold = l <= kGateHold;
    const Decay d = decay_of(hold ? 0.f : sigmoid_f(l), a.rate[c] * kLog2e);
    const float in = hold ? 0.f : __builtin_amdgcn_sqrtf(d.beta2) * sigmoid_f(at(a.gi)) * at(a.x);
    const size_t o = (size_t)slot * a.C + c;
    const float h = fmaf(d.a, a.h_in[o], in);
    a.h_out[o] = h;
    static_cast<typename En::T*>(a.y)[(size_t)b * a.C + c] = En::put(h);
}

}  // namespace

size_t gated_workspace(int T, int C, int S, bool bwd) {
    if (chunks_of(T) <= 1) return 0;
    return blocks_of(C) * kTicketStride + words_of(T, C) * 8 + (bwd ? (size_t)chunks_of(T) * C * 4 : 0);
}

namespace {
void clear_words(const GatedArgs& a, hipStream_t s) {
    const int NB = blocks_of(a.C);
    const size_t n = words_of(a.T, a.C);  // at least 128 for each counter
    hipLaunchKernelGGL(k_gated_clear, dim3((n + 255) / 256), dim3(256), 0, s, a.ws, NB, n);
}
}  // namespace

hipError_t launch_gated_fwd(const GatedArgs& a, hipStream_t s) {
    const int NC = chunks_of(a.T), NB = blocks_of(a.C);
    if (NC == 0) {
        hipLaunchKernelGGL(k_gated_none, dim3(NB), dim3(64), 0, s, a, a.h0, a.h_final);
        return hipGetLastError();
    }
    if (NC > 1) clear_words(a, s);
    constexpr int kWaves = kGatedChunk / kFwdRows;
    auto* f = a.io == kRowBf16 ? (a.q[0] ? k_gated_fwd<kRowBf16, true> : k_gated_fwd<kRowBf16, false>)
                               : (a.q[0] ? k_gated_fwd<kRowF32, true> : k_gated_fwd<kRowF32, false>);
    hipLaunchKernelGGL(f, dim3((unsigned)NC * NB), dim3(kWaves * 64), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_gated_bwd(const GatedArgs& a, hipStream_t s) {
    const int NC = chunks_of(a.T), NB = blocks_of(a.C);
    if (NC == 0) {
        hipLaunchKernelGGL(k_gated_none, dim3(NB), dim3(64), 0, s, a, a.dhf, a.dh0);
        return hipGetLastError();
    }
    float* part = nullptr;
    if (NC > 1) {
        clear_words(a, s);
        part = reinterpret_cast<float*>(words_in(a.ws, NB) + words_of(a.T, a.C));
    }
    constexpr int kWaves = kGatedChunk / kBwdRows;
    auto* f = a.io == kRowBf16 ? (a.kept ? k_gated_bwd<kRowBf16, kRowKept> : k_gated_bwd<kRowBf16, kRowBf16>)
                               : (a.kept ? k_gated_bwd<kRowF32, kRowKept> : k_gated_bwd<kRowF32, kRowF32>);
    hipLaunchKernelGGL(f, dim3((unsigned)NC * NB), dim3(kWaves * 64), 0, s, a, part);
    if (NC > 1 && a.drate) hipLaunchKernelGGL(k_gated_rate, dim3(NB), dim3(1024), 0, s, part, a.rate, a.drate, NC, a.C);
    return hipGetLastError();
}

hipError_t launch_gated_step(const GatedStepArgs& a, hipStream_t s) {
    auto* f = a.io == kRowBf16 ? k_gated_step<kRowBf16> : k_gated_step<kRowF32>;
    hipLaunchKernelGGL(f, dim3((a.C + 255) / 256, a.B), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace pdssm

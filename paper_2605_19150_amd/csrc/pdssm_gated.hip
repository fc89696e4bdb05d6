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
// eight waves of 16 rows, a channel (or two, see Shape) a lane.  A wave folds its rows into one
// step (A, B): h_out = A h_in + B; the wave steps are folded in LDS into the
// chunk's; and the state that enters the chunk comes from the chunks before
// it, whose workgroups publish their step as soon as they have it and the state
// behind them when they know it: a chunk takes the nearest known state and the
// steps from there on (chunk_entry).  Then the rows run again, from registers.
//
// Every fold goes in row order from left to right (the backward one from right
// to left), whatever was known when: results do not depend on timing.
//
// Bound by memory, with the arithmetic close behind: six to nine hardware
// exponentials, reciprocals and roots and about as many other operations as fit
// under an entry's bytes.  At B16 L2048 C1024 bf16 a forward call takes 59 us
// (270 MB, 4.6 TB/s; a large copy reaches 5.2), a backward call 122 us (471 MB,
// 3.9 TB/s), the vector units about 70% busy; in fp32 the kernels take about 100
// and 180 us (539 and 942 MB, 5.2 to 5.4 TB/s).  Forward with the 8-bit form and
// backward from it, B8 L18000 C1024 bf16: 915 us (3.28 GB), the vector units 80%
// busy.
#include "pdssm_gated.h"

#include "pdssm_device.h"
#include "pdssm_gated_math.h"

namespace pdssm {
namespace {

constexpr int kWaves = 8, kWaveRows = kGatedChunk / kWaves;  // of a workgroup; 64 channels wide
// Rows the compiler may work on at once: more would cost registers, and with
// them a workgroup of the CU.
constexpr int kTogether = 4;
static_assert(kKeptRows == 2 * kWaveRows, "two waves share an exponent");

// How a wave's lanes lie on its 16 rows of 64 channels: V channels next to each
// other in a lane, V groups of lanes one below the other.  The backward pass
// takes two where the rows are bf16 and of even width and alignment: half as
// many accesses, each of them 4 bytes a lane.  With fp32 a lane's one entry
// has those 4 bytes already, and two cost registers that then spill (184 ->
// 226 us at B16 L2048 C1024, bf16 134 -> 128 us).  The forward pass has one:
// two leave room for 6 waves instead of 8 (60 -> 66 us there).
template <int V>
struct Shape {
    static constexpr int ROWS = kWaveRows / V, LANES = 64 / V;
    static constexpr int TOGETHER = kTogether / V;
};

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

// Four words a thread (n is a multiple of 64).
__global__ __launch_bounds__(256) void k_gated_clear(void* ws, int NB, size_t n) {
    typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i < (size_t)NB) *reinterpret_cast<unsigned*>(static_cast<char*>(ws) + i * kTicketStride) = 0;
    if (i * 4 >= n) return;
    u64x2* w = reinterpret_cast<u64x2*>(words_in(ws, NB) + i * 4);
    w[0] = w[1] = u64x2{kEmpty, kEmpty};
}

// The state (or gradient) that enters a chunk, for the 64 channels of a wave:
// near points at the words of the chunk it comes from, step is the distance to
// the next one further away, n their number.  Words are looked at in batches,
// the nearest first, until one has a state with no gap in front of it; then
// they are folded from there towards the chunk: a state sets the value, a step
// advances it.  Chunks are handed out in the order in which they depend on
// each other (chunk_ticket), so the chunks waited for are running or done, the
// first one waits for nobody, and every wait ends; a wait of kWaitLimit looks
// (seconds) ends all the same, reports PDSSM_ERR_HIP and gives NaN.
constexpr int kBatch = 4, kBatches = 16;  // with batches of 8 the forward at B16 L2048 C1024 bf16 takes 56.5 us, of 4 53.8, of 2 55.4
constexpr int kWaitLimit = 1 << 22;
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
};
constexpr uint32_t kAllRows = (1u << kWaveRows) - 1;

__device__ __forceinline__ RowKinds row_kinds(const GatedArgs& a, int row0) {
    RowKinds k;
    const int lane = lane_id();
    k.id = lane < kWaveRows + 2 ? sequence_of(a, row0 - 1 + lane) : -1;
    const int before = __shfl_up(k.id, 1), after = __shfl_down(k.id, 1);
    k.used = (uint32_t)(__ballot(k.id >= 0) >> 1) & kAllRows;
    k.first = (uint32_t)(__ballot(k.id >= 0 && k.id != before) >> 1) & kAllRows;
    k.last = (uint32_t)(__ballot(k.id >= 0 && k.id != after) >> 1) & kAllRows;
    return k;
}

// A lane's part of them.  The masks with _any are those of all groups of lanes
// laid over each other, the same in every lane: what few rows need stands in
// branches on them that the other rows jump over.
template <int V>
struct LaneRows {
    static constexpr int ROWS = Shape<V>::ROWS;
    static constexpr uint32_t kAll = (1u << ROWS) - 1;
    uint32_t used, first, last, unused_any, first_any, last_any;
    int id, g;
    __device__ __forceinline__ LaneRows(const RowKinds& k, int g_) : id(k.id), g(g_) {
        used = k.used >> (g * ROWS) & kAll;
        first = k.first >> (g * ROWS) & kAll;
        last = k.last >> (g * ROWS) & kAll;
        unused_any = first_any = last_any = 0;
#pragma unroll
        for (int n = 0; n < V; ++n) {
            unused_any |= ~k.used >> (n * ROWS) & kAll;
            first_any |= k.first >> (n * ROWS) & kAll;
            last_any |= k.last >> (n * ROWS) & kAll;
        }
    }
    // bit i of a lane's mask, formed where it is asked for (see rare)
    static __device__ __forceinline__ bool is(uint32_t mask, int i) {
        asm volatile("" : "+v"(mask));
        return mask >> i & 1;
    }
    // Sequence of row i, 0 where it has none.  Waited for here and not behind
    // the branch: there the wait would hold for all rows' loads and stores, of
    // the many waves too that do not take it.
    __device__ __forceinline__ int sequence(int i) const {
        int q = V == 1 ? readlane_i(id, i + 1) : __shfl(id, g * ROWS + i + 1);
        if constexpr (V == 2) asm volatile("" : "+v"(q));
        return max(q, 0);
    }
    // s[sequence of row i][c] where wanted (0 without s), else what it was
    __device__ __forceinline__ float state(const float* s, int i, int C, int c, bool wanted, float else_) const {
        const int q = sequence(i);
        if (wanted) {
            else_ = s ? s[(size_t)q * C + c] : 0.f;
            asm volatile("" : "+v"(else_));
        }
        return else_;
    }
    __device__ __forceinline__ float* place(float* s, int i, int C, int c) const { return s + (size_t)sequence(i) * C + c; }
};

// cu is in order and in range, or the call is reported; out[s] = in[s] (0 if
// in is null) for the sequences without rows.  Wave `turn` of `waves` takes its
// part of them for 64 channels.  Behind everything that another workgroup waits
// for, and by all waves: one wave in front of the first chunk's step took 34 ms
// for 131072 sequences (T131072 C64 bf16, now 0.07), and every chunk waited for it.
__device__ void empty_sequences(const GatedArgs& a, const float* in, float* out, int c, bool check, int turn, int64_t waves) {
    if (!a.cu) return;
    const int lane = lane_id();
    for (int64_t s0 = 64LL * turn; s0 < a.S; s0 += 64 * waves) {
        const int s = (int)s0 + lane;  // S <= 2^30
        const int lo = s < a.S ? a.cu[s] : 0, hi = s < a.S ? a.cu[s + 1] : 0;
        if (check && s < a.S && (lo < 0 || hi < lo || hi > a.T || (s == 0 && lo != 0))) report_index_error(a.status);
        uint64_t none = __ballot(s < a.S && lo == hi);
        while (none) {
            const int k = (int)s0 + __builtin_ctzll(none);
            none &= none - 1;
            if (out && c < a.C) out[(size_t)k * a.C + c] = in ? in[(size_t)k * a.C + c] : 0.f;
        }
    }
}

// ------------------------------------------------------------------ rows
// A wave's rows as a buffer.  A row behind the last one is, to the first group of
// lanes, the last one again (the scalar offset ends there), to the second one
// past the buffer, which reads 0: either way a row in no sequence, which the
// masks of RowKinds leave out.  Stores of such rows, and of lanes past the last
// channel, get an offset past every buffer and are dropped.
struct RowBlock {
    __amdgpu_buffer_rsrc_t r;
    uint32_t ld;    // bytes from row to row
    uint32_t last;  // offset of the last row (the scalar offset stays within the buffer)
    __device__ __forceinline__ uint32_t at(int i) const { return min((uint32_t)i * ld, last); }
};
constexpr uint32_t kPast = 0x80000000u;  // 16 rows of at most 2^26 bytes and an entry end below it

__device__ __forceinline__ RowBlock row_block_of(const void* p, int64_t ld, int size, int T, int C, int row0) {
    RowBlock b;
    const int n = min(T - row0, kWaveRows);
    b.ld = (uint32_t)ld * size;
    b.last = n > 0 ? (uint32_t)(n - 1) * b.ld : 0;
    b.r = row_block(static_cast<const char*>(p) + (n > 0 ? (int64_t)row0 * ld * size : 0),
                    n > 0 ? b.last + (uint32_t)C * size : 0);
    return b;
}

// V neighbouring entries of a row in a register, and row i of a lane's group in
// memory.  Nobody reads the outputs here again: they are stored past the caches
// (nontemporal), 147 -> 138 us for the backward at B16 L2048 C1024 bf16.
// In 32 bits the sigmoid is 1 from kOpen = 127 * 2^-2 up (1 - 1.6e-14) and 0
// from kShut down (its reciprocal is past the largest number): what the 8-bit
// form keeps of logits further out need not tell them apart.
constexpr float kOpen = 31.75f, kShut = -89.f;
template <int IO, int V>
struct Some;
template <>
struct Some<kRowF32, 1> {
    using R = float;
    static constexpr int SIZE = 4;
    static __device__ __forceinline__ R load(const RowBlock& b, int i, uint32_t voff) {
        return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(b.r, voff, b.at(i), 0));
    }
    static __device__ __forceinline__ float get(R v, int, float = 1.f) { return v; }
    static __device__ __forceinline__ void store(const RowBlock& b, int i, uint32_t voff, float v) {
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), b.r, voff, b.at(i), kLoadStream);
    }
};
template <>
struct Some<kRowBf16, 1> {
    using R = uint32_t;
    static constexpr int SIZE = 2;
    static __device__ __forceinline__ R load(const RowBlock& b, int i, uint32_t voff) {
        return (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(b.r, voff, b.at(i), 0);
    }
    static __device__ __forceinline__ float get(R v, int, float = 1.f) { return __uint_as_float(v << 16); }
    static __device__ __forceinline__ void store(const RowBlock& b, int i, uint32_t voff, float v) {
        __builtin_amdgcn_raw_buffer_store_b16(Entry<kRowBf16>::put(v), b.r, voff, b.at(i), kLoadStream);
    }
};
template <>
struct Some<kRowBf16, 2> {
    using R = uint32_t;
    static constexpr int SIZE = 2;
    static __device__ __forceinline__ R load(const RowBlock& b, int i, uint32_t voff) {
        return __builtin_amdgcn_raw_buffer_load_b32(b.r, voff, b.at(i), 0);
    }
    static __device__ __forceinline__ float get(R v, int n, float = 1.f) {
        return __uint_as_float(n ? v & 0xffff0000u : v << 16);
    }
    static __device__ __forceinline__ void store(const RowBlock& b, int i, uint32_t voff, const float (&v)[2]) {
        __builtin_amdgcn_raw_buffer_store_b32(f2_to_bf2(make_float2(v[0], v[1])), b.r, voff, b.at(i), kLoadStream);
    }
};
template <>
struct Some<kRowKept, 1> {
    using R = int;
    static constexpr int SIZE = 1;
    static __device__ __forceinline__ R load(const RowBlock& b, int i, uint32_t voff) {
        return (int8_t)__builtin_amdgcn_raw_buffer_load_b8(b.r, voff, b.at(i), 0);
    }
    static __device__ __forceinline__ int code(R v, int) { return v; }
    static __device__ __forceinline__ float get(R v, int, float scale) { return (float)v * scale; }
    static __device__ __forceinline__ void store(const RowBlock& b, int i, uint32_t voff, int v) {
        __builtin_amdgcn_raw_buffer_store_b8((uint8_t)v, b.r, voff, b.at(i), kLoadStream);
    }
};
template <>
struct Some<kRowKept, 2> {
    using R = uint32_t;
    static constexpr int SIZE = 1;
    static __device__ __forceinline__ R load(const RowBlock& b, int i, uint32_t voff) {
        return (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(b.r, voff, b.at(i), 0);
    }
    static __device__ __forceinline__ int code(R v, int n) { return (int8_t)(v >> (8 * n)); }
    static __device__ __forceinline__ float get(R v, int n, float scale) { return (float)code(v, n) * scale; }
};

// A gate logit; in the 8-bit form with the code of -inf.
template <int IO, int V>
__device__ __forceinline__ float logit(typename Some<IO, V>::R v, int n, float scale) {
    if constexpr (IO == kRowKept)
        if (Some<IO, V>::code(v, n) == kKeptLow) return -INFINITY;
    return Some<IO, V>::get(v, n, scale);
}

// This lane's entries of the wave's rows, channels c ...; row by row, in the
// order of their use, so that the first row's work begins when it is there
// (backward at B16 L2048 C1024 bf16: 124 -> 119 us).
template <int IO, int V>
struct RowsOf {
    using S = Some<IO, V>;
    RowBlock b;
    uint32_t voff;
    __device__ __forceinline__ RowsOf(const RowsIn& r, int T, int C, int row0, int g, int c)
        : b(row_block_of(r.p, r.ld, S::SIZE, T, C, row0)), voff((uint32_t)(g * Shape<V>::ROWS) * b.ld + (uint32_t)c * S::SIZE) {}
    __device__ __forceinline__ typename S::R row(int i) const { return S::load(b, i, voff); }
};

// The same entry of the other group of lanes.
__device__ __forceinline__ float other_group(float v) { return __shfl_xor(v, 32); }

// A barrier for LDS alone: __syncthreads would also wait for the stores of rows.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// The 64 channels of a workgroup.  The XCDs take workgroups in turn; kRun column
// blocks next to each other go to one XCD one after the other, so that lines
// that two of them share are mostly read once (forward at B16 L2048 C1024 bf16
// 58.7 -> 56.3 us, backward at C1023 152 -> 145 us).  From row of blocks to row
// they move on by one: with the same columns always on the same XCD the backward
// from the 8-bit form took a tenth longer (T144000 C1024).
constexpr int kXcds = 8, kRun = 4;
__device__ __forceinline__ int block_of(int NB) {
    const int b = blockIdx.x, whole = gridDim.x & ~(kXcds * kRun - 1);
    const int j = b < whole ? (b & ~(kXcds * kRun - 1)) + b % kXcds * kRun + b / kXcds % kRun : b;
    return (j + j / NB) % NB;
}

// The turn of this workgroup among those of its 64 channels (cb), in the order
// in which they begin.  One counter for all of them would hand out tickets
// 12.5 ns apart, 51 us at B16 L2048 C1024, as long as the data takes.
__device__ __forceinline__ int chunk_ticket(void* ws, int cb) {
    __shared__ int mine;
    if (threadIdx.x == 0) mine = (int)atomicAdd(reinterpret_cast<unsigned*>(static_cast<char*>(ws) + cb * kTicketStride), 1u);
    lds_barrier();
    return __builtin_amdgcn_readfirstlane(mine);
}

// Whether row i is one of mask, the same in every lane; for what few rows need.
// Tested where it is used: the compiler would form the tests of all rows at
// once and keep them, in more scalar registers than there are (forward that
// keeps its rows, C1024 T32768 fp32, with the backward: 310 -> 293 us).
__device__ __forceinline__ bool rare(uint32_t mask, int i) {
    mask = __builtin_amdgcn_readfirstlane(mask);
    asm volatile("" : "+s"(mask));
    return __builtin_expect(mask >> i & 1, 0);
}

// A kernel argument that stays in a scalar register from here on: past the
// one-lane branch of the ticket the compiler has carried such values in vector
// registers, and then loops over the lanes for every buffer access.
__device__ __forceinline__ void keep_scalar(int& v) { asm volatile("" : "+s"(v)); }

// ------------------------------------------------------------------ forward
template <int IO, bool KEEP>
__global__ __launch_bounds__(kWaves * 64, 6) void k_gated_fwd(GatedArgs a) {
    using S = Some<IO, 1>;
    constexpr int ROWS = kWaveRows;
    __shared__ float fold[2][kWaves][64];  // a wave's step: A, B
    __shared__ float entry[64];
    __shared__ uint32_t tops[KEEP ? 3 : 1][kWaves][64];
    __shared__ int cuts[kWaves], some[kWaves];
    const int wv = wave_id(), lane = lane_id();
    const int NC = chunks_of(a.T), NB = blocks_of(a.C);
    const int cb = block_of(NB);
    const int k = NC > 1 ? chunk_ticket(a.ws, cb) : 0;
    keep_scalar(a.T);
    keep_scalar(a.C);
    const int row0 = k * kGatedChunk + wv * kWaveRows;
    const int c = cb * 64 + lane;
    const bool live = c < a.C;
    const int cc = live ? c : a.C - 1;

    typename S::R x[ROWS], ga[ROWS], gi[ROWS];
    const float rate_in = a.rate[cc];
    const RowsOf<IO, 1> xs(a.x, a.T, a.C, row0, 0, cc), gas(a.ga, a.T, a.C, row0, 0, cc), gis(a.gi, a.T, a.C, row0, 0, cc);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        ga[i] = gas.row(i);
        gi[i] = gis.row(i);
        x[i] = xs.row(i);
        __builtin_amdgcn_sched_barrier(0);
    }
    const RowKinds kinds = row_kinds(a, row0);
    const LaneRows<1> rows(kinds, 0);
    const float rate = rate_of(rate_in);  // looked at behind the rows' loads: it would hold them up
    // whether row i, in no sequence, is written all the same: a zero
    auto rest = [&](int i) { return a.zero_rest && row0 + i < a.T; };
    if constexpr (KEEP) {
        // the 8-bit form of the rows in sequences; held rows keep only that
        uint32_t top[3] = {0, 0, 0};
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const float l = S::get(ga[i], 0);
            bool skip = l <= kGateHold;
            if (rare(rows.unused_any, i)) skip |= !rows.is(rows.used, i);
            const float v[3] = {S::get(x[i], 0), l, S::get(gi[i], 0)};
#pragma unroll
            for (int m = 0; m < 3; ++m) top[m] = max(top[m], skip ? 0u : __float_as_uint(v[m]) & 0x7fffffffu);
        }
        // A gate far out is no reason to lose the codes of its block: past kOpen,
        // +inf too, both gates count as kOpen and get the largest code at most,
        // and an input gate from kShut down (-inf, the type's lowest value) has
        // no part in the exponent and gets the code that reads -inf, or its own.
        // In a branch that waves without such gates jump over (forward at B8 L18000
        // C1024 bf16 407 us, with such a gate in every wave 430; 624 when the
        // branch read its rows again).
        constexpr uint32_t kOpenBits = 0x41fe0000u;
        // widened and compared again from here on: kept for the codes, across the
        // branch, what the rows above made would spill
#pragma unroll
        for (int i = 0; i < ROWS; ++i) asm volatile("" : "+v"(ga[i]), "+v"(gi[i]), "+v"(x[i]));
        if (__builtin_expect(__any(top[1] > kOpenBits || top[2] > kOpenBits), 0)) {
            auto counts = [](float v) { return __float_as_uint(v > kOpen ? kOpen : v) & 0x7fffffffu; };
            top[1] = top[2] = 0;
#pragma unroll
            for (int i = 0; i < ROWS; ++i) {
                const float l = S::get(ga[i], 0), n = S::get(gi[i], 0);
                bool skip = l <= kGateHold;
                if (rare(rows.unused_any, i)) skip |= !rows.is(rows.used, i);
                top[1] = max(top[1], skip ? 0u : counts(l));
                top[2] = max(top[2], skip || n <= kShut ? 0u : counts(n));
                if (i % kTogether == kTogether - 1) __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int m = 0; m < 3; ++m) tops[m][wv][lane] = top[m];
        if (lane == 0) some[wv] = kinds.used != 0;
        __syncthreads();
        float inv[3], lim[3], low = 0.f;
        const bool any = __builtin_amdgcn_readfirstlane(some[wv & ~1] | some[wv | 1]);
#pragma unroll
        for (int m = 0; m < 3; ++m) {
            const int e = kept_exponent(max(top[m], tops[m][wv ^ 1][lane]));
            inv[m] = kept_inverse(e);
            lim[m] = kept_limit(e);
            if (m == 2) low = kept_low(e);
            if (!(wv & 1) && (any || rest(0)) && live) a.e[m][(size_t)(row0 / kKeptRows) * a.C + c] = (int8_t)e;
        }
        RowBlock q[3];
#pragma unroll
        for (int m = 0; m < 3; ++m) q[m] = row_block_of(a.q[m], a.C, 1, a.T, a.C, row0);
        const uint32_t voff = live ? (uint32_t)c : kPast;
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            uint32_t to = voff;
            const float l = S::get(ga[i], 0);
            const bool hold = l <= kGateHold;
            int code[3] = {hold ? 0 : kept_code(S::get(x[i], 0), inv[0], lim[0]), hold ? kKeptLow : kept_code(l, inv[1], lim[1]),
                           hold ? 0 : kept_code_or_low(S::get(gi[i], 0), inv[2], low, lim[2])};
            if (rare(rows.unused_any, i) && !rows.is(rows.used, i)) {
                to = rest(i) ? voff : kPast;
                code[0] = code[1] = code[2] = 0;
            }
#pragma unroll
            for (int m = 0; m < 3; ++m) Some<kRowKept, 1>::store(q[m], i, to, code[m]);
        }
    }

    const uint32_t special = rows.unused_any | rows.first_any | rows.last_any;
    float av[ROWS], bv[ROWS], A = 1.f, B = 0.f;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const float l = S::get(ga[i], 0);
        float r = sigmoid_f(l), in = sigmoid_f(S::get(gi[i], 0)), xi = S::get(x[i], 0);
        const bool hold = l <= kGateHold;
        if (__builtin_expect(__any(hold), 0)) {
            r = hold ? 0.f : r;  // a = 1 and beta = 0
            in = hold ? 0.f : in;
            xi = hold ? 0.f : xi;
        }
        const Decay d = decay_of(r, rate);
        av[i] = d.a;
        bv[i] = __builtin_amdgcn_sqrtf(d.beta2) * in * xi;
        float h = B;
        if (rare(special, i)) {
            if (!rows.is(rows.used, i)) av[i] = 1.f, bv[i] = 0.f;
            const bool first = rows.is(rows.first, i);
            bv[i] = fmaf(av[i], rows.state(a.h0, i, a.C, cc, first, 0.f), bv[i]);
            h = first ? 0.f : h;
        }
        B = fmaf(av[i], h, bv[i]);
        A *= av[i];
        if (i % kTogether == kTogether - 1) __builtin_amdgcn_sched_barrier(0);
    }
    fold[0][wv][lane] = A;
    fold[1][wv][lane] = B;
    if (lane == 0) cuts[wv] = kinds.first != 0;
    __syncthreads();
    const uint32_t cut_waves = (uint32_t)__ballot(lane < kWaves && cuts[lane & (kWaves - 1)]);
    if (wv == 0) {
        float At = 1.f, Bt = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            Bt = cut_waves >> w & 1 ? fold[1][w][lane] : fmaf(fold[0][w][lane], Bt, fold[1][w][lane]);
            At *= fold[0][w][lane];
        }
        const bool cut = k == 0 || cut_waves;  // nothing from the left reaches the last row
        uint64_t* mine = words_in(a.ws, NB) + ((size_t)k * NB + cb) * 64;
        const bool more = k + 1 < NC;
        if (more) put_word(mine + lane, cut ? state_word(Bt) : step_word(At, Bt));
        float h = 0.f;
        if (k > 0 && !(kinds.first & 1)) {
            h = chunk_entry(mine - (size_t)NB * 64, -(ptrdiff_t)NB * 64, k, a.status);
            if (more && !cut) put_word(mine + lane, state_word(fmaf(At, h, Bt)));
        }
        entry[lane] = h;
        const bool used = kinds.used & 1;
        if (a.saved && live && (used || rest(0))) a.saved[(size_t)k * a.C + c] = used ? h : 0.f;
    }
    __syncthreads();
    float h = entry[lane];
#pragma unroll 4
    for (int w = 0; w < wv; ++w)
        h = cut_waves >> w & 1 ? fold[1][w][lane] : fmaf(fold[0][w][lane], h, fold[1][w][lane]);
    const RowBlock y = row_block_of(a.y, a.C, S::SIZE, a.T, a.C, row0);
    const uint32_t voff = live ? (uint32_t)c * S::SIZE : kPast;
    if (special == 0) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            h = fmaf(av[i], h, bv[i]);
            S::store(y, i, voff, h);
        }
    } else {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            h = rows.is(rows.first, i) ? bv[i] : fmaf(av[i], h, bv[i]);
            const bool used = rows.is(rows.used, i);
            S::store(y, i, used || rest(i) ? voff : kPast, used ? h : 0.f);
            float* f = rows.place(a.h_final, i, a.C, cc);
            if (rows.is(rows.last, i) && live && a.h_final) *f = h;
        }
    }
    empty_sequences(a, a.h0, a.h_final, c, cb == 0, k * kWaves + wv, (int64_t)NC * kWaves);
}

// ------------------------------------------------------------------ backward
// IN: format of x, ga, gi (IO's, or the 8-bit form).
template <int IO, int IN, int V>
__global__ __launch_bounds__(kWaves * 64, 4) void k_gated_bwd(GatedArgs a, float* part) {
    using S = Some<IO, V>;
    using N = Some<IN, V>;
    constexpr int ROWS = Shape<V>::ROWS;
    __shared__ __align__(8) float fold[3][kWaves][64];  // a wave's steps: A, B from the left, G from the right
    __shared__ __align__(8) float entry[64];
    __shared__ float sums[kWaves * V][64];
    __shared__ int cuts[2][kWaves];
    const int wv = wave_id(), lane = lane_id();
    const int NC = chunks_of(a.T), NB = blocks_of(a.C);
    const int cb = block_of(NB);
    const int k = NC - 1 - (NC > 1 ? chunk_ticket(a.ws, cb) : 0);  // from the last chunk to the first
    keep_scalar(a.T);
    keep_scalar(a.C);
    const int row0 = k * kGatedChunk + wv * kWaveRows;
    const int g = V == 1 ? 0 : lane / Shape<V>::LANES, lc = lane % Shape<V>::LANES * V;
    const int c = cb * 64 + lc;
    const bool live = c < a.C;
    const int cc = live ? c : a.C - V;

    float scale[3][V], rate[V], h[V];
#pragma unroll
    for (int n = 0; n < V; ++n) {
        scale[0][n] = scale[1][n] = scale[2][n] = 1.f;
        if constexpr (IN == kRowKept) {
            const size_t o = (size_t)(min(row0, a.T - 1) / kKeptRows) * a.C + cc + n;
            scale[0][n] = kept_scale(a.x.e[o]);
            scale[1][n] = kept_scale(a.ga.e[o]);
            scale[2][n] = kept_scale(a.gi.e[o]);
        }
        rate[n] = a.rate[cc + n];
        h[n] = a.saved[(size_t)k * a.C + cc + n];  // the state before the chunk
    }
    typename N::R xr[ROWS], gar[ROWS], gir[ROWS];
    typename S::R dyr[ROWS];
    const RowsOf<IN, V> xs(a.x, a.T, a.C, row0, g, cc), gas(a.ga, a.T, a.C, row0, g, cc), gis(a.gi, a.T, a.C, row0, g, cc);
    const RowsOf<IO, V> dys(a.dy, a.T, a.C, row0, g, cc);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        gar[i] = gas.row(i);
        gir[i] = gis.row(i);
        xr[i] = xs.row(i);
        dyr[i] = dys.row(i);
        __builtin_amdgcn_sched_barrier(0);
    }
    const RowKinds kinds = row_kinds(a, row0);
    const LaneRows<V> rows(kinds, g);
#pragma unroll
    for (int n = 0; n < V; ++n) rate[n] = rate_of(rate[n]);
    // gates, and the two folds: states from the left, gradients from the right.
    // hb: the row's input term, later the state before it; r = 0 where the state
    // is held (no other logit gives it).  a and beta are computed anew from r
    // wherever they are needed: kept, they would not leave room for a second
    // workgroup on the CU, which is what hides this one's waits (half the rows,
    // all kept, one workgroup a CU: 203 us, where this took 149 then, at B16 L2048
    // C1024 bf16; all kept and spilled in part: 161 us, now 120).
    float r[ROWS][V], in[ROWS][V], hb[ROWS][V], A[V], B[V], G[V], Gend[V];
#pragma unroll
    for (int n = 0; n < V; ++n) A[n] = 1.f, B[n] = G[n] = Gend[n] = 0.f;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
#pragma unroll
        for (int n = 0; n < V; ++n) {
            const float l = logit<IN, V>(gar[i], n, scale[1][n]);
            r[i][n] = sigmoid_f(l);
            in[i][n] = sigmoid_f(logit<IN, V>(gir[i], n, scale[2][n]));
            float ix = in[i][n] * N::get(xr[i], n, scale[0][n]);
            const bool hold = l <= kGateHold;
            r[i][n] = hold ? 0.f : r[i][n];
            ix = hold ? 0.f : ix;
            float before = B[n];
            if (rare(rows.unused_any | rows.first_any, i)) {
                if (!rows.is(rows.used, i)) r[i][n] = 0.f;
                before = rows.state(a.h0, i, a.C, cc + n, rows.is(rows.first, i), before);
            }
            const Decay d = decay_of(r[i][n], rate[n]);
            hb[i][n] = __builtin_amdgcn_sqrtf(d.beta2) * ix;
            B[n] = fmaf(d.a, before, hb[i][n]);
            A[n] *= d.a;
            // the gradient that leaves the first row: dy of each row times the a's up to it ...
            G[n] = fmaf(A[n], S::get(dyr[i], n), G[n]);
            // ... as far as the first row that ends a sequence
            if (rare(rows.last_any, i)) {
                const bool end = rows.is(rows.last & (0u - rows.last), i);
                const float from = rows.state(a.dhf, i, a.C, cc + n, end, 0.f);
                if (end) Gend[n] = fmaf(A[n], from, G[n]);
            }
        }
        if (i % Shape<V>::TOGETHER == Shape<V>::TOGETHER - 1) __builtin_amdgcn_sched_barrier(0);
    }
    // the wave's steps from its groups'; Ag, Bg: the upper group's, Al, Gl: the lower one's
    const bool first_upper = (kinds.first & LaneRows<V>::kAll) != 0, first_lower = kinds.first >> ROWS != 0;
    const bool last_upper = (kinds.last & LaneRows<V>::kAll) != 0, last_lower = kinds.last >> ROWS != 0;
    float Ag[V], Bg[V], Al[V], Gl[V];
#pragma unroll
    for (int n = 0; n < V; ++n) {
        if (rows.last) G[n] = Gend[n];
        Ag[n] = Al[n] = A[n];
        Bg[n] = B[n];
        Gl[n] = G[n];
        if constexpr (V == 2) {
            const float Ao = other_group(A[n]), Bo = other_group(B[n]), Go = other_group(G[n]);
            const float Bl = g ? B[n] : Bo, Gu = g ? Go : G[n];
            Al[n] = g ? A[n] : Ao;
            Ag[n] = g ? Ao : A[n];
            Bg[n] = g ? Bo : B[n];
            Gl[n] = g ? G[n] : Go;
            A[n] = Al[n] * Ag[n];
            B[n] = first_lower ? Bl : fmaf(Al[n], Bg[n], Bl);
            G[n] = last_upper ? Gu : fmaf(Ag[n], Gl[n], Gu);
        }
        if (g == 0) {
            fold[0][wv][lc + n] = A[n];
            fold[1][wv][lc + n] = B[n];
            fold[2][wv][lc + n] = G[n];
        }
    }
    if (lane == 0) {
        cuts[0][wv] = kinds.first != 0;
        cuts[1][wv] = kinds.last != 0;
    }
    __syncthreads();
    const uint32_t first_waves = (uint32_t)__ballot(lane < kWaves && cuts[0][lane & (kWaves - 1)]);
    const uint32_t last_waves = (uint32_t)__ballot(lane < kWaves && cuts[1][lane & (kWaves - 1)]);
    // the last wave's rows end the chunk: it finds what comes from the right
    if (wv == kWaves - 1) {
        float At = 1.f, Gt = 0.f;
#pragma unroll 4
        for (int w = kWaves - 1; w >= 0; --w) {
            Gt = last_waves >> w & 1 ? fold[2][w][lane] : fmaf(fold[0][w][lane], Gt, fold[2][w][lane]);
            At *= fold[0][w][lane];
        }
        const bool cut = k == NC - 1 || last_waves;
        uint64_t* mine = words_in(a.ws, NB) + ((size_t)k * NB + cb) * 64;
        if (k > 0) put_word(mine + lane, cut ? state_word(Gt) : step_word(At, Gt));
        float u = 0.f;
        if (k + 1 < NC && !(kinds.last >> (kWaveRows - 1) & 1)) {
            u = chunk_entry(mine + (size_t)NB * 64, (ptrdiff_t)NB * 64, NC - 1 - k, a.status);
            if (k > 0 && !cut) put_word(mine + lane, state_word(fmaf(At, u, Gt)));
        }
        entry[lane] = u;
    }
    // the states before the rows, while that wave may wait
#pragma unroll
    for (int n = 0; n < V; ++n) {
#pragma unroll 4
        for (int w = 0; w < wv; ++w)
            h[n] = first_waves >> w & 1 ? fold[1][w][lc + n] : fmaf(fold[0][w][lc + n], h[n], fold[1][w][lc + n]);
        if (g) h[n] = first_upper ? Bg[n] : fmaf(Ag[n], h[n], Bg[n]);
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
#pragma unroll
        for (int n = 0; n < V; ++n) {
            if (rare(rows.first_any, i)) h[n] = rows.state(a.h0, i, a.C, cc + n, rows.is(rows.first, i), h[n]);
            const float b = hb[i][n];
            hb[i][n] = h[n];
            h[n] = fmaf(decay_of(r[i][n], rate[n]).a, h[n], b);
            asm volatile("" : "+v"(r[i][n]));  // what comes of these is computed again below, not kept
        }
        asm volatile("" : "+v"(xr[i]), "+v"(dyr[i]));
    }
    __syncthreads();
    float u[V], sum[V];
#pragma unroll
    for (int n = 0; n < V; ++n) {
        u[n] = entry[lc + n];
        sum[n] = 0.f;
#pragma unroll 4
        for (int w = kWaves - 1; w > wv; --w)
            u[n] = last_waves >> w & 1 ? fold[2][w][lc + n] : fmaf(fold[0][w][lc + n], u[n], fold[2][w][lc + n]);
        if (V == 2 && g == 0) u[n] = last_lower ? Gl[n] : fmaf(Al[n], u[n], Gl[n]);
    }
    RowBlock out[3];
#pragma unroll
    for (int m = 0; m < 3; ++m) out[m] = row_block_of(a.d[m], a.ldd, S::SIZE, a.T, a.C, row0);
    const uint32_t voff = live ? (uint32_t)(g * ROWS) * out[0].ld + (uint32_t)c * S::SIZE : kPast;
#pragma unroll
    for (int i = ROWS - 1; i >= 0; --i) {
        float d0[V], d1[V], d2[V];
#pragma unroll
        for (int n = 0; n < V; ++n) {
            if (rare(rows.last_any, i)) u[n] = rows.state(a.dhf, i, a.C, cc + n, rows.is(rows.last, i), u[n]);
            const float gr = S::get(dyr[i], n) + u[n], x = N::get(xr[i], n, scale[0][n]);
            const Decay d = decay_of(r[i][n], rate[n]);
            const float t = in[i][n] * __builtin_amdgcn_rsqf(d.beta2);  // i / beta
            float dx = gr * d.beta2 * t;
            u[n] = gr * d.a;
            float w = d.s * u[n] * fmaf(x * d.a, t, -hb[i][n]);
            float dxx = dx * x;
            dxx = fmaf(-dxx, in[i][n], dxx);
            const bool hold = d.beta2 < 1.17549435e-38f;  // r = 0; roots know no smaller numbers either
            d0[n] = hold ? 0.f : dx;
            w = hold ? 0.f : w;
            d2[n] = hold ? 0.f : dxx;
            sum[n] += w;
            d1[n] = fmaf(-w, r[i][n], w);
        }
        uint32_t to = voff;
        if (rare(rows.unused_any | rows.first_any, i)) {
            to = rows.is(rows.used, i) ? voff : kPast;
#pragma unroll
            for (int n = 0; n < V; ++n) {
                float* f = rows.place(a.dh0, i, a.C, cc + n);
                if (rows.is(rows.first, i) && live && a.dh0) *f = u[n];
            }
        }
        if constexpr (V == 1) {
            S::store(out[0], i, to, d0[0]);
            S::store(out[1], i, to, d1[0]);
            S::store(out[2], i, to, d2[0]);
        } else {
            S::store(out[0], i, to, d0);
            S::store(out[1], i, to, d1);
            S::store(out[2], i, to, d2);
        }
        if (i % Shape<V>::TOGETHER == 0) __builtin_amdgcn_sched_barrier(0);
    }
    // the rows behind the last sequence are zero if the caller asks for it (the
    // stores above drop them)
    if (a.zero_rest && a.cu)
        for (int t = max(row0, a.cu[a.S]); t < min(a.T, row0 + kWaveRows); ++t)
#pragma unroll
            for (int m = 0; m < 3; ++m)
                if (cb * 64 + lane < a.C) static_cast<typename Entry<IO>::T*>(a.d[m])[t * a.ldd + cb * 64 + lane] = 0;
    empty_sequences(a, a.dhf, a.dh0, cb * 64 + lane, cb == 0, (NC - 1 - k) * kWaves + wv, (int64_t)NC * kWaves);
    if (!a.drate) return;
#pragma unroll
    for (int n = 0; n < V; ++n) sums[wv * V + g][lc + n] = sum[n];
    __syncthreads();
    const int ch = cb * 64 + lane;
    if (wv == 0 && ch < a.C) {
        float all = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves * V; ++w) all += sums[w][lane];
        if (NC > 1) part[(size_t)k * a.C + ch] = all;
        else a.drate[ch] = all / rate_of(a.rate[ch]);
    }
}

// drate from the chunks' sums, 16 channels a workgroup: quarter q of wave w
// takes every 64th chunk from 4 w + q on.
__global__ __launch_bounds__(1024) void k_gated_rate(const float* part, const float* rate, float* drate, int NC, int C) {
    __shared__ float sums[16][16];
    const int wv = wave_id(), lane = lane_id(), ch = lane & 15, c = blockIdx.x * 16 + ch;
    float s = 0.f;
    if (c < C) {
#pragma unroll 4
        for (int k = wv * 4 + lane / 16; k < NC; k += 64) s += part[(size_t)k * C + c];
    }
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    if (lane < 16) sums[wv][ch] = s;
    __syncthreads();
    if (wv != 0 || lane >= 16 || c >= C) return;
    s = 0.f;
#pragma unroll
    for (int w = 0; w < 16; ++w) s += sums[w][ch];
    drate[c] = s / rate_of(rate[c]);
}

// No rows at all: out = in for every sequence, and a zero rate gradient.  A
// workgroup along y takes its part of the sequences.
__global__ __launch_bounds__(64) void k_gated_none(GatedArgs a, const float* in, float* out) {
    const int c = blockIdx.x * 64 + threadIdx.x;
    if (a.cu) empty_sequences(a, in, out, c, blockIdx.x == 0, blockIdx.y, gridDim.y);
    if (c >= a.C) return;
    if (!a.cu && out)
        for (int s = blockIdx.y; s < a.S; s += gridDim.y) out[(size_t)s * a.C + c] = in ? in[(size_t)s * a.C + c] : 0.f;
    if (a.drate && blockIdx.y == 0) a.drate[c] = 0.f / rate_of(a.rate[c]);
}

// V entries of a row, next to each other and aligned as one.
template <int IO, int V>
struct alignas(V * sizeof(typename Entry<IO>::T)) Pack {
    typename Entry<IO>::T v[V];
};

// One row b of a batch, V channels a thread.
template <int IO, int V>
__global__ __launch_bounds__(256) void k_gated_step(GatedStepArgs a) {
    using En = Entry<IO>;
    using Row = Pack<IO, V>;
    using State = Pack<kRowF32, V>;
    const int c = (blockIdx.x * 256 + threadIdx.x) * V, b = blockIdx.y;
    const bool live = c < a.C;
    int slot = b;
    if (a.slots) {
        slot = a.slots[b];
        if (slot < 0 || slot >= a.pool) {
            if (slot >= a.pool) report_index_error(a.status);
            return;
        }
    }
    auto at = [&](const RowsIn& r) {
        return *reinterpret_cast<const Row*>(static_cast<const typename En::T*>(r.p) + (size_t)b * r.ld + c);
    };
    const size_t o = (size_t)slot * a.C + c;
    Row x = {}, ga = {}, gi = {};
    State rate = {}, h = {};
    if (live) {
        x = at(a.x);
        ga = at(a.ga);
        gi = at(a.gi);
        rate = *reinterpret_cast<const State*>(a.rate + c);
        h = *reinterpret_cast<const State*>(a.h_in + o);
    }
    // the first row that names a slot has it; others of the same batch are refused
    bool again = false;
    if (a.slots)
        for (int k = threadIdx.x; k < b; k += 256) again |= a.slots[k] == slot;
    if (__syncthreads_or(again)) {
        report_index_error(a.status);
        return;
    }
    if (!live) return;
    Row y;
#pragma unroll
    for (int n = 0; n < V; ++n) {
        const float l = En::get(ga.v[n]);
        const bool hold = l <= kGateHold;
        const Decay d = decay_of(hold ? 0.f : sigmoid_f(l), rate_of(rate.v[n]));
        const float in = hold ? 0.f : __builtin_amdgcn_sqrtf(d.beta2) * sigmoid_f(En::get(gi.v[n])) * En::get(x.v[n]);
        h.v[n] = fmaf(d.a, h.v[n], in);
        y.v[n] = En::put(h.v[n]);
    }
    *reinterpret_cast<State*>(a.h_out + o) = h;
    *reinterpret_cast<Row*>(static_cast<typename En::T*>(a.y) + (size_t)b * a.C + c) = y;
}

}  // namespace

size_t gated_workspace(int T, int C, bool bwd) {
    if (chunks_of(T) <= 1) return 0;
    return blocks_of(C) * kTicketStride + words_of(T, C) * 8 + (bwd ? (size_t)chunks_of(T) * C * 4 : 0);
}

namespace {
void clear_words(const GatedArgs& a, hipStream_t s) {
    const int NB = blocks_of(a.C);
    const size_t n = words_of(a.T, a.C);  // at least 128 for each counter, so there are threads for all of them
    hipLaunchKernelGGL(k_gated_clear, dim3((n / 4 + 255) / 256), dim3(256), 0, s, a.ws, NB, n);
}
}  // namespace

namespace {
hipError_t launch_none(const GatedArgs& a, const float* in, float* out, hipStream_t s) {
    const int parts = a.S < 1024 ? a.S : 1024;
    hipLaunchKernelGGL(k_gated_none, dim3(blocks_of(a.C), parts), dim3(64), 0, s, a, in, out);
    return hipGetLastError();
}

// Whether rows of size-byte entries can be read n channels at a time.
bool by(int n, const void* p, int64_t ld, int size) {
    return reinterpret_cast<uintptr_t>(p) % (n * size) == 0 && ld % n == 0;
}
}  // namespace

hipError_t launch_gated_fwd(const GatedArgs& a, hipStream_t s) {
    const int NC = chunks_of(a.T), NB = blocks_of(a.C);
    if (NC == 0) return launch_none(a, a.h0, a.h_final, s);
    if (NC > 1) clear_words(a, s);
    auto go = [&](auto* f) { hipLaunchKernelGGL(f, dim3((unsigned)NC * NB), dim3(kWaves * 64), 0, s, a); };
    const bool keep = a.q[0] != nullptr;
    if (a.io == kRowBf16) {
        keep ? go(k_gated_fwd<kRowBf16, true>) : go(k_gated_fwd<kRowBf16, false>);
    } else {
        keep ? go(k_gated_fwd<kRowF32, true>) : go(k_gated_fwd<kRowF32, false>);
    }
    return hipGetLastError();
}

hipError_t launch_gated_bwd(const GatedArgs& a, hipStream_t s) {
    const int NC = chunks_of(a.T), NB = blocks_of(a.C);
    if (NC == 0) return launch_none(a, a.dhf, a.dh0, s);
    float* part = nullptr;
    if (NC > 1) {
        clear_words(a, s);
        part = reinterpret_cast<float*>(words_in(a.ws, NB) + words_of(a.T, a.C));
    }
    bool two = a.io == kRowBf16 && a.C % 2 == 0 && by(2, a.dy.p, a.dy.ld, 2);
    for (const RowsIn* r : {&a.x, &a.ga, &a.gi}) two = two && by(2, r->p, r->ld, a.kept ? 1 : 2);
    for (const void* d : a.d) two = two && by(2, d, a.ldd, 2);
    auto go = [&](auto* f) { hipLaunchKernelGGL(f, dim3((unsigned)NC * NB), dim3(kWaves * 64), 0, s, a, part); };
    if (a.io == kRowBf16) {
        if (two) a.kept ? go(k_gated_bwd<kRowBf16, kRowKept, 2>) : go(k_gated_bwd<kRowBf16, kRowBf16, 2>);
        else a.kept ? go(k_gated_bwd<kRowBf16, kRowKept, 1>) : go(k_gated_bwd<kRowBf16, kRowBf16, 1>);
    } else {
        a.kept ? go(k_gated_bwd<kRowF32, kRowKept, 1>) : go(k_gated_bwd<kRowF32, kRowF32, 1>);
    }
    if (NC > 1 && a.drate) hipLaunchKernelGGL(k_gated_rate, dim3((a.C + 15) / 16), dim3(1024), 0, s, part, a.rate, a.drate, NC, a.C);
    return hipGetLastError();
}

hipError_t launch_gated_step(const GatedStepArgs& a, hipStream_t s) {
    // four channels a thread where width and alignment allow: 11.5 -> 7.6 us for 512 rows of 4096 bf16 channels
    const int size = a.io == kRowBf16 ? 2 : 4;
    bool four = a.C % 4 == 0 && by(4, a.y, a.C, size);
    for (const RowsIn* r : {&a.x, &a.ga, &a.gi}) four = four && by(4, r->p, r->ld, size);
    for (const float* p : {a.rate, a.h_in, static_cast<const float*>(a.h_out)}) four = four && by(4, p, a.C, 4);
    const int wide = four ? 1024 : 256;
    auto* f = a.io == kRowBf16 ? (four ? k_gated_step<kRowBf16, 4> : k_gated_step<kRowBf16, 1>)
                               : (four ? k_gated_step<kRowF32, 4> : k_gated_step<kRowF32, 1>);
    hipLaunchKernelGGL(f, dim3((a.C + wide - 1) / wide, a.B), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace pdssm

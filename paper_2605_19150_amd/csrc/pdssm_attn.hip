// pdssm_attn.hip -- linear attention with a decay for each head: the launches
// of whole sequences, and the step of one token.
//
// With S_t = a S_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t and G_t the gradient
// that reaches S_t (G_t = scale q_t do_t^T + a G_{t+1}) the gradients are
//   dq_t = scale S_t do_t,   dk_t = G_t v_t,   dv_t = G_t^T k_t:
// the forward scan with (do, v, k) in the places of (q, k, v), and two scans from the
// last row to the first with (v, do, q) and (k, q, do).  One kernel has all four
// (pdssm_attn_scan.hip); the three of a backward pass run in one launch where
// their rows have one length, as neighbours that share what they read.
//
// Where sequences and heads are too few to fill the card a sequence is cut into
// segments: a first launch adds up what the rows of each segment do to the state
// (it reads k and v once more), k_segments joins them, and the scan begins every
// segment from its state.  Nothing waits for another workgroup, sums have one order.
#include <math.h>

#include "pdssm_attn.h"
#include "pdssm_device.h"
#include "pdssm_rows.h"

namespace pdssm {

namespace {

constexpr int kFill = 512;      // workgroups that fill the card: two on each of 256 CUs
// A row output goes past the caches from kPast bytes on, which they would not keep for its reader, if a head's rows are
// whole pieces of kPiece bytes: neighbours in a piece come from other workgroups.  Backward at 65536 rows of 32 heads of
// 64, bf16, that takes 670 us, and of 24 heads of 96 1150 for 1168 through the caches.  Where pieces are not
// whole it is slower: 32 heads of 48 take 815 for 783, of 40 690 for 673, 24 of 104 forward 590 for 565.
constexpr int64_t kPast = 64 << 20;
constexpr int kPiece = 64;
constexpr int kFillPacked = 768;  // the same where lengths differ
constexpr int kSegmentMin = 128;  // rows below which a segment is not worth its state

struct Plan {
    int seg_rows, items;
    int64_t slots;  // states that segments begin with; 0: no sequence is cut
};

int slices(int cols, bool wide) { return (cols + (wide ? 127 : 63)) / (wide ? 128 : 64); }
bool wide_cols(const AttnArgs& a, bool bwd) { return (bwd ? max(a.Dk, a.Dv) : a.Dv) > 64; }
int members(const AttnArgs& a, bool bwd) {
    const bool wide = wide_cols(a, bwd);
    return bwd ? 2 * slices(a.Dk, wide) + slices(a.Dv, wide) : slices(a.Dv, wide);
}

Plan plan(const AttnArgs& a, bool bwd) {
    const int chunk = a.io == kRowBf16 ? 64 : 32;
    const int64_t heads = (int64_t)a.H * members(a, bwd);
    Plan p = {};
    if (!a.cu) {
        const int64_t whole = a.S * heads;
        const int fill = max(a.Dk, a.Dv) <= 64 ? kFill * 3 / 2 : kFill;
        int64_t n = whole >= fill ? 1 : min((fill + whole - 1) / whole, max((int64_t)a.L / kSegmentMin, (int64_t)1));
        const int64_t rows = (max(a.L, 1) + n - 1) / n;
        p.seg_rows = (int)((rows + chunk - 1) / chunk * chunk);
        n = max((a.L + p.seg_rows - 1) / p.seg_rows, 1);
        p.items = (int)(n * a.S);
        p.slots = n > 1 ? a.T / p.seg_rows + 1 : 0;
    } else {
        // lengths are not known here: segments of what a workgroup has if all rows are shared out
        int64_t rows = max((int64_t)kSegmentMin, (a.T * heads + kFillPacked - 1) / kFillPacked);
        rows = min(rows, (int64_t)max(a.T, 1));
        p.seg_rows = (int)((rows + chunk - 1) / chunk * chunk);
        p.items = a.T / p.seg_rows + a.S;
        p.slots = a.T > p.seg_rows ? a.T / p.seg_rows + 1 : 0;
    }
    return p;
}

size_t aligned(size_t n) { return (n + 255) / 256 * 256; }

struct Space {
    size_t states, dq, dk, dv, all;  // bytes of a set of states, of gradients for each state's head
};
Space space(const AttnArgs& a, const Plan& p, bool bwd) {
    Space s = {};
    s.states = aligned((size_t)p.slots * a.H * a.Dk * a.Dv * 4);
    s.all = s.states * (bwd ? 2 : 1);
    if (bwd) {
        auto part = [&](const HeadsIn& x, int D) { return x.share > 1 ? aligned((size_t)a.T * a.H * D * 4) : 0; };
        s.dq = part(a.q, a.Dk);
        s.dk = part(a.k, a.Dk);
        s.dv = part(a.v, a.Dv);
        s.all += s.dq + s.dk + s.dv;
    }
    return s;
}

// From what the segments add to the states that they begin with.  A workgroup has kPart
// entries of a head's state, of the sequence whose second segment has the slot (cu), or
// of one sequence.  kAhead loads of a thread are under way at a time.
constexpr int kPart = 1024, kAhead = 4;

__global__ __launch_bounds__(256) void k_segments(AttnScan a) {
    const AttnRole& R = a.role[blockIdx.z];
    const int h = blockIdx.y, parts = (a.state + kPart - 1) / kPart;
    const int e0 = (int)(blockIdx.x % parts) * kPart + threadIdx.x;
    int s = blockIdx.x / parts;
    int64_t begin, len;
    if (a.cu) {
        const int64_t slot = s, row = slot * a.seg_rows;
        int lo = 0, n = a.S;
        while (n > 1) {  // the last sequence that begins at or before the slot's row
            const int step = (n + 255) / 256, at = lo + (int)threadIdx.x * step;
            const bool in = (int)threadIdx.x * step < n && min(max(a.cu[at], 0), a.T) <= row;
            const int k = max(__syncthreads_count(in) - 1, 0);
            n = min(step, n - k * step);
            lo += k * step;
        }
        s = lo;
        begin = min(max(a.cu[s], 0), a.T);
        len = min(max(a.cu[s + 1], (int)begin), a.T) - begin;
        if (begin / a.seg_rows != slot - 1) return;
    } else {
        begin = (int64_t)s * a.L;
        len = a.L;
    }
    if (len <= a.seg_rows) return;
    const float rate = a.rate[h];
    const float keep = rate >= 0.f && rate < INFINITY ? (float)exp(-(double)rate * a.seg_rows) : NAN;
    const int n = (int)((len + a.seg_rows - 1) / a.seg_rows);
    const size_t next = (size_t)a.H * a.state;
    float* p = const_cast<float*>(R.seg) + ((size_t)(begin / a.seg_rows + 1) * a.H + h) * a.state + e0;
    const float* x0 = R.x0 ? R.x0 + ((size_t)s * a.H + h) * a.state + e0 : nullptr;
    constexpr int E = kPart / 256;
    float x[E];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = x0 && e0 + e * 256 < a.state ? x0[e * 256] : 0.f;
    for (int seg = 1; seg < n; seg += kAhead) {
        float add[kAhead][E];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) add[k][e] = seg + k < n && e0 + e * 256 < a.state ? p[k * next + e * 256] : 0.f;
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                x[e] = fmaf(keep, x[e], add[k][e]);
                if (seg + k < n && e0 + e * 256 < a.state) p[k * next + e * 256] = x[e];
            }
        p += kAhead * next;
    }
}

// The gradients of shared heads: the sums over the states' heads that read them, of up
// to three tensors.  A thread has V entries of a head, of every so many-th row.
struct ShareArgs {
    struct {
        const float* part;  // [T, heads * share, D]
        void* out;          // [T, heads, D]
        int heads, share, D;
    } of[3];
    int T, S;
    const int* cu;
};
constexpr int kShareRows = 2048;  // workgroups, or rows, that are under way

template <int IO, int V>
__global__ __launch_bounds__(256) void k_share(ShareArgs a) {
    typedef float vec __attribute__((ext_vector_type(V)));
    const auto& o = a.of[blockIdx.z];
    const int rest = a.cu ? min(max(a.cu[a.S], 0), a.T) : a.T;
    const int per = o.D / V, all = o.heads * per;  // vectors of a head, of a row
    const int rows = max(256 / all, 1);            // rows that a workgroup has at a time
    const int e = blockIdx.x * 256 + threadIdx.x % (256 / rows), row = blockIdx.y * rows + threadIdx.x / (256 / rows);
    if (e >= all || (int)threadIdx.x / (256 / rows) >= rows) return;
    const int head = e / per, d = e % per * V, step = gridDim.y * rows;
    const int64_t wide = (int64_t)o.heads * o.D;
    const float* p = o.part + (row * wide + (int64_t)head * o.D) * o.share + d;
    auto* out = static_cast<typename Entry<IO>::T*>(o.out) + row * wide + (int64_t)head * o.D + d;
    for (int t = row; t < a.T; t += step, p += step * wide * o.share, out += step * wide) {
        vec sum = {};
        if (t < rest)
            for (int r = 0; r < o.share; ++r) sum += *reinterpret_cast<const vec*>(p + r * o.D);
#pragma unroll
        for (int k = 0; k < V; ++k) out[k] = Entry<IO>::put(sum[k]);
    }
}

__global__ __launch_bounds__(256) void k_bounds(const int* cu, int S, int T, int* status) {
    bool bad = false;
    for (int s = threadIdx.x; s <= S; s += 256) bad |= s == 0 ? cu[0] != 0 : cu[s] < cu[s - 1];
    bad |= cu[S] > T;
    if (bad) report_index_error(status);
}

hipError_t scan(const AttnScan& a, bool full, bool wide, hipStream_t s) {
    const int Dc = a.role[0].Dc;
    if (Dc <= 64) return launch_attn_scan<64>(a, full, wide, s);
    if (Dc <= 128) return launch_attn_scan<128>(a, full, wide, s);
    return launch_attn_scan<256>(a, full, wide, s);
}
int length_class(int Dc) { return Dc <= 64 ? 0 : Dc <= 128 ? 1 : 2; }

AttnScan scan_args(const AttnArgs& a, const Plan& p) {
    AttnScan n = {};
    n.T = a.T;
    n.S = a.S;
    n.H = a.H;
    n.L = a.L;
    n.io = a.io;
    n.seg_rows = p.seg_rows;
    n.items = p.items;
    n.state = a.Dk * a.Dv;
    n.scale = a.scale;
    n.rate = a.rate;
    n.cu = a.cu;
    n.groups = (int64_t)p.items * a.H;
    return n;
}

void add_role(AttnScan& n, const AttnRole& r, bool wide) {
    AttnRole& to = n.role[n.roles++];
    to = r;
    to.slices = slices(r.Do, wide);
    n.members += to.slices;
    const int64_t row = (int64_t)r.Do * (n.io == kRowBf16 && !r.out32 ? 2 : 4);  // bytes of a head's
    to.past = (int64_t)n.T * n.H * row >= kPast && row % kPiece == 0 && reinterpret_cast<uintptr_t>(r.out) % kPiece == 0;
}

// The states that segments begin with, of the roles in n.
hipError_t begin_segments(const AttnScan& n, const Plan& p, bool wide, hipStream_t s) {
    hipError_t e = scan(n, false, wide, s);
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)((n.cu ? p.slots : n.S) * ((n.state + kPart - 1) / kPart)), n.H, n.roles);
    hipLaunchKernelGGL(k_segments, grid, dim3(256), 0, s, n);
    return hipGetLastError();
}

hipError_t check_bounds(const AttnArgs& a, hipStream_t s) {
    if (!a.cu || !a.status) return hipSuccess;
    hipLaunchKernelGGL(k_bounds, dim3(1), dim3(256), 0, s, a.cu, a.S, a.T, a.status);
    return hipGetLastError();
}

hipError_t add_shared(const AttnArgs& a, float* const (&part)[3], hipStream_t s) {
    ShareArgs n = {};
    int z = 0, most = 0;
    bool four = true;
    auto add = [&](const float* p, void* out, const HeadsIn& x, int D) {
        if (x.share == 1) return;
        n.of[z++] = {p, out, a.H / x.share, x.share, D};
        four = four && D % 4 == 0;
        most = max(most, a.H / x.share * D);
    };
    add(part[0], a.dq, a.q, a.Dk);
    add(part[1], a.dk, a.k, a.Dk);
    add(part[2], a.dv, a.v, a.Dv);
    if (z == 0 || a.T == 0) return hipSuccess;
    n.T = a.T;
    n.S = a.S;
    n.cu = a.cu;
    const int wide = four ? 1024 : 256;
    void (*f)(ShareArgs) = a.io == kRowBf16 ? (four ? k_share<kRowBf16, 4> : k_share<kRowBf16, 1>)
                                            : (four ? k_share<kRowF32, 4> : k_share<kRowF32, 1>);
    hipLaunchKernelGGL(f, dim3((most + wide - 1) / wide, min(a.T, kShareRows), z), dim3(256), 0, s, n);
    return hipGetLastError();
}

}  // namespace

size_t attn_workspace(const AttnArgs& a, bool bwd) { return space(a, plan(a, bwd), bwd).all; }

bool attn_fits(const AttnArgs& a, bool bwd) {
    const Plan p = plan(a, bwd);
    const bool wide = wide_cols(a, bwd);
    const int64_t groups = ((int64_t)p.items * a.H + 7) / 8 * 8, most = 1LL << 32;
    auto fits = [&](int Dc, bool full, int members) { return groups * members * attn_threads(Dc, full, wide) < most; };
    const int k = slices(a.Dk, wide), v = slices(a.Dv, wide);
    if (p.slots) {
        const int64_t parts = ((int64_t)a.Dk * a.Dv + kPart - 1) / kPart;
        if (!fits(a.Dk, false, bwd ? 2 * v : v) || (a.cu ? p.slots : a.S) * parts * a.H * 2 >= (1 << 24)) return false;
    }
    if (!bwd) return fits(a.Dk, true, v);
    if (length_class(a.Dk) == length_class(a.Dv)) return fits(a.Dk, true, 2 * k + v);
    return fits(a.Dv, true, 2 * k) && fits(a.Dk, true, v);
}

hipError_t launch_attn_fwd(const AttnArgs& a, hipStream_t s) {
    const Plan p = plan(a, false);
    const bool wide = wide_cols(a, false);
    hipError_t e = check_bounds(a, s);
    if (e != hipSuccess) return e;
    AttnRole r = {};
    r.q = a.q;
    r.k = a.k;
    r.v = a.v;
    r.out = a.o;
    r.x0 = a.h0;
    r.seg = static_cast<const float*>(a.ws);
    r.fin = a.h_final;
    r.keep = a.h0;
    r.Dc = a.Dk;
    r.Do = a.Dv;
    r.rs = a.Dv;
    r.cs = 1;
    AttnScan n = scan_args(a, p);
    add_role(n, r, wide);
    if (p.slots && (e = begin_segments(n, p, wide, s)) != hipSuccess) return e;
    return scan(n, true, wide, s);
}

hipError_t launch_attn_bwd(const AttnArgs& a, hipStream_t s) {
    const Plan p = plan(a, true);
    const Space sp = space(a, p, true);
    const bool wide = wide_cols(a, true);
    hipError_t e = check_bounds(a, s);
    if (e != hipSuccess) return e;
    char* ws = static_cast<char*>(a.ws);
    float* S = reinterpret_cast<float*>(ws);
    float* G = reinterpret_cast<float*>(ws + sp.states);
    ws += 2 * sp.states;
    float* part[3] = {reinterpret_cast<float*>(ws), reinterpret_cast<float*>(ws + sp.dq), reinterpret_cast<float*>(ws + sp.dq + sp.dk)};
    AttnRole dq = {}, dk = {}, dv = {}, fs = {};
    dq.q = a.dout;
    dq.k = a.v;
    dq.v = a.k;
    dq.out32 = a.q.share > 1;
    dq.out = dq.out32 ? part[0] : a.dq;
    dq.x0 = a.h0;
    dq.seg = S;
    dq.Dc = a.Dv;
    dq.Do = a.Dk;
    dq.rs = 1;
    dq.cs = a.Dv;
    dq.inner = 1;
    dk = dq;
    dk.q = a.v;
    dk.k = a.dout;
    dk.v = a.q;
    dk.out32 = a.k.share > 1;
    dk.out = dk.out32 ? part[1] : a.dk;
    dk.x0 = a.dhf;
    dk.seg = G;
    dk.late = 1;
    dv.q = a.k;
    dv.k = a.q;
    dv.v = a.dout;
    dv.out32 = a.v.share > 1;
    dv.out = dv.out32 ? part[2] : a.dv;
    dv.x0 = a.dhf;
    dv.seg = G;
    dv.fin = a.dh0;
    dv.keep = a.dhf;
    dv.Dc = a.Dk;
    dv.Do = a.Dv;
    dv.rs = a.Dv;
    dv.cs = 1;
    dv.late = 1;
    if (p.slots) {
        fs = dv;  // the forward's states
        fs.k = a.k;
        fs.v = a.v;
        fs.x0 = a.h0;
        fs.seg = S;
        fs.late = 0;
        AttnScan n = scan_args(a, p);
        add_role(n, fs, wide);
        add_role(n, dv, wide);
        if ((e = begin_segments(n, p, wide, s)) != hipSuccess) return e;
    }
    AttnScan n = scan_args(a, p);
    add_role(n, dq, wide);
    add_role(n, dk, wide);
    if (length_class(a.Dk) == length_class(a.Dv)) {
        add_role(n, dv, wide);
    } else {
        AttnScan m = scan_args(a, p);
        add_role(m, dv, wide);
        if ((e = scan(m, true, wide, s)) != hipSuccess) return e;
    }
    if ((e = scan(n, true, wide, s)) != hipSuccess) return e;
    return add_shared(a, part, s);
}

// ---- one token -------------------------------------------------------------------------------------------------------

namespace {

// S' = a S + k v^T, o = scale S'^T q: the state is read and written once, and nothing
// else counts.  TX threads beside each other have V columns each, 256 / TX rows are under way at a time.
template <int IO, int V, int TX>
__global__ __launch_bounds__(256) void k_attn_step(AttnStepArgs a) {
    using En = Entry<IO>;
    using T = typename En::T;
    constexpr int TY = 256 / TX;
    __shared__ float qs[kAttnMaxDim], ks[kAttnMaxDim];
    __shared__ float sum[TY][TX * V + 1];
    const int parts = (a.Dv + TX * V - 1) / (TX * V);
    const int h = blockIdx.x / parts, b = blockIdx.y, tx = threadIdx.x % TX, ty = threadIdx.x / TX;
    const int o = ((int)(blockIdx.x % parts) * TX + tx) * V;
    int slot = b;
    if (a.slots) {
        slot = a.slots[b];
        if (slot < 0 || slot >= a.pool) {
            if (slot >= a.pool && threadIdx.x == 0) report_index_error(a.status);
            return;
        }
    }
    auto row = [&](const HeadsIn& r) { return static_cast<const T*>(r.p) + (int64_t)b * r.ld + (int64_t)(h / r.share) * r.hs; };
    for (int c = threadIdx.x; c < a.Dk; c += 256) {
        qs[c] = En::get(row(a.q)[c]);
        ks[c] = En::get(row(a.k)[c]);
    }
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = o + e < a.Dv ? En::get(row(a.v)[o + e]) : 0.f;
    const float rate = a.rate[h];
    const float decay = rate >= 0.f && rate < INFINITY ? (float)exp(-(double)rate) : NAN;
    // the first row that names a slot has it; others of the same batch are refused
    bool again = false;
    if (a.slots)
        for (int k = threadIdx.x; k < b; k += 256) again |= a.slots[k] == slot;
    if (__syncthreads_or(again)) {
        if (threadIdx.x == 0) report_index_error(a.status);
        return;
    }
    const size_t at = ((size_t)slot * a.H + h) * a.Dk * a.Dv + o;
    typedef float vec __attribute__((ext_vector_type(V)));
    float acc[V] = {};
    if (o < a.Dv) {
#pragma unroll 4
        for (int c = ty; c < a.Dk; c += TY) {
            vec s = *reinterpret_cast<const vec*>(a.h_in + at + (size_t)c * a.Dv);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                s[e] = fmaf(decay, s[e], ks[c] * v[e]);
                acc[e] = fmaf(qs[c], s[e], acc[e]);
            }
            *reinterpret_cast<vec*>(a.h_out + at + (size_t)c * a.Dv) = s;
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) sum[ty][tx * V + e] = acc[e];
    __syncthreads();
    const int c = threadIdx.x, col = (int)(blockIdx.x % parts) * TX * V + c;
    if (c < TX * V && col < a.Dv) {
        float x = 0.f;
#pragma unroll
        for (int r = 0; r < TY; ++r) x += sum[r][c];
        static_cast<T*>(a.o)[((size_t)b * a.H + h) * a.Dv + col] = En::put(a.scale * x);
    }
}

}  // namespace

bool attn_step_fits(int B, int H, int Dv) { return (int64_t)B * H * ((Dv + 15) / 16) < (1 << 24); }

hipError_t launch_attn_step(const AttnStepArgs& a, hipStream_t s) {
    const bool four = a.Dv % 4 == 0 && reinterpret_cast<uintptr_t>(a.h_in) % 16 == 0 && reinterpret_cast<uintptr_t>(a.h_out) % 16 == 0;
    const bool b = a.io == kRowBf16;
    const int cols = four ? 32 : 16;
    void (*f)(AttnStepArgs) = four ? (b ? k_attn_step<kRowBf16, 4, 8> : k_attn_step<kRowF32, 4, 8>)
                                   : (b ? k_attn_step<kRowBf16, 1, 16> : k_attn_step<kRowF32, 1, 16>);
    hipLaunchKernelGGL(f, dim3(a.H * ((a.Dv + cols - 1) / cols), a.B), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace pdssm

// pdssm_attn.h -- host-side launch interface of linear attention with a decay
// for each head (pdssm_attn.hip).  Not installed; not part of the ABI.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "pdssm_kept.h"

namespace pdssm {

// A tensor of heads' rows: entry (t, head, d) at p + t * ld + head * hs + d; state h reads head h / share.
struct HeadsIn {
    const void* p;
    int64_t ld, hs;
    int share;
};

constexpr int kAttnMaxDim = 256;  // entries of a head's row

struct AttnArgs {
    int T, S, H, Dk, Dv;
    int L;             // rows of a sequence where cu is null
    int io;            // kRowF32, kRowBf16
    float scale;
    HeadsIn q, k, v;
    const float* rate;  // [H]
    const int* cu;      // [S + 1], or null: S sequences of L rows (which may be 0)
    const float* h0;    // [S, H, Dk, Dv] or null
    int* status;
    void* ws;
    // forward
    void* o;         // [T, H, Dv]
    float* h_final;  // [S, H, Dk, Dv] or null
    // backward
    HeadsIn dout;       // [T, H, Dv]
    const float* dhf;   // [S, H, Dk, Dv] or null
    void *dq, *dk, *dv; // [T, H / share, D]
    float* dh0;         // [S, H, Dk, Dv] or null
};
size_t attn_workspace(const AttnArgs& a, bool bwd);
// Whether the launches of these sizes stay below 2^32 threads along an axis of the grid.
bool attn_fits(const AttnArgs& a, bool bwd);
hipError_t launch_attn_fwd(const AttnArgs& a, hipStream_t s);
hipError_t launch_attn_bwd(const AttnArgs& a, hipStream_t s);

// One row for each of B sequences whose states are entries of a pool.
struct AttnStepArgs {
    int B, pool, H, Dk, Dv;
    int io;
    float scale;
    HeadsIn q, k, v;
    const float* rate;  // [H]
    const int* slots;   // [B] or null (row b is state b)
    const float* h_in;  // [pool, H, Dk, Dv]
    float* h_out;       // [pool, H, Dk, Dv], may be h_in
    void* o;            // [B, H, Dv]
    int* status;
};
bool attn_step_fits(int B, int H, int Dv);
hipError_t launch_attn_step(const AttnStepArgs& a, hipStream_t s);

// What the launches of pdssm_attn.hip hand to the kernels of one row length
// (pdssm_attn_scan.hip): sums over earlier (reverse: later) rows j and the row itself,
//   out_i = sa * sum_j a^|i-j| (q_i . k_j) v_j  +  what the state x0 hands on.
// Forward (late = 0) a row reads the state behind its own step, so the i-th row
// has sa * a^(i+1) q_i^T x0 of it.  In reverse (late = 1), where the state is the
// gradient that reaches a step, the i-th row from the end has a^i q_i^T x0, and
// sa is the rows' part of the state.
struct AttnRole {
    HeadsIn q, k, v;
    void* out;            // rows [T, H, Do]
    int out32;            // out is fp32, whatever the rows are
    const float* x0;      // [S, H, ..] or null: states that the sequences begin with
    const float* seg;     // states that the segments after the first begin with, [slot, H, ..]; state-only: written
    float* fin;           // [S, H, ..] or null
    const float* keep;    // what fin has for a sequence without rows (null: zeros)
    int Dc, Do;           // entries of q and k rows, of v rows
    int rs, cs;           // entry (c, o) of a state at c * rs + o * cs
    int late;
    int inner;            // dq and dk: rows alone are made of the states
    int past;             // out goes past the caches: large, and its heads' rows are whole pieces
    int slices;           // workgroups that share the Do columns
};
struct AttnScan {
    AttnRole role[3];
    int roles;
    int T, S, H, L, io;
    int seg_rows;        // rows of a segment, a multiple of the chunk
    int items;           // segments at most, over all sequences
    int state;           // Dk * Dv
    float scale;
    const float* rate;
    const int* cu;
    int members;         // workgroups of a head's segment, over all roles
    int64_t groups;      // items * H
};

// Threads of a workgroup of the scan of rows of up to Dc entries.
constexpr int attn_threads(int Dc, bool full, bool wide) { return wide && (!full || Dc > 128) ? 512 : 256; }

// States only (full = 0): what the rows of each segment but the last add.
template <int DC>
hipError_t launch_attn_scan(const AttnScan& a, bool full, bool wide, hipStream_t s);

}  // namespace pdssm

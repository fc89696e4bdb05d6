// pdssm_gated.h -- host-side launch interface of the gated linear recurrence
// (pdssm_gated.hip).  Not installed; not part of the ABI.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "pdssm_kept.h"

namespace pdssm {

constexpr int kGatedChunk = 128;  // rows between two saved states
struct GatedArgs {
    int T, C;
    // one word: with a scalar register more than 80 the forward has three workgroups
    // on a CU in place of four (54 -> 57 us at B16 L2048 C1024 bf16)
    unsigned S : 31;
    unsigned zero_rest : 1;  // outputs of rows behind the last sequence are zero; else they are not written
    int L;               // rows of a sequence where cu is null
    int io;              // format of y, dy, dx, dga, dgi; and of x, ga, gi unless kept
    int kept;            // backward: x, ga, gi are in the 8-bit form
    RowsIn x, ga, gi;
    const float* rate;   // [C]
    const int* cu;       // [S + 1], or null: S sequences of L rows (which may be 0)
    const float* h0;     // [S, C] or null
    int* status;
    void* ws;
    // forward
    void* y;             // [T, C]
    float* h_final;      // [S, C] or null
    float* saved;        // [ceil(T / kGatedChunk), C]; forward: or null
    int8_t* q[3];        // x, ga, gi in the 8-bit form, or null
    int8_t* e[3];
    // backward
    RowsIn dy;
    const float* dhf;    // [S, C] or null
    void* d[3];          // dx, dga, dgi: rows of ldd entries
    int64_t ldd;
    float* drate;        // [C] or null
    float* dh0;          // [S, C] or null
};

// Workspace bytes of a forward (bwd = false) or backward pass.
size_t gated_workspace(int T, int C, bool bwd);

hipError_t launch_gated_fwd(const GatedArgs& a, hipStream_t s);
hipError_t launch_gated_bwd(const GatedArgs& a, hipStream_t s);

// One row for each of B sequences whose states are rows of a pool.
struct GatedStepArgs {
    int B, C, pool;
    int io;
    RowsIn x, ga, gi;
    const float* rate;
    const int* slots;    // [B] or null (row b is state b)
    const float* h_in;   // [pool, C]
    float* h_out;        // [pool, C], may be h_in
    void* y;             // [B, C]
    int* status;
};
hipError_t launch_gated_step(const GatedStepArgs& a, hipStream_t s);

}  // namespace pdssm

// pdssm_norm.h -- host-side launch interface of the group norm of rows
// (pdssm_norm.hip).  Not installed; not part of the ABI.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "pdssm_kept.h"

namespace pdssm {

struct NormArgs {
    int T, C, G;
    int io;     // kRowF32, kRowBf16
    int silu;   // the activation is silu, else none
    float eps;
    RowsIn x, gate;  // gate.p null: the activation stands behind the norm
    const float* w;  // [C] or null: ones
    const float* b;  // [C] or null: zeros
    void* y;         // [T, C]
    // backward
    RowsIn dy;
    void* dx;        // [T, C]
    void* dgate;     // [T, C], with a gate
    float* dw;       // [C] or null
    float* db;       // [C] or null
    float* part;     // sums of the rows of a block, [blocks, 2, C]
    // filled in by the launches
    int team;        // lanes that share a group's row, a power of two up to 64
    int blocks;      // blocks of rows: one wave's (or workgroup's) rows of some groups
};
size_t norm_workspace(int T, int C);
bool norm_fits(int T, int C, int G);
hipError_t launch_norm_fwd(NormArgs a, hipStream_t s);
hipError_t launch_norm_bwd(NormArgs a, hipStream_t s);

}  // namespace pdssm

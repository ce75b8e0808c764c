// rotary.hpp -- arguments of the rotation kernels (k_rotary.hip).
#pragma once

#include "common.hpp"

namespace nmg_internal {

// One matrix of heads of a call
struct RotaryRows {
    const void *X;
    void *Y;
    int64_t ldx, ldy;
    const float *weight;  // of the norm; NULL: ones
    int32_t heads;
};

struct RotaryArgs {
    RotaryRows part[2];  // queries and keys; heads 0: absent
    int32_t N, D, R;
    int32_t interleaved;
    int64_t length;
    const float *table;
    const int32_t *positions;
    float eps;
    // the plan of the launch
    int32_t lanes;    // threads of a workgroup along the tokens
    int32_t blocks;   // workgroups along the tokens
    int32_t run;      // heads a workgroup takes one after another
    int32_t groups0;  // runs of part[0]
};

nmg_status launch_rotary(nmg_dtype dtype, const RotaryArgs &a, bool norm, hipStream_t stream);

struct RotaryTableArgs {
    int32_t half;         // R / 2
    int64_t length;
    double log_base;      // of the (NTK-changed) base
    int32_t scaling;
    double factor, original, slow, fast, magnitude;
    float *table;
};
nmg_status launch_rotary_table(const RotaryTableArgs &a, hipStream_t stream);

}  // namespace nmg_internal

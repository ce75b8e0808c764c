// norm.hpp -- arguments of the residual norm's launch (k_norm.hip).
#pragma once

#include "common.hpp"

namespace nmg_internal {

struct NormArgs {
    const void *A, *G, *R;               // G, R may be NULL
    void *H, *Y;                         // either may be NULL
    int64_t lda, ldg, ldr, ldh, ldy;
    int32_t M, N;
    float scale;
    nmg_norm after, before;
    int32_t lanes;                       // the plan: threads of a row in a tile
};

nmg_status launch_residual_norm(nmg_dtype dtype, NormArgs a, hipStream_t stream);

}  // namespace nmg_internal

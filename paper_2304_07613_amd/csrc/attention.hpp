// attention.hpp -- shared by the attention kernels and their C ABI: arguments
// of one call, and the walk from a workgroup's number to the sequence and the
// query rows it works on.
//
// The rows of a (sequence, key head) are its queries in every query head that
// shares the key head: with n query columns and S = heads / kv_heads, row
// r = g n + t is query column t of head kv_head * S + g.  They all meet the same
// keys, so they are tiled together.
#pragma once

#include "common.hpp"

namespace nmg_internal {

struct AttnArgs {
    const void *Q, *K, *V;
    void *O;
    int64_t ldq, ldk, ldv, ldo, ldtree;
    const int32_t *q_offsets, *kv_begin, *kv_end;
    const uint8_t *key_mask, *tree;  // at most one of the two
    int32_t Nq, Nk;                  // columns
    int32_t width;                   // of the tree
    int32_t sequences, kv_heads, share, D;
    float scale;
};

nmg_status launch_attention(nmg_dtype dtype, const AttnArgs &a, void *workspace,
                            int64_t workspace_bytes, hipStream_t stream);
int64_t attention_workspace_bytes(nmg_dtype dtype, const AttnArgs &a);

}  // namespace nmg_internal

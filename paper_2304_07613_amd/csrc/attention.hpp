// attention.hpp -- shared by the attention kernels and their C ABI: arguments
// of one call and its plan.
//
// The rows of a (sequence, key head) are its queries in every query head that
// shares the key head: with n query columns and `share` = heads / kv_heads, row
// r = g n + t is query column t of head kv_head * share + g.  They all meet the
// same keys, so they are tiled together: a tile is `tile_rows` consecutive rows
// of one (sequence, key head).
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
    // the plan of the launch
    int32_t tiles;                   // row tiles of one key head, at most
    int32_t splits;                  // parts of every key range
    int32_t join_rows;               // splits > 1: rows of a head a joining workgroup takes
    int32_t align;                   // key tiles start at a multiple of this column
    float *part;                     // splits > 1: sums, maxima and totals of every part
};

// How rows of K and V are read: one buffer a head; 64-bit addresses, for heads that
// span 2^31 bytes or more; the same for binary16 rows that do not all start on 4 bytes
enum AttnRows { kAttnNarrow, kAttnWide, kAttnShift };

// Workgroups that share key tiles (128 rows) or split them (32 rows)
nmg_status launch_attention_f16(const AttnArgs &a, bool shared, AttnRows how, hipStream_t stream);
nmg_status launch_attention_f32(const AttnArgs &a, bool shared, AttnRows how, hipStream_t stream);

nmg_status launch_attention(nmg_dtype dtype, const AttnArgs &a, void *workspace,
                            int64_t workspace_bytes, hipStream_t stream);
int64_t attention_workspace_bytes(nmg_dtype dtype, const AttnArgs &a);

constexpr int kAttnMostSplits = 64;   // parts of a key range
constexpr int kAttnSharedRows = 128;  // rows of a tile whose waves share key tiles
constexpr int kAttnSplitRows = 32;    // ... whose waves split the keys

// Rows of a head padded to whole matrix instructions
inline int attn_padded_dim(int D) {
    return D <= 32 ? 32 : D <= 64 ? 64 : D <= 96 ? 96 : D <= 128 ? 128 : 256;
}

// Waves of a workgroup that splits the keys: as many as 128 KB hold tiles of
constexpr int attn_split_waves(int padded_dim) {
    return padded_dim <= 64 ? 8 : padded_dim <= 128 ? 4 : 2;
}

}  // namespace nmg_internal

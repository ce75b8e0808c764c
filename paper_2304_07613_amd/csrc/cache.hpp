// cache.hpp -- shared by the kernels of the 8-bit cache (include/nmg.h): where its
// tokens lie, how values become codes, and the arguments of the launches.
//
// Position p of a sequence with n kept tokens: p < n - n % block lies in page
// table[p / block], every later one (open tokens: kept ones of the last block,
// drafted ones) in slot p % room of the sequence's ring.  room is a multiple of block,
// so an aligned block's slots follow one another.
#pragma once

#include "common.hpp"

namespace nmg_internal {

// What the kernels read of a cache, by value
struct CacheView {
    uint8_t *k_pages, *v_pages;
    float *k_scales, *v_scales;
    void *k_open, *v_open;
    int32_t *table, *references;
    int32_t layers, heads, D, D16;   // D16: D rounded up to 16, the width of a key's row
    int32_t block, pages, sequences, row, room;
};

// A device-side length, cut to what the table can hold
__device__ __forceinline__ int cache_length(const CacheView &c, const int32_t *lengths, int b) {
    const int n = lengths[b], most = c.row * c.block + c.block - 1;
    return n < 0 ? 0 : n > most ? most : n;
}

constexpr int kSlotListSize = 128;   // sequences of one launch of fork and free
struct SlotList {
    int32_t from[kSlotListSize], to[kSlotListSize];
};

struct CacheAttnArgs {
    CacheView c;
    int32_t layer, share;            // query heads of a key head
    const int32_t *q_offsets, *lengths;
    const void *Q;
    void *O;
    int64_t ldq, ldo;
    int32_t Nq;
    const uint8_t *tree;             // NULL: every drafted token sees those before it
    int64_t ldtree;
    int32_t width;
    float scale;
    // the plan of the launch
    int32_t slots;                   // row tiles of all sequences, at most
    int32_t target;                  // workgroups that splitting the keys aims at, 0: no splitting
    int64_t part_count;              // parts whose results there is room for
    float *part;
};

// Rows of a workgroup: 16 or 32 that its four waves split the keys of; 64 (head_dim > 128) or
// 128, a quarter for each wave (binary16)
enum CacheAttnRows { kRows16 = 16, kRows32 = 32, kRows64 = 64, kRows128 = 128 };

nmg_status launch_cache_append(nmg_dtype dtype, const CacheView &c, int32_t layer,
                               const int32_t *q_offsets, const int32_t *lengths, const void *K,
                               int64_t ldk, const void *V, int64_t ldv, int32_t N, hipStream_t stream);
nmg_status launch_cache_commit(nmg_dtype dtype, nmg_cache_format format, const CacheView &c,
                               const int32_t *lengths, const int32_t *kept_offsets,
                               const int32_t *kept, int32_t n_kept, int32_t *new_lengths,
                               hipStream_t stream);
nmg_status launch_cache_reserve(const CacheView &c, const int32_t *lengths, const int32_t *tokens,
                                int32_t *missing, hipStream_t stream);
nmg_status launch_cache_fork(nmg_dtype dtype, const CacheView &c, int32_t *lengths, const SlotList &list,
                             int32_t count, hipStream_t stream);
nmg_status launch_cache_free(const CacheView &c, int32_t *lengths, const SlotList &list, int32_t count,
                             hipStream_t stream);
nmg_status launch_cache_compact(const CacheView &c, int32_t *table_out, int32_t *references_out,
                                int32_t *live, int32_t *workspace, hipStream_t stream);
// int32 values of launch_cache_compact's workspace
inline int64_t cache_compact_words(const CacheView &c) { return 4 * (int64_t)c.pages + 1; }

nmg_status launch_cache_attention(nmg_dtype dtype, nmg_cache_format format, CacheAttnArgs a,
                                  int64_t longest, void *workspace, int64_t workspace_bytes,
                                  hipStream_t stream);
int64_t cache_attention_workspace(nmg_dtype dtype, const CacheAttnArgs &a, int64_t longest);

}  // namespace nmg_internal

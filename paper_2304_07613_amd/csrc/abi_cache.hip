// abi_cache.hip -- the C ABI of the 8-bit cache and of the residual norm
// (include/nmg.h): host-side validation and dispatch to the launchers.
#include <math.h>

#include <vector>

#include "cache.hpp"
#include "norm.hpp"

using namespace nmg_internal;

namespace {

bool dtype_ok(nmg_dtype d) { return d == NMG_F32 || d == NMG_F16; }

// The cache's sizes; `view` without the pointers' checks
nmg_status check_sizes(const nmg_cache *c, CacheView *v) {
    if (!c) return NMG_ERR_NULL;
    if (!dtype_ok(c->dtype)) return NMG_ERR_DTYPE;
    if (c->format != NMG_CACHE_E4M3 && c->format != NMG_CACHE_INT8) return NMG_ERR_PARAM;
    if (c->layers < 1 || c->kv_heads < 1 || c->head_dim < 1 || c->pages < 1 || c->sequences < 1 ||
        c->row < 1 || c->room < 1)
        return NMG_ERR_PARAM;
    if (c->head_dim > 256 || (c->block != 64 && c->block != 128)) return NMG_ERR_UNSUPPORTED;
    if (c->room % c->block) return NMG_ERR_PARAM;
    // positions and their slots in 31 bits, rows of heads in 31 bits, grids
    if (((int64_t)c->row + 1) * c->block + c->room > INT32_MAX) return NMG_ERR_UNSUPPORTED;
    if ((int64_t)c->kv_heads * c->head_dim > INT32_MAX) return NMG_ERR_PARAM;
    if (2 * (int64_t)c->layers * c->kv_heads > 65535 ||
        (int64_t)c->kv_heads * ((c->head_dim + 63) / 64) > 65535)
        return NMG_ERR_UNSUPPORTED;
    if ((int64_t)c->sequences * kBlock >= ((int64_t)1 << 32)) return NMG_ERR_UNSUPPORTED;
    // pages that sequences ask for are counted in 31 bits
    if ((int64_t)c->sequences * c->row > INT32_MAX) return NMG_ERR_UNSUPPORTED;
    *v = CacheView{static_cast<uint8_t *>(c->k_pages), static_cast<uint8_t *>(c->v_pages), c->k_scales,
                   c->v_scales, c->k_open, c->v_open, c->table, c->references,
                   c->layers, c->kv_heads, c->head_dim, (c->head_dim + 15) / 16 * 16,
                   c->block, c->pages, c->sequences, c->row, c->room};
    return NMG_OK;
}

nmg_status check_cache(const nmg_cache *c, CacheView *v) {
    const nmg_status st = check_sizes(c, v);
    if (st != NMG_OK) return st;
    if (!c->k_pages || !c->v_pages || !c->k_scales || !c->v_scales || !c->k_open || !c->v_open ||
        !c->table || !c->references)
        return NMG_ERR_NULL;
    if (!aligned(c->k_pages, 16) || !aligned(c->v_pages, 16) || !aligned(c->k_open, 16) ||
        !aligned(c->v_open, 16) || !aligned(c->k_scales, 4) || !aligned(c->v_scales, 4) ||
        !aligned(c->table, 4) || !aligned(c->references, 4))
        return NMG_ERR_ALIGN;
    return NMG_OK;
}

nmg_status check_ints(const int32_t *p) {
    return !p ? NMG_ERR_NULL : !aligned(p, 4) ? NMG_ERR_ALIGN : NMG_OK;
}

// A list of sequences on the host: each in range and once
nmg_status check_list(const int32_t *list, int32_t count, int32_t sequences, std::vector<uint8_t> *seen) {
    for (int32_t i = 0; i < count; ++i) {
        if (list[i] < 0 || list[i] >= sequences) return NMG_ERR_PARAM;
        if (seen) {
            if ((*seen)[(size_t)list[i]]) return NMG_ERR_PARAM;
            (*seen)[(size_t)list[i]] = 1;
        }
    }
    return NMG_OK;
}

nmg_status attention_args(const nmg_cache *c, int32_t heads, int64_t Nq, int64_t longest, CacheAttnArgs *a) {
    const nmg_status st = check_sizes(c, &a->c);
    if (st != NMG_OK) return st;
    if (heads < 1 || heads % c->kv_heads || Nq < 1 || Nq > INT32_MAX || longest < 0) return NMG_ERR_PARAM;
    if (Nq * (heads / c->kv_heads) > INT32_MAX || (int64_t)heads * c->head_dim > INT32_MAX)
        return NMG_ERR_UNSUPPORTED;
    a->share = heads / c->kv_heads;
    a->Nq = (int32_t)Nq;
    return NMG_OK;
}

int64_t keys_of(const nmg_cache *c, int64_t longest) {
    const int64_t most = (int64_t)c->row * c->block + c->block - 1;
    return longest == 0 || longest > most ? most : longest;
}

nmg_status check_norm(const nmg_norm &n) {
    if (n.kind != NMG_NORM_NONE && n.kind != NMG_NORM_RMS && n.kind != NMG_NORM_LAYER) return NMG_ERR_PARAM;
    if (!(n.eps >= 0.f) || !isfinite(n.eps)) return NMG_ERR_PARAM;
    if ((n.weight && !aligned(n.weight, 4)) || (n.bias && !aligned(n.bias, 4))) return NMG_ERR_ALIGN;
    return NMG_OK;
}

}  // namespace

extern "C" {

nmg_status nmg_cache_append(const nmg_cache *cache, int32_t layer, const int32_t *q_offsets,
                            const int32_t *lengths, const void *K, int64_t ldk, const void *V,
                            int64_t ldv, int64_t N, hipStream_t stream) {
    CacheView v;
    nmg_status st = check_cache(cache, &v);
    if (st != NMG_OK) return st;
    if (layer < 0 || layer >= cache->layers || N < 1 || N > INT32_MAX) return NMG_ERR_PARAM;
    if (!K || !V) return NMG_ERR_NULL;
    if ((st = check_ints(q_offsets)) != NMG_OK || (st = check_ints(lengths)) != NMG_OK) return st;
    if (ldk < N || ldv < N) return NMG_ERR_PARAM;
    const size_t es = elem_size(cache->dtype);
    if (!aligned(K, es) || !aligned(V, es)) return NMG_ERR_ALIGN;
    if ((N + 63) / 64 * kBlock >= ((int64_t)1 << 32)) return NMG_ERR_UNSUPPORTED;
    prelaunch();
    return launch_cache_append(cache->dtype, v, layer, q_offsets, lengths, K, ldk, V, ldv, (int32_t)N,
                               stream);
}

int64_t nmg_cache_attention_workspace_bytes(const nmg_cache *cache, int32_t heads, int64_t Nq,
                                            int64_t longest) {
    CacheAttnArgs a = {};
    if (attention_args(cache, heads, Nq, longest, &a) != NMG_OK) return -1;
    return cache_attention_workspace(cache->dtype, a, keys_of(cache, longest));
}

nmg_status nmg_cache_attention(const nmg_cache *cache, int32_t layer, int32_t heads,
                               const int32_t *q_offsets, const int32_t *lengths, const void *Q,
                               int64_t ldq, int64_t Nq, const uint8_t *tree, int64_t ldtree,
                               int64_t width, int64_t longest, float scale, void *O, int64_t ldo,
                               void *workspace, int64_t workspace_bytes, hipStream_t stream) {
    CacheAttnArgs a = {};
    nmg_status st = check_cache(cache, &a.c);
    if (st != NMG_OK || (st = attention_args(cache, heads, Nq, longest, &a)) != NMG_OK) return st;
    if (layer < 0 || layer >= cache->layers) return NMG_ERR_PARAM;
    if (!Q || !O) return NMG_ERR_NULL;
    if ((st = check_ints(q_offsets)) != NMG_OK || (st = check_ints(lengths)) != NMG_OK) return st;
    if (ldq < Nq || ldo < Nq || !(scale > 0.f) || !isfinite(scale) || workspace_bytes < 0)
        return NMG_ERR_PARAM;
    if (tree && (width < 1 || ldtree < width || width > INT32_MAX)) return NMG_ERR_PARAM;
    const size_t es = elem_size(cache->dtype);
    if (!aligned(Q, es) || !aligned(O, es) || (workspace && !aligned(workspace, 256))) return NMG_ERR_ALIGN;
    a.layer = layer;
    a.q_offsets = q_offsets;
    a.lengths = lengths;
    a.Q = Q;
    a.O = O;
    a.ldq = ldq;
    a.ldo = ldo;
    a.tree = tree;
    a.ldtree = ldtree;
    a.width = (int32_t)width;
    a.scale = scale;
    prelaunch();
    return launch_cache_attention(cache->dtype, cache->format, a, keys_of(cache, longest), workspace,
                                  workspace_bytes, stream);
}

nmg_status nmg_cache_commit(const nmg_cache *cache, const int32_t *lengths, const int32_t *kept_offsets,
                            const int32_t *kept, int64_t n_kept, int32_t *new_lengths,
                            hipStream_t stream) {
    CacheView v;
    nmg_status st = check_cache(cache, &v);
    if (st != NMG_OK) return st;
    if ((st = check_ints(lengths)) != NMG_OK || (st = check_ints(kept_offsets)) != NMG_OK ||
        (st = check_ints(new_lengths)) != NMG_OK)
        return st;
    if (new_lengths == lengths || n_kept < 0 || n_kept > INT32_MAX) return NMG_ERR_PARAM;
    if (kept && !aligned(kept, 4)) return NMG_ERR_ALIGN;
    prelaunch();
    return launch_cache_commit(cache->dtype, cache->format, v, lengths, kept_offsets, kept,
                               (int32_t)n_kept, new_lengths, stream);
}

nmg_status nmg_cache_reserve(const nmg_cache *cache, const int32_t *lengths, const int32_t *tokens,
                             int32_t *missing, hipStream_t stream) {
    CacheView v;
    nmg_status st = check_cache(cache, &v);
    if (st != NMG_OK) return st;
    if ((st = check_ints(lengths)) != NMG_OK || (st = check_ints(tokens)) != NMG_OK ||
        (st = check_ints(missing)) != NMG_OK)
        return st;
    prelaunch();
    return launch_cache_reserve(v, lengths, tokens, missing, stream);
}

nmg_status nmg_cache_fork(const nmg_cache *cache, int32_t *lengths, int32_t count, const int32_t *from,
                          const int32_t *to, hipStream_t stream) {
    CacheView v;
    nmg_status st = check_cache(cache, &v);
    if (st != NMG_OK) return st;
    if ((st = check_ints(lengths)) != NMG_OK) return st;
    if (count < 0 || count > cache->sequences) return NMG_ERR_PARAM;
    if (count == 0) return NMG_OK;
    if (!from || !to) return NMG_ERR_NULL;
    try {
        std::vector<uint8_t> target((size_t)cache->sequences);
        if ((st = check_list(to, count, cache->sequences, &target)) != NMG_OK ||
            (st = check_list(from, count, cache->sequences, nullptr)) != NMG_OK)
            return st;
        for (int32_t i = 0; i < count; ++i)
            if (target[(size_t)from[i]]) return NMG_ERR_PARAM;
    } catch (...) {
        return NMG_ERR_CAPACITY;
    }
    prelaunch();
    for (int32_t i = 0; i < count; i += kSlotListSize) {
        SlotList list;
        const int32_t n = std::min(count - i, kSlotListSize);
        std::copy(from + i, from + i + n, list.from);
        std::copy(to + i, to + i + n, list.to);
        if ((st = launch_cache_fork(cache->dtype, v, lengths, list, n, stream)) != NMG_OK) return st;
    }
    return NMG_OK;
}

nmg_status nmg_cache_free(const nmg_cache *cache, int32_t *lengths, int32_t count, const int32_t *which,
                          hipStream_t stream) {
    CacheView v;
    nmg_status st = check_cache(cache, &v);
    if (st != NMG_OK) return st;
    if ((st = check_ints(lengths)) != NMG_OK) return st;
    if (count < 0 || count > cache->sequences) return NMG_ERR_PARAM;
    if (count == 0) return NMG_OK;
    if (!which) return NMG_ERR_NULL;
    try {
        std::vector<uint8_t> seen((size_t)cache->sequences);
        if ((st = check_list(which, count, cache->sequences, &seen)) != NMG_OK) return st;
    } catch (...) {
        return NMG_ERR_CAPACITY;
    }
    prelaunch();
    for (int32_t i = 0; i < count; i += kSlotListSize) {
        SlotList list = {};
        const int32_t n = std::min(count - i, kSlotListSize);
        std::copy(which + i, which + i + n, list.to);
        if ((st = launch_cache_free(v, lengths, list, n, stream)) != NMG_OK) return st;
    }
    return NMG_OK;
}

int64_t nmg_cache_compact_workspace_bytes(const nmg_cache *cache) {
    CacheView v;
    return check_sizes(cache, &v) == NMG_OK ? 4 * cache_compact_words(v) : -1;
}

nmg_status nmg_cache_compact(const nmg_cache *cache, int32_t *table, int32_t *references, int32_t *live,
                             void *workspace, int64_t workspace_bytes, hipStream_t stream) {
    CacheView v;
    nmg_status st = check_cache(cache, &v);
    if (st != NMG_OK) return st;
    if ((st = check_ints(table)) != NMG_OK || (st = check_ints(references)) != NMG_OK ||
        (st = check_ints(live)) != NMG_OK)
        return st;
    if (!workspace) return NMG_ERR_NULL;
    if (!aligned(workspace, 256)) return NMG_ERR_ALIGN;
    if (workspace_bytes < 4 * cache_compact_words(v)) return NMG_ERR_CAPACITY;
    prelaunch();
    return launch_cache_compact(v, table, references, live, static_cast<int32_t *>(workspace), stream);
}

nmg_status nmg_residual_norm(nmg_dtype dtype, int64_t M, int64_t N, const void *A, int64_t lda,
                             const nmg_norm *after, const void *G, int64_t ldg, float scale,
                             const void *R, int64_t ldr, const nmg_norm *before, void *H, int64_t ldh,
                             void *Y, int64_t ldy, hipStream_t stream) {
    if (!dtype_ok(dtype)) return NMG_ERR_DTYPE;
    if (!A || (!H && !Y)) return NMG_ERR_NULL;
    if (M < 1 || M > INT32_MAX || N < 1 || N > INT32_MAX || !isfinite(scale)) return NMG_ERR_PARAM;
    NormArgs a = {};
    if (after) a.after = *after;
    if (before) a.before = *before;
    nmg_status st;
    if ((st = check_norm(a.after)) != NMG_OK || (st = check_norm(a.before)) != NMG_OK) return st;
    if (lda < N || (G && ldg < N) || (R && ldr < N) || (H && ldh < N) || (Y && ldy < N))
        return NMG_ERR_PARAM;
    // in place: an output over an input has the input's rows, and the outputs are two
    const void *in[3] = {A, G, R};
    const int64_t ld[3] = {lda, ldg, ldr};
    for (int i = 0; i < 3; ++i)
        if (in[i] && ((in[i] == H && ld[i] != ldh) || (in[i] == Y && ld[i] != ldy))) return NMG_ERR_PARAM;
    if (H && H == Y) return NMG_ERR_PARAM;
    const size_t es = elem_size(dtype);
    if (!aligned(A, es) || !aligned(G, es) || !aligned(R, es) || !aligned(H, es) || !aligned(Y, es))
        return NMG_ERR_ALIGN;
    a.A = A;
    a.G = G;
    a.R = R;
    a.H = H;
    a.Y = Y;
    a.lda = lda;
    a.ldg = ldg;
    a.ldr = ldr;
    a.ldh = ldh;
    a.ldy = ldy;
    a.M = (int32_t)M;
    a.N = (int32_t)N;
    a.scale = scale;
    prelaunch();
    return launch_residual_norm(dtype, a, stream);
}

}  // extern "C"

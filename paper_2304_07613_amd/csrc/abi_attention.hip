// abi_attention.hip -- the C ABI of the attention operators (include/nmg.h):
// host-side validation and dispatch to the launchers.
#include <math.h>

#include "attention.hpp"
#include "rotary.hpp"

using namespace nmg_internal;

namespace {

bool dtype_ok(nmg_dtype d) { return d == NMG_F32 || d == NMG_F16; }

// Rows of one matrix: the launchers take row counts and column counts in 32 bits
bool rows_ok(int64_t heads, int64_t dim) {
    return heads >= 1 && dim >= 1 && heads * dim <= INT32_MAX;
}

nmg_status check_rotary(const nmg_rotary_desc *r, int32_t D) {
    if (!r) return NMG_ERR_NULL;
    if (r->dim < 0 || r->dim % 2 || r->dim > D) return NMG_ERR_PARAM;
    if (r->pairs != NMG_ROTARY_HALF && r->pairs != NMG_ROTARY_INTERLEAVED) return NMG_ERR_PARAM;
    if (r->dim == 0) return NMG_OK;
    if (r->length < 1 || r->length > INT32_MAX) return NMG_ERR_PARAM;
    if (!r->table || !r->positions) return NMG_ERR_NULL;
    if (!aligned(r->table, 4) || !aligned(r->positions, 4)) return NMG_ERR_ALIGN;
    return NMG_OK;
}

nmg_status check_part(nmg_dtype dtype, const RotaryRows &p, int64_t N, int32_t D) {
    if (!rows_ok(p.heads, D)) return NMG_ERR_PARAM;
    if (!p.X || !p.Y) return NMG_ERR_NULL;
    if (p.ldx < N || p.ldy < N) return NMG_ERR_PARAM;
    const size_t es = elem_size(dtype);
    if (!aligned(p.X, es) || !aligned(p.Y, es) || (p.weight && !aligned(p.weight, 4)))
        return NMG_ERR_ALIGN;
    if (p.X == p.Y && p.ldx != p.ldy) return NMG_ERR_PARAM;
    return NMG_OK;
}

nmg_status run_rotary(nmg_dtype dtype, RotaryArgs a, const nmg_rotary_desc *r, int64_t N,
                      bool norm, hipStream_t stream) {
    if (!dtype_ok(dtype)) return NMG_ERR_DTYPE;
    nmg_status st = check_rotary(r, a.D);
    if (st != NMG_OK) return st;
    if (N < 1 || N > INT32_MAX || a.D < 1) return NMG_ERR_PARAM;
    if ((st = check_part(dtype, a.part[0], N, a.D)) != NMG_OK) return st;
    if (a.part[1].heads && (st = check_part(dtype, a.part[1], N, a.D)) != NMG_OK) return st;
    a.N = (int32_t)N;
    a.R = r->dim;
    a.interleaved = r->pairs == NMG_ROTARY_INTERLEAVED;
    a.length = r->length;
    a.table = r->table;
    a.positions = r->positions;
    prelaunch();
    return launch_rotary(dtype, a, norm, stream);
}

nmg_status check_heads(const nmg_heads *h) {
    if (!h) return NMG_ERR_NULL;
    if (!dtype_ok(h->dtype)) return NMG_ERR_DTYPE;
    if (h->heads < 1 || h->kv_heads < 1 || h->heads % h->kv_heads || h->head_dim < 1)
        return NMG_ERR_PARAM;
    if (!rows_ok(h->heads, h->head_dim)) return NMG_ERR_PARAM;
    if (h->head_dim > 256) return NMG_ERR_UNSUPPORTED;
    return NMG_OK;
}

// The sizes alone; pointers unset
AttnArgs attn_sizes(const nmg_heads *h, int32_t sequences, int64_t Nq, int64_t Nk) {
    AttnArgs a = {};
    a.Nq = (int32_t)Nq;
    a.Nk = (int32_t)Nk;
    a.sequences = sequences;
    a.kv_heads = h->kv_heads;
    a.share = h->heads / h->kv_heads;
    a.D = h->head_dim;
    return a;
}

nmg_status run_attention(const nmg_heads *h, const nmg_sequences *s, const void *Q, int64_t ldq,
                         int64_t Nq, const void *K, int64_t ldk, const void *V, int64_t ldv,
                         int64_t Nk, const uint8_t *key_mask, const uint8_t *tree, int64_t ldtree,
                         int32_t width, float scale, void *O, int64_t ldo, void *workspace,
                         int64_t workspace_bytes, hipStream_t stream) {
    const nmg_status st = check_heads(h);
    if (st != NMG_OK) return st;
    if (!s || !Q || !O || (Nk > 0 && (!K || !V))) return NMG_ERR_NULL;
    if (s->count < 1 || Nq < 1 || Nq > INT32_MAX || Nk < 0 || Nk > INT32_MAX)
        return NMG_ERR_PARAM;
    if (!s->q_offsets || !s->kv_begin || !s->kv_end) return NMG_ERR_NULL;
    if (ldq < Nq || ldo < Nq || ldk < Nk || ldv < Nk) return NMG_ERR_PARAM;
    if (!(scale > 0.f) || !isfinite(scale)) return NMG_ERR_PARAM;
    const size_t es = elem_size(h->dtype);
    if (!aligned(Q, es) || !aligned(K, es) || !aligned(V, es) || !aligned(O, es) ||
        !aligned(s->q_offsets, 4) || !aligned(s->kv_begin, 4) || !aligned(s->kv_end, 4))
        return NMG_ERR_ALIGN;
    if (workspace_bytes < 0) return NMG_ERR_PARAM;
    if (workspace && !aligned(workspace, 256)) return NMG_ERR_ALIGN;
    AttnArgs a = attn_sizes(h, s->count, Nq, Nk);
    a.Q = Q;
    a.K = K;
    a.V = V;
    a.O = O;
    a.ldq = ldq;
    a.ldk = ldk;
    a.ldv = ldv;
    a.ldo = ldo;
    a.ldtree = ldtree;
    a.width = width;
    a.q_offsets = s->q_offsets;
    a.kv_begin = s->kv_begin;
    a.kv_end = s->kv_end;
    a.key_mask = key_mask;
    a.tree = tree;
    a.scale = scale;
    prelaunch();
    return launch_attention(h->dtype, a, workspace, workspace ? workspace_bytes : 0, stream);
}

}  // namespace

extern "C" {

nmg_status nmg_rotary_table(int32_t dim, int64_t length, double base, nmg_rotary_scaling scaling,
                            double factor, double original, double slow, double fast,
                            double magnitude, float *table, hipStream_t stream) {
    if (!table) return NMG_ERR_NULL;
    if (dim < 2 || dim % 2 || dim > 131070 || length < 1 || length > INT32_MAX ||
        !(base > 0) || !isfinite(base) || !isfinite(magnitude))
        return NMG_ERR_PARAM;
    if ((int)scaling < NMG_ROTARY_PLAIN || (int)scaling > NMG_ROTARY_PARTS) return NMG_ERR_PARAM;
    if (scaling != NMG_ROTARY_PLAIN && (!(factor >= 1) || !isfinite(factor))) return NMG_ERR_PARAM;
    if (scaling == NMG_ROTARY_NTK && dim < 4) return NMG_ERR_PARAM;
    if (scaling == NMG_ROTARY_PARTS &&
        (!(original > 0) || !isfinite(original) || !(slow >= 0) || !(fast > slow) ||
         !isfinite(fast)))
        return NMG_ERR_PARAM;
    if (!aligned(table, 4)) return NMG_ERR_ALIGN;
    RotaryTableArgs a;
    a.half = dim / 2;
    a.length = length;
    a.log_base = log(base);
    if (scaling == NMG_ROTARY_NTK) a.log_base += log(factor) * dim / (dim - 2);
    a.scaling = scaling;
    a.factor = factor;
    a.original = original;
    a.slow = slow;
    a.fast = fast;
    a.magnitude = magnitude;
    a.table = table;
    prelaunch();
    return launch_rotary_table(a, stream);
}

nmg_status nmg_rotary(nmg_dtype dtype, int32_t heads, int32_t head_dim,
                      const nmg_rotary_desc *rotary, const void *X, int64_t ldx, int64_t N,
                      void *Y, int64_t ldy, hipStream_t stream) {
    RotaryArgs a = {};
    a.part[0] = RotaryRows{X, Y, ldx, ldy, nullptr, heads};
    a.D = head_dim;
    return run_rotary(dtype, a, rotary, N, false, stream);
}

nmg_status nmg_qk_norm_rotary(nmg_dtype dtype, int32_t q_heads, int32_t k_heads, int32_t head_dim,
                              const nmg_rotary_desc *rotary, const float *q_weight,
                              const float *k_weight, float eps, const void *Q, int64_t ldq,
                              const void *K, int64_t ldk, int64_t N, void *YQ, int64_t ldyq,
                              void *YK, int64_t ldyk, hipStream_t stream) {
    if (k_heads < 0) return NMG_ERR_PARAM;
    if (!(eps >= 0.f) || !isfinite(eps)) return NMG_ERR_PARAM;
    RotaryArgs a = {};
    a.part[0] = RotaryRows{Q, YQ, ldq, ldyq, q_weight, q_heads};
    if (k_heads) a.part[1] = RotaryRows{K, YK, ldk, ldyk, k_weight, k_heads};
    a.D = head_dim;
    a.eps = eps;
    return run_rotary(dtype, a, rotary, N, true, stream);
}

nmg_status nmg_attention(const nmg_heads *heads, const nmg_sequences *sequences, const void *Q,
                         int64_t ldq, int64_t Nq, const void *K, int64_t ldk, const void *V,
                         int64_t ldv, int64_t Nk, const uint8_t *key_mask, float scale, void *O,
                         int64_t ldo, void *workspace, int64_t workspace_bytes,
                         hipStream_t stream) {
    return run_attention(heads, sequences, Q, ldq, Nq, K, ldk, V, ldv, Nk, key_mask, nullptr, 0, 0,
                         scale, O, ldo, workspace, workspace_bytes, stream);
}

nmg_status nmg_tree_attention(const nmg_heads *heads, const nmg_sequences *sequences,
                              const void *Q, int64_t ldq, int64_t Nq, const void *K, int64_t ldk,
                              const void *V, int64_t ldv, int64_t Nk, const uint8_t *tree,
                              int64_t ldtree, int64_t width, float scale, void *O, int64_t ldo,
                              void *workspace, int64_t workspace_bytes, hipStream_t stream) {
    if (!tree) return NMG_ERR_NULL;
    if (width < 1 || ldtree < width) return NMG_ERR_PARAM;
    if (Nq > 0 && Nq <= INT32_MAX && ldtree > INT32_MAX / Nq)
        return NMG_ERR_UNSUPPORTED;  // offsets of 31 bits
    return run_attention(heads, sequences, Q, ldq, Nq, K, ldk, V, ldv, Nk, nullptr, tree, ldtree,
                         (int32_t)width, scale, O, ldo, workspace, workspace_bytes, stream);
}

int64_t nmg_attention_workspace_bytes(const nmg_heads *heads, int32_t sequences, int64_t Nq,
                                      int64_t Nk) {
    if (check_heads(heads) != NMG_OK || sequences < 1 || Nq < 1 || Nq > INT32_MAX || Nk < 0 ||
        Nk > INT32_MAX)
        return -1;
    return attention_workspace_bytes(heads->dtype, attn_sizes(heads, sequences, Nq, Nk));
}

}  // extern "C"

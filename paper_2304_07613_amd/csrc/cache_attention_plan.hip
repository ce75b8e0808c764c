// cache_attention_plan.hip -- which workgroups an attention over the 8-bit cache gets.
#include "cache.hpp"

namespace nmg_internal {

nmg_status cache_attention_f16(nmg_cache_format format, const CacheAttnArgs &a, CacheAttnRows rows,
                               hipStream_t stream);
nmg_status cache_attention_f32(nmg_cache_format format, const CacheAttnArgs &a, CacheAttnRows rows,
                               hipStream_t stream);

namespace {

struct Plan {
    CacheAttnRows rows;
    int64_t slots;       // row tiles of all sequences, at most
    int64_t target;      // workgroups that splitting the keys aims at, 0: no splitting
};

int64_t part_bytes(const CacheAttnArgs &a, const Plan &p) { return 4 * (int64_t)(a.c.D + 2) * p.rows; }
// Parts' results: a sequence has up to one part more than its share of the target
int64_t part_count(const CacheAttnArgs &a, const Plan &p) { return p.target + p.slots * a.c.heads; }

Plan plan(nmg_dtype dtype, const CacheAttnArgs &a, int64_t longest) {
    Plan p;
    // the lengths are on the device: sequences with the same number of drafted tokens
    const int64_t rows = ((int64_t)a.Nq + a.c.sequences - 1) / a.c.sequences * a.share;
    const bool wide = a.c.D > 128;
    // Binary32 heads of 65 to 96: 32 rows do not fit the registers of two waves a SIMD beside their
    // six tiles of features.  8 sequences of 12 drafted tokens over 1032 to 2000, 8 / 4 heads of 96: 24.7 us with 16
    // rows, 33.3 with 32 and one wave, 37.5 with 32 and spills; 200 tokens over 2000, 12 heads: 49, 64, 58.
    const bool tight = a.c.D > 64 && a.c.D <= 96;
    if (dtype == NMG_F32)
        p.rows = rows <= 16 || wide || tight ? kRows16 : kRows32;
    else if (rows > (wide ? 16 : 64))
        p.rows = wide ? kRows64 : kRows128;
    else
        p.rows = rows <= 16 || wide ? kRows16 : kRows32;
    p.slots = (int64_t)a.Nq * a.share / p.rows + a.c.sequences;
    const int64_t full = (rows + p.rows - 1) / p.rows * a.c.sequences * a.c.heads;
    // two workgroups a compute unit, where the keys give each 8 tiles
    const int64_t tiles = longest / 64 + 1, most = 2 * device_cus();
    p.target = 2 * full <= most && tiles >= 16 ? most : 0;
    return p;
}

}  // namespace

int64_t cache_attention_workspace(nmg_dtype dtype, const CacheAttnArgs &a, int64_t longest) {
    const Plan p = plan(dtype, a, longest);
    return p.target ? part_bytes(a, p) * part_count(a, p) : 0;
}

nmg_status launch_cache_attention(nmg_dtype dtype, nmg_cache_format format, CacheAttnArgs a,
                                  int64_t longest, void *workspace, int64_t workspace_bytes,
                                  hipStream_t stream) {
    Plan p = plan(dtype, a, longest);
    if (!workspace) workspace_bytes = 0;
    if (p.slots * a.c.heads > INT32_MAX / 256) return NMG_ERR_UNSUPPORTED;
    // less room: fewer parts, none where not every row tile has two
    a.part_count = std::min(part_count(a, p), workspace_bytes / part_bytes(a, p));
    p.target = std::min(p.target, a.part_count - p.slots * a.c.heads);
    a.slots = (int32_t)p.slots;
    a.target = (int32_t)(p.target >= p.slots * a.c.heads ? p.target : 0);
    a.part = static_cast<float *>(workspace);
    return dtype == NMG_F32 ? cache_attention_f32(format, a, p.rows, stream)
                            : cache_attention_f16(format, a, p.rows, stream);
}

}  // namespace nmg_internal

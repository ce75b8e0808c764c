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
    int64_t parts;
};

int64_t part_bytes(const CacheAttnArgs &a, const Plan &p, int64_t parts) {
    return parts > 1 ? 4 * parts * p.slots * a.c.heads * (a.c.D + 2) * p.rows : 0;
}

Plan plan(nmg_dtype dtype, const CacheAttnArgs &a, int64_t longest) {
    Plan p;
    // the lengths are on the device: sequences with the same number of drafted tokens
    const int64_t rows = ((int64_t)a.Nq + a.c.sequences - 1) / a.c.sequences * a.share;
    const bool wide = a.c.D > 128;
    if (dtype == NMG_F32)
        p.rows = rows <= 16 || wide ? kRows16 : kRows32;
    else if (rows > (wide ? 16 : 64))
        p.rows = wide ? kRows64 : kRows128;
    else
        p.rows = rows <= 16 || wide ? kRows16 : kRows32;
    p.slots = (int64_t)a.Nq * a.share / p.rows + a.c.sequences;
    const int64_t full = (rows + p.rows - 1) / p.rows * a.c.sequences * a.c.heads;
    const int64_t tiles = longest / 64 + 1;
    p.parts = std::max<int64_t>(1, std::min((int64_t)2 * device_cus() / full, std::min<int64_t>(32, tiles / 8)));
    return p;
}

}  // namespace

int64_t cache_attention_workspace(nmg_dtype dtype, const CacheAttnArgs &a, int64_t longest) {
    const Plan p = plan(dtype, a, longest);
    return part_bytes(a, p, p.parts);
}

nmg_status launch_cache_attention(nmg_dtype dtype, nmg_cache_format format, CacheAttnArgs a,
                                  int64_t longest, void *workspace, int64_t workspace_bytes,
                                  hipStream_t stream) {
    Plan p = plan(dtype, a, longest);
    if (!workspace) workspace_bytes = 0;
    while (p.parts > 1 && part_bytes(a, p, p.parts) > workspace_bytes) --p.parts;
    if (p.slots * a.c.heads > INT32_MAX / 256) return NMG_ERR_UNSUPPORTED;
    a.slots = (int32_t)p.slots;
    a.parts = (int32_t)p.parts;
    a.part = static_cast<float *>(workspace);
    return dtype == NMG_F32 ? cache_attention_f32(format, a, p.rows, stream)
                            : cache_attention_f16(format, a, p.rows, stream);
}

}  // namespace nmg_internal

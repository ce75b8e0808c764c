// cache_attention_plan.hip -- which workgroups an attention over the 8-bit cache gets.
#include "cache.hpp"

namespace nmg_internal {

nmg_status cache_attention_f16(nmg_cache_format format, const CacheAttnArgs &a, int nt, hipStream_t stream);
nmg_status cache_attention_f32(nmg_cache_format format, const CacheAttnArgs &a, int nt, hipStream_t stream);

namespace {

struct Plan {
    int nt;              // tiles of 16 rows a workgroup has
    int64_t slots;       // row tiles of all sequences, at most
    int64_t parts;
};

int64_t part_bytes(const CacheAttnArgs &a, const Plan &p, int64_t parts) {
    return parts > 1 ? 4 * parts * p.slots * a.c.heads * (a.c.D + 2) * 16 * p.nt : 0;
}

Plan plan(nmg_dtype dtype, const CacheAttnArgs &a, int64_t longest) {
    Plan p;
    const int64_t rows = ((int64_t)a.Nq + a.c.sequences - 1) / a.c.sequences * a.share;
    const int most = dtype == NMG_F32 ? (a.c.D > 128 ? 1 : 2) : 2;
    p.nt = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    if (p.nt > most) p.nt = most;
    p.slots = (int64_t)a.Nq * a.share / (16 * p.nt) + a.c.sequences;
    const int64_t full = (rows + 16 * p.nt - 1) / (16 * p.nt) * a.c.sequences * a.c.heads;
    const int64_t tiles = longest / 64 + 1;
    p.parts = std::max<int64_t>(1, std::min((int64_t)2 * device_cus() / full, std::min<int64_t>(64, tiles / 8)));
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
    return dtype == NMG_F32 ? cache_attention_f32(format, a, p.nt, stream)
                            : cache_attention_f16(format, a, p.nt, stream);
}

}  // namespace nmg_internal

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
    // Binary16, us with the shared tiles (kRows64, kRows128) / with waves that have keys of their own, 8 sequences: 33 to
    // 64 rows over 4096, 8 heads of 128: 43 / 36; 65 to 96: 47 / 53; 128: 49.5 / 49; over 3000, heads of 96, 65 to
    // 96: 40 / 42, 128: 41 / 35.5; over 2000, 12 heads of 64, 65 to 128: 32 / 24, but over 500 of 16 sequences
    // 22 / 26.  Heads of 129 and more, 4 sequences of 3000: 17 rows 37 / 49, 64 rows 38.5 / 63.
    if (dtype == NMG_F32)
        p.rows = rows <= 16 || wide || tight ? kRows16 : kRows32;
    else if (rows > (wide ? 16 : 64))
        p.rows = wide ? kRows64 : kRows128;
    else
        p.rows = rows <= 16 || wide ? kRows16 : kRows32;
    p.slots = (int64_t)a.Nq * a.share / p.rows + a.c.sequences;
    const int64_t full = (rows + p.rows - 1) / p.rows * a.c.sequences * a.c.heads;
    // Two workgroups a compute unit, where that splits row tiles in two or more and there are 16 key tiles.
    // Split / not, single tokens: 2 sequences of 500 tokens, 8 heads of 128: 19 / 14 us, 1100: 18.7 / 16.6,
    // 1900: 19 / 20.4; heads of 256, 1100: 27.6 / 30.4; binary32, 1100: 26 / 32, 1900: 27 / 46; 8 of 1900, 12 heads of
    // 64: 17.7 / 13.3.  8 sequences of 8192 tokens, 32 heads of 128 (256 row tiles): 113 / 102; 9: 141 / 150; 12: 165 /
    // 161.  Past 256 nothing is split, whatever the lengths: 32768 tokens and 7 times 100 take 68 us, 8 times 100 194.
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

// attention_plan.hip -- how one attention call is laid over the GPU: the kernel,
// its row tiles, and into how many parts every key range is split.
#include "attention.hpp"

namespace nmg_internal {

namespace {

struct Plan {
    bool shared;
    int64_t tiles;   // of one key head: an upper bound, the sequences' lengths are on the device
    int splits;      // wanted
    int64_t part_bytes;  // of one part of every range
};

Plan plan_of(nmg_dtype dtype, const AttnArgs &a) {
    Plan p;
    const int64_t rows = (int64_t)a.Nq * a.share;
    const int64_t each = (rows + a.sequences - 1) / a.sequences;  // of equal sequences
    const int64_t keys = (a.Nk + a.sequences - 1) / a.sequences;  // that share Nk
    const int dp = attn_padded_dim(a.D);
    const int kt = dtype == NMG_F16 ? 64 : 32;
    // One or two waves' rows cover a sequence: the waves of a workgroup split the keys
    // rather than the rows, while a compute unit has one such workgroup to run (12 heads
    // x 64, 512 keys: 8 sequences of 64 columns 11.7 -> 7.4 us, of 128 11.7 -> 13.3; 64 of
    // 64 23 -> 41).  With more of them one wave's rows, and keys enough that the waves
    // are worth their start (64 sequences of 1 column: binary16 with 512 keys 22 -> 25 us,
    // 2048 81 -> 79, binary32 with 128 30 -> 23; 256 of 64 75 -> 92); always for heads
    // over 128, of which a compute unit holds one workgroup either way (8 x 256, 64
    // sequences, 256 keys: 51 -> 47).
    const int64_t few = (each + kAttnSplitRows - 1) / kAttnSplitRows;
    const bool once = few <= 2 && few * a.sequences <= device_cus() / a.kv_heads;
    const int64_t enough = dtype == NMG_F16 ? 1024 : 128;
    p.shared = !once && !(few <= 1 && (dp > 128 || keys >= enough));
    const int tr = p.shared ? kAttnSharedRows : kAttnSplitRows;
    // sum of ceil(rows_b / tr) over sequences that hold `rows` rows together: at most ...
    p.tiles = a.sequences == 1 ? (rows + tr - 1) / tr : std::min(rows / tr + a.sequences, rows);
    // ... and for equal lengths
    const int64_t items = std::min((each + tr - 1) / tr * a.sequences, p.tiles) * a.kv_heads;
    const int waves = p.shared ? 1 : attn_split_waves(dp);  // that split a part's keys
    const int64_t steps = (keys + (int64_t)kt * waves - 1) / (kt * waves);
    // workgroups a compute unit holds (binary32 16 heads x 128, 2 sequences of 512
    // columns over 1024 keys: 87 us in the 4 parts for two of them, 77 in 2 for one)
    const int held = p.shared && dp <= (dtype == NMG_F16 ? 128 : 64) ? 2 : 1;
    const int64_t slots = (int64_t)device_cus() * held;
    // The split that ends first, in steps of one key tile: rounds of workgroups
    // times (its steps + about 2 to start), and with parts their traffic (an
    // item's sums written and read: for 512 of 128 rows about 8 steps) and a launch.
    // (One part against the split taken: 12 heads x 64, 1 column over 8192 keys 26 ->
    // 12.6 us; 32 / 8 x 128, 1 over 32768 243 -> 33, 4 of 63 over 32768 601 -> 188; 16 x
    // 64, 512 over 16384 218 -> 58; binary32 12 x 64, 256 over 8192 507 -> 61.)
    // A step is longer in binary32 (16 x 128, 2 of 512 over 600: 75 us with 40, 56), and of
    // waves that split the keys the fewer they are, so the join (4 us) is fewer of them
    // (32 / 8 x 128, 4 of 1 over 2000: 25.6 us with 40 and 16 for all, 18.4; binary32
    // 12 x 64, 1 over 1000 22.9 and 14.6, 8 of 1 24.4 and 20.7).
    const bool f32 = dtype == NMG_F32;
    const int64_t traffic = p.shared ? 32 : f32 ? 8 : 16;
    const int64_t join = p.shared ? (f32 ? 30 : 40) : f32 ? 7 : dp <= 64 ? 32 : 14;
    p.splits = 1;
    int64_t best = INT64_MAX;
    for (int64_t s = 1; s <= kAttnMostSplits && (s == 1 || steps / s >= (p.shared ? 4 : 1)); ++s) {
        const int64_t rounds = (items * s + slots - 1) / slots;
        const int64_t cost = 8 * rounds * ((steps + s - 1) / s + 2) +
                             (s > 1 ? items * s * traffic / device_cus() + join : 0);
        if (cost < best) {
            best = cost;
            p.splits = (int)s;
        }
    }
    const int64_t blocks = p.tiles * a.kv_heads;
    p.part_bytes = blocks * (dp + 2) * tr * (int64_t)sizeof(float);
    return p;
}

}  // namespace

int64_t attention_workspace_bytes(nmg_dtype dtype, const AttnArgs &a) {
    const Plan p = plan_of(dtype, a);
    return p.splits > 1 ? p.splits * p.part_bytes : 0;
}

nmg_status launch_attention(nmg_dtype dtype, const AttnArgs &args, void *workspace,
                            int64_t workspace_bytes, hipStream_t stream) {
    AttnArgs a = args;
    const Plan p = plan_of(dtype, a);
    int64_t splits = std::min<int64_t>(p.splits, workspace_bytes / p.part_bytes);
    if (splits < 2) splits = 1;
    const int threads = p.shared ? 4 * 64 : attn_split_waves(attn_padded_dim(a.D)) * 64;
    if (!launchable(p.tiles * splits * a.kv_heads, std::max(threads, kBlock)))
        return NMG_ERR_UNSUPPORTED;
    a.tiles = (int32_t)p.tiles;
    a.splits = (int32_t)splits;
    a.part = (float *)workspace;
    // a joining thread waits for every row it takes: one each, until that is more than
    // about 8 workgroups for every compute unit, which read the parts' maxima again
    a.join_rows = kBlock / (p.shared ? kAttnSharedRows : kAttnSplitRows);
    while (a.join_rows < 32 && p.tiles * a.kv_heads * a.D / a.join_rows > 8 * device_cus())
        a.join_rows *= 2;
    const int64_t es = (int64_t)elem_size(dtype);
    auto rows_at = [&](int64_t to) {  // rows of K and V start at multiples of `to` bytes
        return aligned(a.K, to) && aligned(a.V, to) && a.ldk * es % to == 0 && a.ldv * es % to == 0;
    };
    // a lane's offset among 8 rows is 32 bits wide
    if (std::max(a.ldk, a.ldv) * es > INT32_MAX / 8) return NMG_ERR_UNSUPPORTED;
    // (a head's padded rows count)
    const bool wide = std::max(a.ldk, a.ldv) * es * attn_padded_dim(a.D) > INT32_MAX - 4096;
    const AttnRows how = !rows_at(4) ? kAttnShift : wide ? kAttnWide : kAttnNarrow;
    // key tiles start at whole 16 bytes of a row where the rows do
    a.align = (int32_t)(how == kAttnShift ? 1 : rows_at(16) ? 16 / es : 4 / es);
    return dtype == NMG_F16 ? launch_attention_f16(a, p.shared, how, stream)
                            : launch_attention_f32(a, p.shared, how, stream);
}

}  // namespace nmg_internal

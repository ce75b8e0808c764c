// k_cache.hip -- what happens to an 8-bit cache between the attentions: drafted
// tokens come in, kept ones become pages, pages are handed out, shared, given back
// and moved together.  (The attention: cache_attention.hpp.)
#include "cache.hpp"

namespace {

// ---------------------------------------------------------------- append

// Columns of K and V (features x tokens) to the rings: a workgroup takes 64 columns
// of 64 features of one key head.  Values stay as they lie, feature after feature, four
// tokens at a time where their slots follow one another; keys are turned through LDS, so that
// both sides are read and written along their rows.  8 tokens of 12 heads of 64: 6.4 us, the
// chain of offsets, places and stores; 4 x 2047 of 8 x 128 (67 MB): 19 us, 3.5 TB/s, odd rows that
// start on no cache line on one side and runs of 128 bytes on the other.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_cache_append(CacheView v, int layer, const int32_t *q_offsets,
                                                         const int32_t *lengths, const T *K, int64_t ldk,
                                                         const T *V, int64_t ldv, int N) {
    __shared__ T tile[64][64 + 4 / sizeof(T)];
    __shared__ int ring[64], at[64];       // of every column: its sequence (-1: none), its slot
    const int n0 = blockIdx.x * 64, d0 = blockIdx.y % ((v.D16 + 63) / 64) * 64,
              head = blockIdx.y / ((v.D16 + 63) / 64);
    const int tid = threadIdx.x;
    // what is read goes on its way before the places are known
    constexpr int kRows = kBlock / 16;
    const int j4 = tid % 16 * 4, left = N - n0 - j4;      // the thread's four columns
    struct alignas(sizeof(T)) Four { T e[4]; };
    Four k[64 / kRows], val[64 / kRows];
#pragma unroll
    for (int i = 0; i < 64 / kRows; ++i) {
        const int d = d0 + tid / 16 + i * kRows;
        const int64_t row = (int64_t)head * v.D + d;
        k[i] = val[i] = Four{};
        if (d >= v.D) continue;
        const T *from_k = K + row * ldk + n0 + j4, *from_v = V + row * ldv + n0 + j4;
        if (left >= 4) {
            __builtin_memcpy(&k[i], from_k, sizeof(Four));
            __builtin_memcpy(&val[i], from_v, sizeof(Four));
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < left) {
                    k[i].e[e] = from_k[e];
                    val[i].e[e] = from_v[e];
                }
        }
    }
    if (tid < 64) {
        const int col = n0 + tid;
        int b = -1, first = 0, n = 0;
        if (v.sequences <= 64) {           // a lane looks up a sequence, then all compare
            const int s = min(tid, v.sequences - 1);
            const int from = q_offsets[s], to = q_offsets[s + 1], length = cache_length(v, lengths, s);
            for (int q = 0; q < v.sequences; ++q) {
                const int lo = __builtin_amdgcn_readlane(from, q), hi = __builtin_amdgcn_readlane(to, q);
                if (col >= lo && col < hi) {
                    b = q;
                    first = lo;
                    n = __builtin_amdgcn_readlane(length, q);
                }
            }
        } else if (col >= q_offsets[0] && col < q_offsets[v.sequences]) {
            b = 0;
            int hi = v.sequences - 1;      // the last b with q_offsets[b] <= col
            while (b < hi) {
                const int mid = (b + hi + 1) / 2;
                if (q_offsets[mid] <= col)
                    b = mid;
                else
                    hi = mid - 1;
            }
            first = q_offsets[b];
            n = cache_length(v, lengths, b);
        }
        const int i = (int)((uint32_t)col - (uint32_t)first);
        const bool in = b >= 0 && col < N && i >= 0 && i < v.room - n % v.block;   // not past the room
        ring[tid] = in ? b : -1;
        at[tid] = in ? (int)((uint32_t)(n + i) % (uint32_t)v.room) : 0;
    }
    __syncthreads();
    const int64_t head_of = (int64_t)layer * v.sequences;
    T *ko = static_cast<T *>(v.k_open), *vo = static_cast<T *>(v.v_open);
    auto head_ring = [&](int j) { return (head_of + ring[j]) * v.heads + head; };
    const bool run = ring[j4] >= 0 && ring[j4] == ring[j4 + 3] && at[j4 + 3] == at[j4] + 3;
#pragma unroll
    for (int i = 0; i < 64 / kRows; ++i) {
        const int r = tid / 16 + i * kRows, d = d0 + r;
#pragma unroll
        for (int e = 0; e < 4; ++e) tile[r][j4 + e] = k[i].e[e];
        if (d >= v.D) continue;
        if (run)
            __builtin_memcpy(vo + (head_ring(j4) * v.D + d) * v.room + at[j4], &val[i], sizeof(Four));
        else
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (ring[j4 + e] >= 0) vo[(head_ring(j4 + e) * v.D + d) * v.room + at[j4 + e]] = val[i].e[e];
    }
    __syncthreads();
    // 16 bytes of a key's row a thread
    constexpr int kE = 16 / sizeof(T), kParts = 64 / kE;
    const int d = tid % kParts * kE;
    if (d0 + d >= v.D16) return;
    for (int j = tid / kParts; j < 64; j += kBlock / kParts) {
        if (ring[j] < 0) continue;
        alignas(16) T row[kE];
#pragma unroll
        for (int e = 0; e < kE; ++e) row[e] = tile[d + e][j];
        *reinterpret_cast<uint4 *>(ko + (head_ring(j) * v.room + at[j]) * v.D16 + d0 + d) =
            *reinterpret_cast<const uint4 *>(row);
    }
}

// ---------------------------------------------------------------- commit

// The scale of a block whose largest magnitude has the bits `top`: the smallest power
// of two from 2^-126 on with max <= scale * (largest code); NaN where a
// value is not finite.  *limit: the largest code that stands for no more than the type's largest
// value -- less than the largest code only at the one scale that reaches past it.
template <typename T, bool kInt8>
__device__ __forceinline__ float block_scale(uint32_t top, float *inverse, float *limit) {
    constexpr bool kF32 = std::is_same<T, float>::value;
    if (top >= 0x7f800000u) {
        *inverse = 0.f;
        *limit = 0.f;
        return __builtin_nanf("");
    }
    // 448 = 1.75 * 2^8, 127 = 1.984375 * 2^6
    int e = (int)(top >> 23) - 127 - (kInt8 ? 6 : 8);
    e += (top & 0x7fffffu) > (kInt8 ? 0x7e0000u : 0x600000u);
    e = e < -126 ? -126 : e;
    constexpr int last = kF32 ? (kInt8 ? 122 : 120) : (kInt8 ? 10 : 8);
    *limit = e == last ? (kInt8 ? 63.f : 240.f) : (kInt8 ? 127.f : 448.f);
    *inverse = __builtin_ldexpf(1.f, -e);
    return __builtin_ldexpf(1.f, e);
}

// Four values as codes; a block that is not finite gets zeros (its scale says so)
template <bool kInt8>
__device__ __forceinline__ uint32_t encode4(v4f x, float inverse, float limit) {
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = inverse == 0.f ? 0.f : fminf(fmaxf(x[i] * inverse, -limit), limit);
    if constexpr (kInt8) {
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) w |= ((uint32_t)(int)rintf(y[i]) & 0xffu) << (8 * i);
        return w;
    } else {
#if defined(__HIP_DEVICE_COMPILE__)
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
#else
        return 0;
#endif
    }
}

__device__ __forceinline__ uint32_t workgroup_max(uint32_t v, uint32_t *lds) {
    for (int d = 1; d < 64; d *= 2) v = max(v, (uint32_t)__shfl_xor((int)v, d));
    __syncthreads();
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    v = lds[0];
    for (int i = 1; i < kBlock / 64; ++i) v = max(v, lds[i]);
    return v;
}

// What one sequence's call does: `open` kept tokens of the last block and `more`
// newly kept ones; the first whole * block of them become pages
struct Commit {
    int n, open, more, whole;
};
__device__ __forceinline__ Commit commit_of(const CacheView &v, const int32_t *lengths,
                                            const int32_t *kept_offsets, bool list, int n_kept, int b) {
    Commit k;
    k.n = cache_length(v, lengths, b);
    k.open = k.n % v.block;
    int lo = kept_offsets[b], hi = kept_offsets[b + 1];
    if (list) {
        lo = min(max(lo, 0), n_kept);
        hi = min(max(hi, 0), n_kept);
    }
    k.more = (int)min((int64_t)max(0, v.room - k.open), max((int64_t)0, (int64_t)hi - lo));
    k.whole = (k.open + k.more) / v.block;
    for (int j0 = 0; j0 < k.whole; j0 += 64) {   // a lane of every wave looks at a block
        const int j = j0 + (threadIdx.x & 63), at = k.n / v.block + j;
        const int page = j < k.whole && at < v.row ? v.table[(int64_t)b * v.row + at] : -1;
        const uint64_t none = __ballot(j < k.whole && (page < 0 || page >= v.pages));
        if (none) {   // no page: the sequence ends before this block does
            k.whole = j0 + __ffsll((unsigned long long)none) - 1;
            k.more = max(0, (k.whole + 1) * v.block - 1 - k.open);
            break;
        }
    }
    return k;
}

// One (sequence, layer and key head, keys or values) and, without a list, every gridDim.z-th
// of its blocks: the largest magnitude, then the codes.  With a list the kept
// tokens lie anywhere among the drafted ones: the workgroup makes all pages, then moves what stays
// open to the front, in pieces that are read before they are written.  (The list
// ascends, so no piece is written over before a later one has been read.)  4 x 2047 tokens of
// 8 heads of 128 (50 MB): 13.8 us, 3.6 TB/s: 1020 blocks for 768 places, each a chain of table, block, maximum and
// codes.  8 sequences of which one fills a block: 3.9 us.
template <typename T, bool kInt8, bool kList>
__global__ __launch_bounds__(kBlock) void k_cache_commit(CacheView v, const int32_t *lengths,
                                                         const int32_t *kept_offsets, const int32_t *kept,
                                                         int n_kept, int32_t *new_lengths) {
    __shared__ uint32_t most[kBlock / 64];
    __shared__ int slots[128];
    const int b = blockIdx.x, is_v = blockIdx.y & 1, lh = blockIdx.y >> 1;   // layer * heads + head
    const int layer = lh / v.heads, head = lh % v.heads, tid = threadIdx.x;
    const Commit k = commit_of(v, lengths, kept_offsets, kList, n_kept, b);
    if (blockIdx.y == 0 && blockIdx.z == 0 && tid == 0) new_lengths[b] = k.n + k.more;
    const int full = k.n - k.open;
    const int64_t ring = ((int64_t)layer * v.sequences + b) * v.heads + head;
    const T *open = static_cast<const T *>(is_v ? v.v_open : v.k_open) +
                    ring * v.room * (is_v ? v.D : v.D16);
    const int first = kList ? max(0, min(kept_offsets[b], n_kept)) : 0;
    // slot of token u of the open list
    auto slot_of = [&](int u) {
        int at = full + u;
        if (kList && u >= k.open) at = k.n + min(max(kept[first + u - k.open], 0), v.room - 1);
        return (int)((uint32_t)at % (uint32_t)v.room);
    };
    for (int j = blockIdx.z; j < k.whole; j += gridDim.z) {
        // without a list the block's slots follow one another
        const int slot0 = slot_of(j * v.block);
        if constexpr (kList) {
            __syncthreads();
            if (tid < v.block) slots[tid] = slot_of(j * v.block + tid);
            __syncthreads();
        }
        const int page = v.table[(int64_t)b * v.row + full / v.block + j];
        const int64_t of = ((int64_t)layer * v.pages + page) * v.heads + head;
        // 16 bytes of neighbours: of a key's features, of a feature's tokens
        constexpr int kE = 16 / sizeof(T);
        struct alignas(16) Some { T e[kE]; };
        const int width = is_v ? v.block : v.D16, units = (is_v ? v.D : v.block) * (width / kE);
        auto some = [&](int i) {
            if (!kList && !is_v)
                return *reinterpret_cast<const Some *>(open + (int64_t)slot0 * v.D16 + i * kE);
            const int r = i / (width / kE), e = i % (width / kE) * kE;
            if (!is_v) return *reinterpret_cast<const Some *>(open + (int64_t)slots[r] * v.D16 + e);
            const T *row = open + (int64_t)r * v.room;
            if (!kList) return *reinterpret_cast<const Some *>(row + slot0 + e);
            Some x;
#pragma unroll
            for (int m = 0; m < kE; ++m) x.e[m] = row[slots[e + m]];
            return x;
        };
        // blocks of up to 16384 values stay in registers between their maximum and their codes
        constexpr int kKeep = 64 / kE;
        const bool keep = units <= kKeep * kBlock;
        Some held[kKeep];
        uint32_t top = 0;
        auto look = [&](const Some &x) {
#pragma unroll
            for (int m = 0; m < kE; ++m) top = max(top, __float_as_uint((float)x.e[m]) & 0x7fffffffu);
        };
        if (keep) {
            // (a thread past the end looks at the last unit once more)
#pragma unroll
            for (int h = 0; h < kKeep; ++h) held[h] = some(min(h * kBlock + tid, units - 1));
#pragma unroll
            for (int h = 0; h < kKeep; ++h) look(held[h]);
        } else {
            for (int i = tid; i < units; i += kBlock) look(some(i));
        }
        top = workgroup_max(top, most);
        float inverse, limit;
        const float scale = block_scale<T, kInt8>(top, &inverse, &limit);
        uint32_t *to = reinterpret_cast<uint32_t *>((is_v ? v.v_pages + of * v.D * v.block
                                                          : v.k_pages + of * v.block * v.D16));
        auto store = [&](int i, const Some &x) {
#pragma unroll
            for (int m = 0; m < kE; m += 4)
                to[(i * kE + m) / 4] = encode4<kInt8>(v4f{(float)x.e[m], (float)x.e[m + 1], (float)x.e[m + 2],
                                                          (float)x.e[m + 3]}, inverse, limit);
        };
        if (keep) {
#pragma unroll
            for (int h = 0; h < kKeep; ++h)
                if (h * kBlock + tid < units) store(h * kBlock + tid, held[h]);
        } else {
            for (int i = tid; i < units; i += kBlock) store(i, some(i));
        }
        if (tid == 0) (is_v ? v.v_scales : v.k_scales)[of] = scale;
    }
    if constexpr (!kList) return;
    T *ring_out = const_cast<T *>(open);
    const int from = max(k.whole * v.block, k.open), end = k.open + k.more;
    const int width = is_v ? v.D : v.D16;
    constexpr int kHold = 4;                  // values of a thread and piece
    const int piece = max(1, kBlock * kHold / width);
    for (int u0 = from; u0 < end; u0 += piece) {
        const int count = min(piece, end - u0) * width;
        T held[kHold];
        __syncthreads();
#pragma unroll
        for (int h = 0; h < kHold; ++h) {
            const int i = h * kBlock + tid;
            if (i >= count) continue;
            const int s = slot_of(u0 + i / width), d = i % width;
            held[h] = is_v ? open[(int64_t)d * v.room + s] : open[(int64_t)s * v.D16 + d];
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < kHold; ++h) {
            const int i = h * kBlock + tid;
            if (i >= count) continue;
            const int s = (int)((uint32_t)(full + u0 + i / width) % (uint32_t)v.room), d = i % width;
            ring_out[is_v ? (int64_t)d * v.room + s : (int64_t)s * v.D16 + d] = held[h];
        }
    }
}

// ------------------------------------------------------------- pages of the pool

constexpr int kWide = 1024;       // threads of the one-workgroup kernels

// Exclusive sums over the workgroup's threads of `mine`; *all: the total
__device__ __forceinline__ int workgroup_scan(int mine, int *all, int *lds) {
    int v = mine;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int d = 1; d < 64; d *= 2) {
        const int up = __shfl_up(v, d);
        if (lane >= d) v += up;
    }
    __syncthreads();
    if (lane == 63) lds[wave] = v;
    __syncthreads();
    int before = 0, sum = 0;
    for (int w = 0; w < kWide / 64; ++w) {
        if (w < wave) before += lds[w];
        sum += lds[w];
    }
    *all = sum;
    return before + v - mine;
}

// Pages for coming tokens, in one launch without a wait of the host: the lowest free ones, sequence after sequence.  One workgroup:
// sequences in pieces of a thread each; while a piece wants pages, the pool is looked through
// from where the last one was found.  8 us where none is wanted or they are among the first; 0.6 to 0.8 ns a page
// that lies before them: 45 us behind 60000 used ones, 785 behind 10^6.
__global__ __launch_bounds__(kWide) void k_cache_reserve(CacheView v, const int32_t *lengths,
                                                         const int32_t *tokens, int32_t *missing) {
    __shared__ int lds[kWide / 64], upto[kWide], entry[kWide];
    const int tid = threadIdx.x;
    int cursor = 0;
    int64_t lacking = 0;
    for (int b0 = 0; b0 < v.sequences; b0 += kWide) {
        const int b = b0 + tid;
        int want = 0, have = 0;
        if (b < v.sequences) {
            const int n = cache_length(v, lengths, b);
            const int64_t blocks = ((int64_t)n + max(tokens[b], 0)) / v.block;
            const int target = (int)min(blocks, (int64_t)v.row);
            have = n / v.block;
            while (have < target && v.table[(int64_t)b * v.row + have] >= 0) ++have;
            want = max(0, target - have);
            lacking += blocks - target;
        }
        int all, got = 0;
        const int before = workgroup_scan(want, &all, lds);
        upto[tid] = before + want;
        entry[tid] = have;
        __syncthreads();
        while (got < all && cursor < v.pages) {        // (uniform: got, all, cursor are)
            const int p = cursor + tid;
            const int free = p < v.pages && v.references[p] == 0;
            int found;
            const int rank = got + workgroup_scan(free, &found, lds);
            if (free && rank < all) {
                int lo = 0, hi = kWide - 1;             // the first sequence with upto > rank
                while (lo < hi) {
                    const int mid = (lo + hi) / 2;
                    if (upto[mid] > rank)
                        hi = mid;
                    else
                        lo = mid + 1;
                }
                const int start = lo ? upto[lo - 1] : 0;
                v.table[(int64_t)(b0 + lo) * v.row + entry[lo] + rank - start] = p;
                v.references[p] = 1;
            }
            got += found;
            if (got <= all) cursor += kWide;            // else some of these are left
        }
        if (tid == 0 && got < all) lacking += all - got;
        __syncthreads();
    }
    int all;
    (void)workgroup_scan((int)min(lacking, (int64_t)INT32_MAX / kWide), &all, lds);
    if (tid == 0) *missing = all;
}

// A row's pages given back
__device__ __forceinline__ void release_row(const CacheView &v, int32_t *row, int i) {
    const int p = row[i];
    if (p >= 0 && p < v.pages) atomicSub(v.references + p, 1);
    row[i] = -1;
}

// Sequence to[i] becomes a copy of from[i]: it shares the pages, which are never written
// again, and has the open tokens for itself.  blockIdx.y 0: the row; others: 16
// bytes a thread and turn of the ring's block.  4 copies in 12 layers of 12 heads of 64 (9 MB): 6.5 us, the
// chain of length and copy.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_cache_fork(CacheView v, int32_t *lengths, SlotList list) {
    const int a = list.from[blockIdx.x], b = list.to[blockIdx.x];
    const int n = cache_length(v, lengths, a), open = n % v.block, pages = n / v.block;
    if (blockIdx.y == 0) {
        int32_t *to = v.table + (int64_t)b * v.row;
        const int32_t *from = v.table + (int64_t)a * v.row;
        for (int i = threadIdx.x; i < v.row; i += kBlock) {
            release_row(v, to, i);
            const int p = i < pages ? from[i] : -1;
            if (p >= 0 && p < v.pages) atomicAdd(v.references + p, 1);
            to[i] = p;
        }
        if (threadIdx.x == 0) lengths[b] = n;
        return;
    }
    constexpr int kE = 16 / sizeof(T);
    const int k_units = v.block * v.D16 / kE, v_units = v.D * v.block / kE;
    const int start = (int)((uint32_t)(n - open) % (uint32_t)v.room);
    const int64_t units = (int64_t)v.layers * v.heads * (k_units + v_units);
    for (int64_t unit = (int64_t)(blockIdx.y - 1) * kBlock + threadIdx.x; unit < units;
         unit += (int64_t)(gridDim.y - 1) * kBlock) {
        const int lh = (int)(unit / (k_units + v_units)), at = (int)(unit % (k_units + v_units));
        const int layer = lh / v.heads, head = lh % v.heads;
        const int64_t ra = ((int64_t)layer * v.sequences + a) * v.heads + head,
                      rb = ((int64_t)layer * v.sequences + b) * v.heads + head;
        if (at < k_units) {
            if (at >= open * v.D16 / kE) continue;
            T *k = static_cast<T *>(v.k_open);
            const int64_t e = (int64_t)start * v.D16 + (int64_t)at * kE;
            *reinterpret_cast<uint4 *>(k + rb * v.room * v.D16 + e) =
                *reinterpret_cast<const uint4 *>(k + ra * v.room * v.D16 + e);
        } else {
            const int d = (at - k_units) / (v.block / kE), u = (at - k_units) % (v.block / kE) * kE;
            if (u >= open) continue;
            T *values = static_cast<T *>(v.v_open);
            const T *from = values + (ra * v.D + d) * v.room + start + u;
            T *to = values + (rb * v.D + d) * v.room + start + u;
            if (u + kE <= open)
                *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(from);
            else
                for (int i = 0; u + i < open; ++i) to[i] = from[i];
        }
    }
}

__global__ __launch_bounds__(kBlock) void k_cache_free(CacheView v, int32_t *lengths, SlotList list) {
    const int b = list.to[blockIdx.x];
    for (int i = threadIdx.x; i < v.row; i += kBlock) release_row(v, v.table + (int64_t)b * v.row, i);
    if (threadIdx.x == 0) lengths[b] = 0;
}

// What moves where: with L pages in use, the k-th free page below L gets the k-th used one
// from L on.  Workspace: moves, then sources, targets, references of the sources and the new
// place of every page.  One workgroup, a run of pages per thread: 6.4 us for 2048 pages.
__global__ __launch_bounds__(kWide) void k_compact_plan(CacheView v, int32_t *references_out,
                                                        int32_t *live, int32_t *ws) {
    __shared__ int lds[kWide / 64];
    const int64_t P = v.pages;
    int32_t *source = ws + 1, *target = source + P, *count = target + P, *place = count + P;
    const int per = (v.pages + kWide - 1) / kWide;
    const int begin = (int)min((int64_t)per * threadIdx.x, P), end = (int)min((int64_t)begin + per, P);
    int mine = 0, L, moves;
    for (int p = begin; p < end; ++p) mine += v.references[p] > 0;
    (void)workgroup_scan(mine, &L, lds);
    int holes = 0, high = 0;
    for (int p = begin; p < end; ++p) {
        const bool used = v.references[p] > 0;
        holes += !used && p < L;
        high += used && p >= L;
    }
    const int hole0 = workgroup_scan(holes, &moves, lds), high0 = workgroup_scan(high, &moves, lds);
    for (int p = begin, i = hole0, j = high0; p < end; ++p) {
        const int r = v.references[p];
        place[p] = p;
        if (r <= 0 && p < L) target[i++] = p;
        if (r > 0 && p >= L) {
            source[j] = p;
            count[j++] = r;
        }
    }
    __syncthreads();
    for (int p = begin, i = hole0; p < end; ++p) {
        const int r = v.references[p];
        if (p >= L) {
            references_out[p] = 0;
        } else if (r <= 0) {
            references_out[p] = count[i];
            place[source[i]] = p;      // (its own thread wrote it before the barrier)
            ++i;
        } else {
            references_out[p] = r;
        }
    }
    if (threadIdx.x == 0) {
        *ws = moves;
        *live = L;
    }
}

constexpr int kMoveChunk = 16384;      // bytes of a page a workgroup moves at once

// The pages of the list move, layer by layer, 16 KB a workgroup and turn; every entry of the table
// follows.  489 pages of 524 KB (4 layers): 110 us, 4.7 TB/s, the rate of a large copy.
__global__ __launch_bounds__(kBlock) void k_compact_move(CacheView v, int32_t *table_out, const int32_t *ws) {
    const int64_t P = v.pages, moves = ws[0];
    const int32_t *source = ws + 1, *target = source + P, *place = target + 2 * P;
    const int64_t entries = (int64_t)v.sequences * v.row;
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < entries; i += (int64_t)gridDim.x * kBlock) {
        const int p = v.table[i];
        table_out[i] = p >= 0 && p < v.pages ? place[p] : p;
    }
    const int64_t kb = (int64_t)v.heads * v.block * v.D16, vb = (int64_t)v.heads * v.D * v.block;
    const int64_t kc = (kb + kMoveChunk - 1) / kMoveChunk, chunks = kc + (vb + kMoveChunk - 1) / kMoveChunk;
    for (int64_t i = blockIdx.x; i < moves * v.layers * chunks; i += gridDim.x) {
        const int64_t chunk = i % chunks, m = i / chunks % moves, layer = i / chunks / moves;
        const int64_t from = layer * P + source[m], to = layer * P + target[m];
        const bool is_v = chunk >= kc;
        const int64_t size = is_v ? vb : kb, at = (chunk - (is_v ? kc : 0)) * kMoveChunk;
        uint8_t *pool = is_v ? v.v_pages : v.k_pages;
        const int n = (int)min((int64_t)kMoveChunk, size - at) / 16;
        const uint4 *src = reinterpret_cast<const uint4 *>(pool + from * size + at);
        uint4 *dst = reinterpret_cast<uint4 *>(pool + to * size + at);
        uint4 held[kMoveChunk / 16 / kBlock];
#pragma unroll
        for (int h = 0; h < kMoveChunk / 16 / kBlock; ++h)
            if (h * kBlock + (int)threadIdx.x < n) held[h] = src[h * kBlock + threadIdx.x];
#pragma unroll
        for (int h = 0; h < kMoveChunk / 16 / kBlock; ++h)
            if (h * kBlock + (int)threadIdx.x < n) dst[h * kBlock + threadIdx.x] = held[h];
        if (chunk == 0)
            for (int g = threadIdx.x; g < v.heads; g += kBlock) {
                v.k_scales[to * v.heads + g] = v.k_scales[from * v.heads + g];
                v.v_scales[to * v.heads + g] = v.v_scales[from * v.heads + g];
            }
    }
}

template <typename T>
nmg_status append(const CacheView &c, int32_t layer, const int32_t *q_offsets, const int32_t *lengths,
                  const void *K, int64_t ldk, const void *V, int64_t ldv, int32_t N, hipStream_t stream) {
    const int64_t y = (int64_t)c.heads * ((c.D16 + 63) / 64);
    k_cache_append<T><<<dim3((N + 63) / 64, (int)y), kBlock, 0, stream>>>(
        c, layer, q_offsets, lengths, static_cast<const T *>(K), ldk, static_cast<const T *>(V), ldv, N);
    return launched();
}

template <typename T, bool kInt8>
nmg_status commit(const CacheView &c, const int32_t *lengths, const int32_t *kept_offsets,
                  const int32_t *kept, int32_t n_kept, int32_t *new_lengths, hipStream_t stream) {
    const int64_t y = 2 * (int64_t)c.layers * c.heads;
    const int z = kept ? 1 : std::min(c.room / c.block, 65535);
    const dim3 grid(c.sequences, (int)y, z);
    if (kept)
        k_cache_commit<T, kInt8, true><<<grid, kBlock, 0, stream>>>(c, lengths, kept_offsets, kept, n_kept, new_lengths);
    else
        k_cache_commit<T, kInt8, false><<<grid, kBlock, 0, stream>>>(c, lengths, kept_offsets, kept, n_kept, new_lengths);
    return launched();
}

template <typename T>
nmg_status fork(const CacheView &c, int32_t *lengths, const SlotList &list, int32_t count, hipStream_t stream) {
    constexpr int kE = 16 / sizeof(T);
    const int64_t units = (int64_t)c.layers * c.heads * (c.block * c.D16 / kE + c.D * c.block / kE);
    const int64_t y = std::min<int64_t>(1 + (units + kBlock - 1) / kBlock, 65535);
    k_cache_fork<T><<<dim3(count, (int)y), kBlock, 0, stream>>>(c, lengths, list);
    return launched();
}

}  // namespace

namespace nmg_internal {

nmg_status launch_cache_append(nmg_dtype dtype, const CacheView &c, int32_t layer,
                               const int32_t *q_offsets, const int32_t *lengths, const void *K,
                               int64_t ldk, const void *V, int64_t ldv, int32_t N, hipStream_t stream) {
    return dtype == NMG_F32 ? append<float>(c, layer, q_offsets, lengths, K, ldk, V, ldv, N, stream)
                            : append<_Float16>(c, layer, q_offsets, lengths, K, ldk, V, ldv, N, stream);
}

nmg_status launch_cache_commit(nmg_dtype dtype, nmg_cache_format format, const CacheView &c,
                               const int32_t *lengths, const int32_t *kept_offsets, const int32_t *kept,
                               int32_t n_kept, int32_t *new_lengths, hipStream_t stream) {
    if (dtype == NMG_F32)
        return format == NMG_CACHE_INT8
                   ? commit<float, true>(c, lengths, kept_offsets, kept, n_kept, new_lengths, stream)
                   : commit<float, false>(c, lengths, kept_offsets, kept, n_kept, new_lengths, stream);
    return format == NMG_CACHE_INT8
               ? commit<_Float16, true>(c, lengths, kept_offsets, kept, n_kept, new_lengths, stream)
               : commit<_Float16, false>(c, lengths, kept_offsets, kept, n_kept, new_lengths, stream);
}

nmg_status launch_cache_reserve(const CacheView &c, const int32_t *lengths, const int32_t *tokens,
                                int32_t *missing, hipStream_t stream) {
    k_cache_reserve<<<1, kWide, 0, stream>>>(c, lengths, tokens, missing);
    return launched();
}

nmg_status launch_cache_fork(nmg_dtype dtype, const CacheView &c, int32_t *lengths, const SlotList &list,
                             int32_t count, hipStream_t stream) {
    return dtype == NMG_F32 ? fork<float>(c, lengths, list, count, stream)
                            : fork<_Float16>(c, lengths, list, count, stream);
}

nmg_status launch_cache_free(const CacheView &c, int32_t *lengths, const SlotList &list, int32_t count,
                             hipStream_t stream) {
    k_cache_free<<<count, kBlock, 0, stream>>>(c, lengths, list);
    return launched();
}

nmg_status launch_cache_compact(const CacheView &c, int32_t *table_out, int32_t *references_out,
                                int32_t *live, int32_t *workspace, hipStream_t stream) {
    k_compact_plan<<<1, kWide, 0, stream>>>(c, references_out, live, workspace);
    nmg_status st = launched();
    if (st != NMG_OK) return st;
    k_compact_move<<<8 * device_cus(), kBlock, 0, stream>>>(c, table_out, workspace);
    return launched();
}

}  // namespace nmg_internal

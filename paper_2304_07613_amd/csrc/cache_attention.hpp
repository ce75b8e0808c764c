// cache_attention.hpp -- attention over an 8-bit cache on the matrix cores: one
// pass over pages and open tokens, online softmax; few rows with nothing staged in LDS,
// many with the decoded tiles there.
//
// The rows of a (sequence, key head) are its drafted tokens in every query head that
// shares the key head: row r = g T + t is token t of query head head * share + g.
// A workgroup of four waves has NT tiles of 16 rows; its waves take key tiles of 64
// tokens in turn, each with a running maximum, total and sum of its own, and join
// them at the end through LDS.
//
// One layout serves both products without moving a value between lanes.  Lane l
// is (x, c) = (l % 16, l / 16).
//   scores  S^T = K Q^T: matrix instruction s of the key tile (s = 0 .. 3) takes as its row x
//           the key 16 (x / 4) + 4 s + x % 4, so that lane (x, c) ends up with the
//           scores of keys 16 c + 4 s + i (i = 0 .. 3) of query row x: over all
//           s the 16 keys 16 c .. 16 c + 15.  A lane's part of a key's row is 16
//           values from feature 64 k + 16 c on (one 16-byte load of codes); the order in
//           which features are summed is the same for Q, which is loaded so once.
//   sums    O^T = V P^T: the lane's weights are those of keys 16 c .. 16 c + 15, its part of
//           V 16 values of feature 16 d + x from key 16 c on (one 16-byte load of
//           codes).
//
// A page's key scale goes into the factor of the scores, its value scale into the units of the
// sums (Pass).
//
// What bounds it (MI355X, e4m3 unless said): a cache of many tokens, the memory -- 4 sequences
// of 32768 tokens, 32 / 8 heads of 128, a token each: 54 us, 5.0 TB/s, and 7 of join.  A
// short one, the chain of a workgroup -- 8 of 512, 12 heads of 64: 8.6 us, of which
// places 1.4, queries beside the first pages 1.6, three key tiles a wave 2.1, the waves' join 1.7,
// stores 1.1.  Many rows, the vector instructions -- 63 drafted tokens over 8 caches of
// 4307 to 8191, 16 / 4 heads of 128, int8: 54 us, 490 TFLOP/s, and 14 of join; they run
// in 52% of the cycles of a busy compute unit, the matrix ones in 28%.
//
// Spilled vector registers of the variants (row tiles of 16: features / 16, row tiles): few rows, binary16
// 8, 2: 34; binary32 16, 1: 4, 8, 1: 5 and 4, 2: 33; the others none.
#pragma once

#include "cache.hpp"

namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

// Parts of a sequence's keys, at most; what the join's LDS holds of many rows
constexpr int max_parts(int rows) { return rows > 32 ? 16 : 64; }
constexpr int kPartUnits = 8;      // key tiles of a part, at least: two a wave
// A larger score moves the reference of a row's weights, and scales its sums, once it is 2^6 times
// larger: for most inputs that happens in the first tile alone, where every new maximum of one
// of 32 rows would do it nearly every time
constexpr float kSlack = 6.f;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kMinusInf = -__builtin_inff();

// ---------------------------------------------------------------- codes

// Two codes of a word (kHigh: its upper two) as binary16, exact
template <bool kInt8, bool kHigh>
__device__ __forceinline__ h2 decode2(uint32_t w) {
    if constexpr (kInt8) {
        // w holds code + 128; 0x6400 + u is 1024 + u in binary16
        const uint32_t u = __builtin_amdgcn_perm(0x64646464u, w, kHigh ? 0x07030702u : 0x07010700u);
        h2 v;
        __builtin_memcpy(&v, &u, 4);
        return v - h2{(_Float16)1152.f, (_Float16)1152.f};
    } else {
#if defined(__HIP_DEVICE_COMPILE__)
        return __builtin_bit_cast(h2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, kHigh));
#else
        return h2{};
#endif
    }
}
template <bool kInt8>
__device__ __forceinline__ h8 decode8(uint32_t a, uint32_t b) {
    if constexpr (kInt8) {
        a ^= 0x80808080u;
        b ^= 0x80808080u;
    }
    const h2 p = decode2<kInt8, false>(a), q = decode2<kInt8, true>(a);
    const h2 r = decode2<kInt8, false>(b), s = decode2<kInt8, true>(b);
    return h8{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
}
// Four codes as binary32, exact
template <bool kInt8>
__device__ __forceinline__ v4f decode4f(uint32_t w) {
    if constexpr (kInt8) {
        return v4f{(float)(int8_t)w, (float)(int8_t)(w >> 8), (float)(int8_t)(w >> 16),
                   (float)((int32_t)w >> 24)};
    } else {
#if defined(__HIP_DEVICE_COMPILE__)
        const v2f a = __builtin_bit_cast(v2f, __builtin_amdgcn_cvt_pk_f32_fp8(w, false));
        const v2f b = __builtin_bit_cast(v2f, __builtin_amdgcn_cvt_pk_f32_fp8(w, true));
        return v4f{a[0], a[1], b[0], b[1]};
#else
        return v4f{};
#endif
    }
}

__device__ __forceinline__ v4f mfma_f16(h8 a, h8 b, v4f c) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
#else
    return c;
#endif
}
__device__ __forceinline__ v4f mfma_f32(float a, float b, v4f c) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
#else
    return c;
#endif
}
// 16 bytes of a buffer at offset `at` of the lane and `first` of the wave
__device__ __forceinline__ u4 buf_load16(buf_rsrc_t r, uint32_t at, uint32_t first) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_bit_cast(u4, __builtin_amdgcn_raw_buffer_load_b128(r, at, first, 0));
#else
    return u4{};
#endif
}
__device__ __forceinline__ float exp2_fast(float x) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_exp2f(x);
#else
    return x;
#endif
}

// ------------------------------------------------------- what a workgroup has

// A workgroup's row tile, key head and part of the keys.  The lengths are on the device and the
// launch has room for any.  Up to 64 sequences: every wave counts the row tiles and key
// tiles of all, so that all parts are about equal whatever the lengths, and the
// workgroups that there are come first (else the idle ones fall on some compute
// units more than on others).
struct RowTile {
    int b, T, q0, n;        // sequence, its query columns and their first; kept tokens
    int first, rows;        // first row of the tile, rows of the sequence
    int head, part, parts;  // parts of the sequence's keys
    int64_t place;          // of the tile's first part among all parts' results
};

// Key tiles of a sequence: whole pages' first, then those of the open tokens
struct KeyTiles {
    int paged, all;         // tiles of pages, and of both
    int open, kept;         // open tokens, and how many of them are kept ones
    // In units of a page's tile, a tile of open tokens is three.  With 1 / 2 / 3 / 4: 8 single tokens over 500,
    // 12 heads of 64, 9.9 / 9.1 / 9.3 / 9.4 us; 63 over 3000, 8 heads of 128, 37.6 / 35.2 / 34.4 / 33.6; binary32
    // 5 over up to 701, 12 heads of 64, 18.7 / 18.3 / 16.9 / 19.4; others differ by 1%.
    __device__ __forceinline__ int units() const { return paged + 3 * (all - paged); }
    __device__ __forceinline__ int tile_at(int unit) const {
        return unit <= paged ? unit : paged + (unit - paged + 1) / 3;
    }
    // the tiles of a part
    __device__ __forceinline__ void range(int part, int parts, int *begin, int *end) const {
        const int per = (units() + parts - 1) / parts;
        *begin = min(all, tile_at(min(part * per, units())));
        *end = min(all, tile_at(min((part + 1) * per, units())));
    }
};
__device__ __forceinline__ KeyTiles key_tiles(const CacheAttnArgs &a, int n, int T) {
    KeyTiles k;
    const int blocks = n / a.c.block;
    k.kept = n - blocks * a.c.block;
    k.paged = blocks * (a.c.block / 64);
    k.open = (int)min((int64_t)k.kept + T, (int64_t)a.c.room);
    k.all = k.paged + (k.open + 63) / 64;
    return k;
}

__device__ __forceinline__ int wave_sum_upto(int v) {      // over this lane and those before it
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int up = __shfl_up(v, d);
        v += lane >= d ? up : 0;
    }
    return v;
}

// kJoin: index runs over row tiles and heads, else over their parts too
template <int kRows, bool kJoin>
__device__ __forceinline__ bool row_tile(const CacheAttnArgs &a, int index, RowTile &t) {
    auto inside = [&](int v) { return v < 0 ? 0 : v > a.Nq ? a.Nq : v; };
    const int lane = threadIdx.x & 63, heads = a.c.heads;
    int at;                                         // of the sequence's row tiles
    if (a.c.sequences <= 64) {
        const int b = min(lane, a.c.sequences - 1);
        const int from = inside(a.q_offsets[b]), columns = inside(a.q_offsets[b + 1]) - from;
        const int kept = cache_length(a.c, a.lengths, b);
        const int tiles = lane < a.c.sequences && columns > 0
                              ? (int)(((int64_t)columns * a.share + kRows - 1) / kRows) : 0;
        int parts = 1;
        const int tiles_upto = wave_sum_upto(tiles), all_tiles = __builtin_amdgcn_readlane(tiles_upto, 63);
        if (all_tiles > a.slots) return false;      // (offsets that are not as described)
        if (a.target > 0) {
            // parts of `per` units: about half a part more each than the units make
            const int units = key_tiles(a, kept, max(columns, 0)).units();
            float work = (float)tiles * units;
            for (int d = 32; d; d /= 2) work += __shfl_xor(work, d);
            const float aim = fmaxf((float)a.target - 0.5f * all_tiles * heads, 1.f);
            const int per = max(kPartUnits, (int)fminf(ceilf(work * heads / aim), 1e9f));
            parts = min(max_parts(kRows), (units + per - 1) / per);
            if (parts < 1) parts = 1;
        }
        const int each = kJoin ? tiles : tiles * parts;
        const int upto = kJoin ? tiles_upto : wave_sum_upto(each);
        const int total = __builtin_amdgcn_readlane(upto, 63);
        if (index >= total * heads) return false;
        const int place = kJoin ? index : xcd_tile(index, total * heads), unit = place % total;
        t.head = place / total;
        t.b = min(__popcll(__ballot(upto <= unit)), a.c.sequences - 1);
        t.q0 = __builtin_amdgcn_readlane(from, t.b);
        t.T = __builtin_amdgcn_readlane(columns, t.b);
        t.n = __builtin_amdgcn_readlane(kept, t.b);
        t.parts = __builtin_amdgcn_readlane(parts, t.b);
        const int before = unit - __builtin_amdgcn_readlane(upto - each, t.b);
        at = kJoin ? before : before % max(1, __builtin_amdgcn_readlane(tiles, t.b));
        t.part = kJoin ? 0 : before / max(1, __builtin_amdgcn_readlane(tiles, t.b));
        if (a.target > 0) {
            const int parts_upto = kJoin ? wave_sum_upto(tiles * parts) : upto;
            const int64_t all = __builtin_amdgcn_readlane(parts_upto, 63);
            t.place = t.head * all + __builtin_amdgcn_readlane(parts_upto - tiles * parts, t.b) +
                      (int64_t)at * t.parts;
            if ((t.head + 1) * all > a.part_count) return false;      // (never, of lengths that stay)
        }
    } else {
        // sequence b has the slots [first(b), first(b + 1)), first(b) = floor(offset(b) share /
        // rows) + b, at least as many as its rows fill: the last b with first(b) <=
        // slot, 64 at a time; the last step has its offsets and length too
        t.parts = max(1, min(a.target / max(1, a.slots * heads), max_parts(kRows)));
        const int slots = a.slots, parts = kJoin ? 1 : t.parts;
        if (index >= slots * parts * heads) return false;
        const int place = kJoin ? index : xcd_tile(index, slots * parts * heads), slot = place % slots;
        t.part = place / slots % parts;
        t.head = place / slots / parts;
        t.place = ((int64_t)t.head * slots + slot) * t.parts;
        int lo = 0, n = a.c.sequences, stride;
        do {
            stride = (n + 63) / 64;
            const int b = lo + min(lane * stride, n - 1);
            const int from = inside(a.q_offsets[b]), to = inside(a.q_offsets[b + 1]);
            const int kept = cache_length(a.c, a.lengths, b), first = (int)((int64_t)from * a.share / kRows) + b;
            const int found = __popcll(__ballot(lane * stride < n && first <= slot)) - 1;
            if (found < 0) return false;
            t.b = lo + found * stride;
            t.q0 = __builtin_amdgcn_readlane(from, found);
            t.T = __builtin_amdgcn_readlane(to, found) - t.q0;
            t.n = __builtin_amdgcn_readlane(kept, found);
            at = slot - __builtin_amdgcn_readlane(first, found);
            lo = t.b;
            n = min(stride, n - found * stride);
        } while (stride > 1);
    }
    if (at < 0 || t.T <= 0 || (int64_t)at * kRows >= (int64_t)t.T * a.share) return false;
    t.first = at * kRows;
    t.rows = t.T * a.share;
    return true;
}

// Tiles past `end` that no row of the tile sees are left out: without a tree a row of one
// head's tokens sees none behind its own
template <int kRows>
__device__ __forceinline__ int seen_end(const CacheAttnArgs &a, const RowTile &t, const KeyTiles &k, int end) {
    const int last = min(t.first + kRows, t.rows) - 1;
    if (a.tree || t.first / t.T != last / t.T) return end;
    return min(end, k.paged + (min(k.open, k.kept + last % t.T + 1) + 63) / 64);
}

// Which of the 16 open tokens from `first` on a drafted token sees, a bit each
__device__ __forceinline__ uint32_t seen_of(const CacheAttnArgs &a, const RowTile &t, const KeyTiles &k,
                                            int token, int first) {
    uint32_t seen = 0;
    if (a.tree) {
        // (all 16 bytes are on their way at once: places past the ends are read inside)
        const uint8_t *line = a.tree + (int64_t)(t.q0 + token) * a.ldtree;
        uint8_t b[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) b[j] = line[min(max(first + j - k.kept, 0), a.width - 1)];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const int e = first + j - k.kept;
            seen |= (uint32_t)(e < 0 || (e < a.width && b[j] != 0)) << j;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) seen |= (uint32_t)(first + j - k.kept <= token) << j;
    }
    const int left = k.open - first;                 // the others are no tokens
    return left >= 16 ? seen : left <= 0 ? 0 : seen & ((1u << left) - 1);
}

// ------------------------------------------------------------------ results

// A factor that only underflowed is not 0: infinities and NaN of sums stay what they are however
// far below the others their scores lie (what it leaves of finite sums is nothing to the others)
__device__ __forceinline__ float not_zero(float f) { return f == 0.f ? 0x1p-149f : f; }
// The root of 2^(m - top), m <= top.  Sums are multiplied by it twice: binary32 values times a
// weight of 2^-140 may still be more than others.
__device__ __forceinline__ float root_weight(float m, float top) {
    return not_zero(exp2_fast(0.5f * (m - top)));
}

// A wave's result of 16 NT rows: sums o (features x rows as the matrix instructions
// leave them), divided by the totals; maxima m and totals l per row.  A row without weight
// (l = 0) has 0 or, of a weight 0 times infinity, NaN.
template <bool kF32, int VT, int NT>
struct Result {
    v4f o[VT][NT];
    float m[NT], l[NT];

    // With another's result of the same rows, which `get(d, n)` and (m2, l2) give
    template <typename F>
    __device__ __forceinline__ void join(int n, float m2, float l2, F &&get) {
        const float top = fmaxf(m[n], m2), base = top == kMinusInf ? 0.f : top;
        // binary32: roots h, and t what is left of the factors
        const float h1 = kF32 ? root_weight(m[n], base) : 1.f, h2 = kF32 ? root_weight(m2, base) : 1.f;
        const float w1 = l[n] * (kF32 ? h1 * h1 : exp2_fast(m[n] - base)), w2 = l2 * (kF32 ? h2 * h2 : exp2_fast(m2 - base));
        const float all = w1 + w2, inv = all == 0.f ? 0.f : 1.f / all;
        const float t1 = not_zero(kF32 ? l[n] * inv * h1 : w1 * inv), t2 = not_zero(kF32 ? l2 * inv * h2 : w2 * inv);
#pragma unroll
        for (int d = 0; d < VT; ++d) {
            const v4f other = get(d, n);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[d][n][i] = o[d][n][i] * h1 * t1 + other[i] * h2 * t2;
        }
        m[n] = top;
        l[n] = all;
    }
};

// The four waves' results joined in wave 0, through LDS: two at a time
template <bool kF32, int VT, int NT>
__device__ __forceinline__ void join_waves(Result<kF32, VT, NT> &r, float *lds) {
    constexpr int kO = VT * NT * 256, kWave = kO + NT * 128;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    auto put = [&](float *to) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int d = 0; d < VT; ++d)
                *reinterpret_cast<v4f *>(to + (d * NT + n) * 256 + lane * 4) = r.o[d][n];
            to[kO + n * 128 + lane] = r.m[n];
            to[kO + n * 128 + 64 + lane] = r.l[n];
        }
    };
    auto take = [&](const float *from) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
            r.join(n, from[kO + n * 128 + lane], from[kO + n * 128 + 64 + lane], [&](int d, int m) {
                return *reinterpret_cast<const v4f *>(from + (d * NT + m) * 256 + lane * 4);
            });
    };
    if (wave >= 2) put(lds + (wave - 2) * kWave);
    __syncthreads();
    if (wave < 2) take(lds + wave * kWave);
    __syncthreads();
    if (wave == 1) put(lds);
    __syncthreads();
    if (wave == 0) take(lds);
}
constexpr int kScores = 68;        // floats of a row of scores in LDS: 64, rows four banks apart
template <int VT, int NT>
constexpr int join_floats() { return std::max(2 * (VT * NT * 256 + NT * 128), 4 * NT * 16 * kScores); }

// The lane's number, of which nothing that follows from it is kept over a loop's turns
__device__ __forceinline__ int lane_here() {
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    return lane;
}

// Floats of one part's result: a row of sums for every feature, then maxima, then totals
__host__ __device__ inline int64_t part_floats(int D, int rows) { return (int64_t)(D + 2) * rows; }

// kRows: of the row tile, of which `at` and what follows are the wave's.  again: only in the
// place of results that are not finite.  Whether the lane stored such.
template <typename T, int kRows, bool kF32, int VT, int NT>
__device__ __forceinline__ bool store_result(const CacheAttnArgs &a, const RowTile &t, int at,
                                             const Result<kF32, VT, NT> &r, bool again = false) {
    const int lane = lane_here(), x = lane % 16, c = lane / 16, D = a.c.D;
    bool odd = false;
    if constexpr (kF32)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int d = 0; d < VT; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) odd |= !(fabsf(r.o[d][n][i]) < __builtin_inff());
    auto put = [&](auto *to, float v) {
        if (!kF32 || !again || !(fabsf((float)*to) < __builtin_inff())) *to = (std::decay_t<decltype(*to)>)v;
    };
    if (t.parts > 1) {
        float *to = a.part + (t.place + t.part) * part_floats(D, kRows);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int d = 0; d < VT; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (16 * d + 4 * c + i < D)
                        put(to + (16 * d + 4 * c + i) * kRows + at + 16 * n + x, r.o[d][n][i]);
            if (c == 0 && !again) {     // (the first ones stay: another shift would only cost the join precision)
                to[D * kRows + at + 16 * n + x] = r.m[n];
                to[(D + 1) * kRows + at + 16 * n + x] = r.l[n];
            }
        }
        return odd;
    }
    T *O = static_cast<T *>(a.O);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int row = t.first + at + 16 * n + x;
        if (row >= t.rows) continue;
        const int64_t h = t.head * a.share + row / t.T;
        T *to = O + h * D * a.ldo + t.q0 + row % t.T;
#pragma unroll
        for (int d = 0; d < VT; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (16 * d + 4 * c + i < D)
                    put(to + (16 * d + 4 * c + i) * a.ldo, r.l[n] == 0.f ? 0.f : r.o[d][n][i]);
    }
    return odd;
}

// ------------------------------------------------------------------ the pass

// The larger of two; of NaN and a number either (a NaN score makes its weight NaN).  fmaxf
// would first quieten both.
__device__ __forceinline__ float larger(float a, float b) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_fmed3f(a, b, __builtin_inff());
#else
    return a;
#endif
}
// The largest of v over the four lanes (x, 0 .. 3)
__device__ __forceinline__ float max_over_c(float v) {
#if defined(__HIP_DEVICE_COMPILE__)
    const uint32_t u = __float_as_uint(v);
    auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    const uint32_t w = __float_as_uint(v);
    auto q = __builtin_amdgcn_permlane16_swap(w, w, false, false);
    return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
#else
    return v;
#endif
}
__device__ __forceinline__ float sum_over_c(float v) {
    v += __shfl_xor(v, 32);
    return v + __shfl_xor(v, 16);
}
// e of v = m 2^e, 1 <= |m| < 2; 0 for 0
__device__ __forceinline__ int exponent_of(float v) {
    return v == 0.f ? 0 : __builtin_amdgcn_frexp_expf(v) - 1;
}
// What was loaded before is loaded again, rather than kept in registers
__device__ __forceinline__ void reload() { asm volatile("" ::: "memory"); }
// 2^(x + e), 2^127 at most.  Whole powers go into the exponent: beside them x would lose bits, and below 2^-126 the
// instruction knows no numbers.
__device__ __forceinline__ float weight_at(float x, int e) {
    x = x < -1000.f ? -1000.f : x;       // (NaN stays)
    const float whole = floorf(x);
    return fminf(__builtin_ldexpf(exp2_fast(x - whole), (int)whole + e), 0x1p127f);
}
// No instruction is moved across
__device__ __forceinline__ void issued() { __builtin_amdgcn_sched_barrier(0); }

// Binary32 sums: any value of the type may meet any weight, and what is large may be what a row does not
// see, or hardly weighs.  So values keep their size, and weights are 2^kShift times larger: of their
// products with values below 2^kLarge none is lost that is 2^-148 or more.  Larger open values (there are
// hardly ever any) take weights of their own, 2^(kLarge - 1) times larger still, and the values as many
// times smaller; page scales from kLargeScale on go into the weights' exponents, with codes times 2^kCodes.
// Those weights are cut at 2^127, where their products with all but zeros are past the range anyway.  A result
// that passes the range -- of values above 2^64 or so, over the number of keys -- is made once more, with
// weights times 2^kShiftAgain, where no sum of any values does (and products below 2^-40 are lost).
constexpr int kShift = 64, kLarge = 64, kCodes = 10, kShiftAgain = -44;
constexpr float kLargeScale = 0x1p55f;

// binary16: the unit of a page's sums.  Codes times less than 2^-64 are nothing to the type, whose
// smallest number is 2^-24; and 2^31 weights of 2^15 times its largest value are 2^126 in units of 2^-64.
__device__ __forceinline__ float value_unit(float scale) { return scale < 0x1p-64f ? 0x1p-64f : scale; }

// What a wave carries from key tile to key tile, for 16 NT rows (lane (x, c): row x of
// every 16, features 16 d + 4 c + i)
template <bool kF32, int VT, int NT>
struct Pass {
    v4f o[VT][NT];          // sums of weights times values
    v4f total[NT];          // of the weights: binary16 by a matrix instruction with ones (four
                            // equal values), binary32 the lane's part
    float m[NT];            // the reference of the weights: no score so far is more than kSlack larger
    // binary16: the sums are in units of the value scale of the tile at hand, since its weights leave
    // no room for another factor.  binary32: see kShift.
    float unit;

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            m[n] = kMinusInf;
            total[n] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int d = 0; d < VT; ++d) o[d][n] = v4f{0.f, 0.f, 0.f, 0.f};
        }
        unit = 1.f;
    }
    __device__ __forceinline__ void new_unit(float vs) {
        if (vs != unit) {
            const float f = unit / vs;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int d = 0; d < VT; ++d) o[d][n] *= f;
            unit = vs;
        }
    }
    // Scores s * f (in units of log 2, f > 0) to weights, in place.  binary32 (f is 1): to their differences
    // from the reference, of which weigh makes weights.
    __device__ __forceinline__ void softmax(v4f (&s)[4][NT], float f) {
        float top[NT];
        bool up = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float t = larger(larger(s[0][n][0], s[0][n][1]), larger(s[0][n][2], s[0][n][3]));
#pragma unroll
            for (int i = 1; i < 4; ++i)
                t = larger(t, larger(larger(s[i][n][0], s[i][n][1]), larger(s[i][n][2], s[i][n][3])));
            top[n] = max_over_c(t) * f;
            up |= top[n] > m[n] + kSlack;
        }
        if (__any(up)) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const bool grows = top[n] > m[n];
                const float h = kF32 && grows ? root_weight(m[n], top[n]) : 1.f;
                const float g = kF32 ? h * h : grows ? not_zero(exp2_fast(m[n] - top[n])) : 1.f;
                m[n] = fmaxf(m[n], top[n]);
                total[n] *= g;
#pragma unroll
                for (int d = 0; d < VT; ++d) o[d][n] = kF32 ? o[d][n] * h * h : o[d][n] * g;
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            // binary16 weights are 2^15 at most, so that the small ones stay normal down to
            // 2^-23 of the reference (totals have the same factor)
            const float base = (m[n] == kMinusInf ? 0.f : m[n]) - (kF32 ? 0.f : 15.f - kSlack);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float v = s[i / 4][n][i % 4];
                s[i / 4][n][i % 4] = kF32 ? v - base : exp2_fast(__builtin_fmaf(v, f, -base));
            }
        }
    }
    // binary32: whether a row's difference is below -120, where exp2_fast may not do, and not minus infinity
    __device__ __forceinline__ static bool deep(const v4f (&s)[4][NT]) {
        uint32_t most = 0;       // of the bits of negative numbers the largest are the smallest; minus infinity, NaN become 0
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float x = s[i / 4][n][i % 4];
                most = max(most, __float_as_uint(x) + 0x800000u);
            }
        return __any(most > 0xc2f00000u + 0x800000u);
    }
    // binary32: the lane's differences to weights, those counted into the total: times f where all are plain,
    // else times f2 2^e
    __device__ __forceinline__ void weigh(v4f (&s)[4][NT], bool plain, float f, float f2, int e) {
        if (__builtin_expect(plain, 1)) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float w = exp2_fast(s[i / 4][n][i % 4]);
                    total[n][0] += w;
                    s[i / 4][n][i % 4] = w * f;
                }
        } else {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float x = s[i / 4][n][i % 4];
                    total[n][0] += exp2_fast(x);
                    s[i / 4][n][i % 4] = weight_at(x, e) * f2;
                }
        }
    }
    // binary16: the lane's 16 weights as the matrix instructions take them, and their total
    __device__ __forceinline__ void weights(const v4f (&s)[4][NT], h8 (&p)[NT][2]) {
        const h8 ones = {1, 1, 1, 1, 1, 1, 1, 1};
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int i = 0; i < 16; ++i) p[n][i / 8][i % 8] = (_Float16)s[i / 4][n][i % 4];
            total[n] = mfma_f16(ones, p[n][0], total[n]);
            total[n] = mfma_f16(ones, p[n][1], total[n]);
        }
    }
    // the sums over their totals
    __device__ __forceinline__ void finish(Result<kF32, VT, NT> &r, int shift = 0) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            r.m[n] = m[n];
            r.l[n] = kF32 ? sum_over_c(total[n][0]) : total[n][0];
            const float inv = r.l[n] == 0.f ? 0.f : 1.f / r.l[n];
#pragma unroll
            for (int d = 0; d < VT; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) r.o[d][n][i] = o[d][n][i] * inv * (kF32 ? __builtin_ldexpf(1.f, -shift) : unit);
        }
    }
};

// Open values in binary16 as the matrix instructions take them, without those that are not finite
__device__ __forceinline__ u4 finite_word(u4 y) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if ((y[e] & 0x7c00u) == 0x7c00u) y[e] &= 0xffff0000u;
        if ((y[e] & 0x7c000000u) == 0x7c000000u) y[e] &= 0xffffu;
    }
    return y;
}
// What a key's score makes of its values that are not finite: nothing where it is not seen (NaN; or the row is NaN
// already), NaN where the weight is 0, themselves else, however small the weight
__device__ __forceinline__ _Float16 odd_weight(float score) {
    return (_Float16)(score == score ? score == kMinusInf ? 16384.f : 1.f : 0.f);
}
// Those values, to the sums: by matrix instructions on numbers that tell them apart -- 1, 128 and 16384 for plus and minus
// infinity and NaN, whose sums over 64 keys do too.  w: the lane's 16 odd_weights; word(d, i): the tile's values.
template <bool kF32, int VT, int NT, typename F>
__device__ __forceinline__ void odd_values(v4f (&o)[VT][NT], int n, const h8 (&w)[2], F &&word) {
#pragma unroll 1
    for (int d = 0; d < VT; ++d) {               // (a loop, since all at once would cost registers)
        h8 kind[2];
        bool some = false;
#pragma unroll
        for (int i = 0; i < (kF32 ? 4 : 2); ++i) {
            const u4 y = word(d, i);
#pragma unroll
            for (int e = 0; e < (kF32 ? 4 : 8); ++e) {
                const uint32_t b = kF32 ? y[e] : y[e / 2] >> (16 * (e % 2)) << 16;      // (16 bits as the upper ones)
                const uint32_t size = b & 0x7fffffffu, infinite = kF32 ? 0x7f800000u : 0x7c000000u;
                const float k = size < infinite ? 0.f : size > infinite ? 16384.f : b >> 31 ? 128.f : 1.f;
                some |= size >= infinite;
                kind[kF32 ? i / 2 : i][kF32 ? 4 * (i % 2) + e : e] = (_Float16)k;
            }
        }
        if (!__any(some)) continue;
        v4f sum = {0.f, 0.f, 0.f, 0.f};
        sum = mfma_f16(kind[0], w[0], sum);
        sum = mfma_f16(kind[1], w[1], sum);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float minus = floorf(sum[i] * 0x1p-7f), plus = sum[i] - 128.f * minus;
            sum[i] = sum[i] >= 16384.f || (minus > 0.f && plus > 0.f) ? __builtin_nanf("")
                     : plus > 0.f  ? __builtin_inff()
                     : minus > 0.f ? kMinusInf
                                   : 0.f;
        }
#pragma unroll
        for (int to = 0; to < VT; ++to)
            if (to == d) o[to][n] += sum;
    }
}

// The pages of a wave's next 64 key tiles (first, first + step, ...) and their scales, a lane
// each: no load of a tile waits for a look at the table
struct Ahead {
    int64_t of;             // where the page's head lies among the heads of all pages
    float ks, vs;

    __device__ __forceinline__ void look(const CacheAttnArgs &a, const RowTile &t, int first, int step, int end) {
        const CacheView &v = a.c;
        const int tile = first + step * (int)(threadIdx.x & 63);
        of = 0;
        ks = vs = 1.f;
        if (tile < end) {
            const int p = v.table[(int64_t)t.b * v.row + min(tile / (v.block / 64), v.row - 1)];
            of = ((int64_t)a.layer * v.pages + min(max(p, 0), v.pages - 1)) * v.heads + t.head;
            ks = v.k_scales[of];
            vs = v.v_scales[of];
        }
    }
    __device__ __forceinline__ int64_t place(int i) const {
        const uint32_t lo = __builtin_amdgcn_readlane((int)of, i), hi = __builtin_amdgcn_readlane((int)(of >> 32), i);
        return (int64_t)((uint64_t)hi << 32 | lo);
    }
    __device__ __forceinline__ float scale(float of_lane, int i) const {
        return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(of_lane), i));
    }
};

// Waves of a SIMD that the registers are to leave room for
template <typename T, int VT, int NT>
constexpr int attention_waves() {
    return VT == 16 || (std::is_same<T, float>::value && VT * NT == 16) ? 1 : 2;
}

// Few rows: 16 or 32 of a workgroup, whose waves have key tiles of their own and join at the
// end.  Keys of the next tile are on their way while one is multiplied, its values from before the
// scores on.  The features of a workgroup's rows stay in registers; binary32 runs on the binary32
// matrix instructions, whose rate a single row a sequence does not reach (8 sequences of
// up to 701 tokens, 12 heads of 64, 5 drafted: 17.3 us, half of them the tile of open tokens,
// whose values are looked at before its sums).
template <typename T, int VT, int NT, bool kInt8>
__global__ __launch_bounds__(256, (attention_waves<T, VT, NT>())) void k_cache_attention(CacheAttnArgs a) {
    constexpr bool kF32 = std::is_same<T, float>::value;
    constexpr int KC = (VT + 3) / 4, W = 16 * NT;
    constexpr int kWords = kF32 ? 4 : 2;          // 16-byte words of 16 open values
    __shared__ __align__(16) float lds[join_floats<VT, NT>()];
    const int lane = threadIdx.x & 63, x = lane % 16, c = lane / 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const CacheView &v = a.c;
    const int D = v.D, D16 = v.D16, room = v.room;

    RowTile t;
    if (!row_tile<W, false>(a, blockIdx.x, t)) return;
    const int head = t.head;
    const KeyTiles kt = key_tiles(a, t.n, t.T);
    int begin, end;
    kt.range(t.part, t.parts, &begin, &end);
    if (begin >= end) return;
    end = seen_end<W>(a, t, kt, end);               // (then the part's result is that of no keys)

    // ---- pages: the first ones are asked for before the queries
    const int two = v.block == 128, paged_end = min(end, kt.paged);   // key tiles of a page: 1 << two
    const int64_t heads = v.heads;
    Ahead pages;
    // A page's part of a head is one buffer: a load takes its base from scalar registers and
    // one offset per lane, what lies behind the head reads as zeros.
    const uint32_t k_bytes = v.block * D16, v_bytes = D * v.block, past = 0x7fffffffu;
    const uint32_t k_at = (16 * (x / 4) + x % 4) * D16 + 16 * c, v_at = x * v.block + 16 * c;
    uint32_t k_off[KC];
#pragma unroll
    for (int k = 0; k < KC; ++k) k_off[k] = 64 * k + 16 * c < D16 ? k_at + 64 * k : past;
    u4 kk[4][KC];
    auto load_keys = [&](int tile, int i) {
        const buf_rsrc_t from = buf_rsrc(v.k_pages + pages.place(i) * k_bytes, k_bytes);
        const uint32_t first = (tile & two) * 64 * D16;
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int k = 0; k < KC; ++k) kk[s][k] = buf_load16(from, k_off[k], first + 4 * s * D16);
    };
    // Whether the lane had results that are not finite.  again: those alone are made, with other weights.
    auto pass = [&](const bool again) __attribute__((always_inline)) {
        const int lane = lane_here(), x = lane % 16, c = lane / 16;
        const int shift = again ? kShiftAgain : kShift;
        // A wave's tiles: open ones from the last wave on, of the pages a run of as many as make the
        // units of all waves about equal
        const int opens = end - max(begin, min(kt.paged, end)), paged = max(0, paged_end - begin);
        const int quota = (paged + 3 * opens + 3) / 4;
        int tile = begin;
        for (int w = 0; w < wave; ++w) tile += max(0, quota - 3 * ((opens + w) / 4));
        const int mine_end = min(paged_end, tile + max(0, quota - 3 * ((opens + wave) / 4)));
        if (tile < mine_end) {
            pages.look(a, t, tile, 1, mine_end);
            load_keys(tile, 0);
        }
        // queries: the lane's features 64 k + 16 c + j of row x of every row tile
        std::conditional_t<kF32, float[NT][KC][16], h8[NT][KC][2]> q;
        int qe[NT];
        int token[NT];
        {
            const T *Q = static_cast<const T *>(a.Q);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int row = min(t.first + 16 * n + x, t.rows - 1);
                token[n] = row % t.T;
                const T *from = Q + ((int64_t)(head * a.share + row / t.T) * D + 16 * c) * a.ldq + t.q0 + token[n];
                float top = 0.f;
#pragma unroll
                for (int k = 0; k < KC; ++k)
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const int d = 64 * k + 16 * c + j;
                        const T value = d < D ? *from : (T)0.f;
                        from += j < 15 ? a.ldq : 49 * a.ldq;
                        if constexpr (kF32) {
                            q[n][k][j] = value;
                            top = fmaxf(top, fabsf(value));
                        } else {
                            q[n][k][j / 8][j % 8] = value;
                        }
                    }
                qe[n] = 0;
                if constexpr (kF32) {
                    // From 2^100 on scaled to 2^60, so that no product with codes passes the range where
                    // the score itself does not.  (Others as they are: beside a large query
                    // small ones count, where they meet large keys.)
                    top = max_over_c(top);
                    if (top >= 0x1p100f && top < __builtin_inff()) qe[n] = exponent_of(top) - 60;
#pragma unroll
                    for (int k = 0; k < KC; ++k)
#pragma unroll
                        for (int j = 0; j < 16; ++j) q[n][k][j] = __builtin_ldexpf(q[n][k][j], -qe[n]);
                }
            }
        }

        Pass<kF32, VT, NT> r;
        r.clear();
        const float factor = a.scale * kLog2e;

        // ---- whole pages
        for (int at = 0; tile < mine_end; ++tile, ++at) {
            u4 vv[VT];
            const int i64 = at & 63;
            const buf_rsrc_t from = buf_rsrc(v.v_pages + pages.place(i64) * v_bytes, v_bytes);
            const uint32_t first = (tile & two) * 64;
#pragma unroll
            for (int d = 0; d < VT; ++d) vv[d] = buf_load16(from, v_at + first + 16 * d * v.block, 0);
            issued();        // before the scores: they are the time that the values have to come
            const float tile_ks = pages.scale(pages.ks, i64), vs = pages.scale(pages.vs, i64);
            const float tile_vs = kF32 ? vs : value_unit(vs);
            v4f s[4][NT];
            // (products that follow one another are of different sums: none waits for the last)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int n = 0; n < NT; ++n) s[i][n] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KC; ++k) {
                if constexpr (kF32) {
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        v4f f[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) f[i] = decode4f<kInt8>(kk[i][k][w]);
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
#pragma unroll
                                for (int n = 0; n < NT; ++n) s[i][n] = mfma_f32(f[i][j], q[n][k][4 * w + j], s[i][n]);
                    }
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const h8 f = decode8<kInt8>(kk[i][k][2 * h], kk[i][k][2 * h + 1]);
#pragma unroll
                            for (int n = 0; n < NT; ++n) s[i][n] = mfma_f16(f, q[n][k][h], s[i][n]);
                        }
                }
            }
            if (tile + 1 < mine_end) {
                if (i64 == 63) pages.look(a, t, tile + 1, 1, mine_end);
                load_keys(tile + 1, (at + 1) & 63);
            }
            issued();
            if constexpr (kF32) {
                const int ke = exponent_of(tile_ks);
                const float f = factor * __builtin_ldexpf(tile_ks, -ke);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[i][n][j] = __builtin_ldexpf(s[i][n][j] * f, qe[n] + ke);
            }
            if constexpr (kF32) {
                const int large = tile_vs > kLargeScale ? exponent_of(tile_vs) - kCodes : 0;
                r.softmax(s, 1.f);
                r.weigh(s, large == 0 && !r.deep(s), tile_vs * __builtin_ldexpf(1.f, shift),
                        large ? __builtin_ldexpf(tile_vs, -large - kCodes) : tile_vs, shift + large);
                auto sums = [&](float by) {
                    // (four features at a time, so that products that follow one another are of different sums)
#pragma unroll
                    for (int d4 = 0; d4 < VT; d4 += 4)
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            v4f g[4];
#pragma unroll
                            for (int d = d4; d < VT && d < d4 + 4; ++d) g[d - d4] = decode4f<kInt8>(vv[d][w]) * by;
#pragma unroll
                            for (int j = 0; j < 4; ++j)
#pragma unroll
                                for (int d = d4; d < VT && d < d4 + 4; ++d)
#pragma unroll
                                    for (int n = 0; n < NT; ++n)
                                        r.o[d][n] = mfma_f32(g[d - d4][j], s[w][n][j], r.o[d][n]);
                        }
                };
                if (__builtin_expect(large != 0, 0))
                    sums((float)(1 << kCodes));
                else
                    sums(1.f);
            } else {
                r.softmax(s, factor * tile_ks);
                r.new_unit(tile_vs);
                h8 p[NT][2];
                r.weights(s, p);
#pragma unroll
                for (int d = 0; d < VT; ++d) {
                    const h8 g0 = decode8<kInt8>(vv[d][0], vv[d][1]), g1 = decode8<kInt8>(vv[d][2], vv[d][3]);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        r.o[d][n] = mfma_f16(g0, p[n][0], r.o[d][n]);
                        r.o[d][n] = mfma_f16(g1, p[n][1], r.o[d][n]);
                    }
                }
            }
        }

        // ---- open tokens
        // (a single tile is wave 0's, whose result is the workgroup's)
        for (tile = max(begin, kt.paged) + (paged ? 3 - wave : wave); tile < end; tile += 4) {
            const int first = 64 * (tile - kt.paged);          // of the open tokens
            const int at_slot = (int)((uint32_t)(t.n - kt.kept + first) % (uint32_t)room);
            const int64_t ring = ((int64_t)a.layer * v.sequences + t.b) * heads + head;
            const T *kf = static_cast<const T *>(v.k_open) + (ring * room + at_slot) * D16;
            const T *vf = static_cast<const T *>(v.v_open) + ring * D * room + at_slot;
            // which of the lane's keys each of its rows sees
            uint32_t seen[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) seen[n] = seen_of(a, t, kt, token[n], first + 16 * c);
            const buf_rsrc_t key_tile = buf_rsrc(kf, 64 * D16 * sizeof(T));
            auto key_word = [&](int m, int k, int w) {
                const uint32_t at = k_off[k] == past ? past : k_off[k] * (uint32_t)sizeof(T);
                return buf_load16(key_tile, at, (4 * m * D16 + w * (16 / kWords)) * sizeof(T));
            };
            // values: those behind the open tokens are whatever the ring held, so none are taken
            const int valid = kt.open - first - 16 * c;       // of the lane's 16
            int feature = x;
            auto value_word = [&](int d, int w) {
                u4 y = 16 * d + feature < D && valid > w * (16 / kWords)
                           ? *reinterpret_cast<const u4 *>(vf + (int64_t)(16 * d + feature) * room + 16 * c +
                                                           w * (16 / kWords))
                           : u4{0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (kF32) {
                        if (4 * w + e >= valid) y[e] = 0;
                    } else {
                        if (8 * w + 2 * e >= valid) y[e] = 0;
                        if (8 * w + 2 * e + 1 >= valid) y[e] &= 0xffffu;
                    }
                }
                return y;
            };
            // Binary32 sums of products that pass the range are made once more from keys 2^kKeys times smaller: the
            // score may be inside it.  (All keys so would lose bits of the small ones.)
            constexpr int kKeys = 112;
            float *scores = lds + wave * NT * 16 * kScores;
            v4f s[4][NT];
#pragma unroll 1
            for (bool smaller = false;; smaller = true) {
                if (kF32) reload();
                const float keys_by = smaller ? __builtin_ldexpf(1.f, -kKeys) : 1.f;
                bool past = false;
#pragma unroll
                for (int m = 0; m < 4; ++m)
#pragma unroll
                    for (int n = 0; n < NT; ++n) s[m][n] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < KC; ++k)
#pragma unroll
                    for (int w = 0; w < kWords; ++w) {
                        u4 y[4];
#pragma unroll
                        for (int m = 0; m < 4; ++m) y[m] = key_word(m, k, w);
                        if constexpr (kF32) {
#pragma unroll
                            for (int e = 0; e < 4; ++e)
#pragma unroll
                                for (int m = 0; m < 4; ++m) {
                                    const float f = __uint_as_float(y[m][e]) * keys_by;
#pragma unroll
                                    for (int n = 0; n < NT; ++n) s[m][n] = mfma_f32(f, q[n][k][4 * w + e], s[m][n]);
                                }
                        } else {
#pragma unroll
                            for (int m = 0; m < 4; ++m)
#pragma unroll
                                for (int n = 0; n < NT; ++n)
                                    s[m][n] = mfma_f16(__builtin_bit_cast(h8, y[m]), q[n][k][w], s[m][n]);
                        }
                    }
#pragma unroll
                for (int m = 0; m < 4; ++m)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            // (kept for odd_values and others, which need them once they are weights)
                            float &kept = scores[(n * 16 + x) * kScores + 16 * c + 4 * m + e];
                            const bool sees = seen[n] >> (4 * m + e) & 1;
                            float y = s[m][n][e];
                            if constexpr (kF32) {
                                y = __builtin_ldexpf(y * factor, qe[n] + (smaller ? kKeys : 0));
                                if (smaller && fabsf(kept) < __builtin_inff()) y = kept;
                                past |= sees && !(fabsf(y) < __builtin_inff());
                            }
                            s[m][n][e] = sees ? y : kMinusInf;
                            kept = sees ? y : __builtin_nanf("");
                        }
                if (!kF32 || smaller || !__builtin_expect(__any(past), 0)) break;
            }
            r.softmax(s, kF32 ? 1.f : factor);
            if constexpr (kF32) r.weigh(s, !r.deep(s), __builtin_ldexpf(1.f, shift), 1.f, shift);
            // a value that is not finite, or larger than the weights are made for
            bool odd = false;
            constexpr uint32_t limit = (127 + kLarge) << 23;
            if constexpr (kF32) {
#pragma unroll 4
                for (int d = 0; d < VT; ++d)
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const u4 y = value_word(d, w);
#pragma unroll
                        for (int e = 0; e < 4; ++e) odd |= (y[e] & 0x7fffffffu) >= limit;
                    }
                reload();
            } else {
                // 0 times a value that is not finite is NaN
                v4f z = {0.f, 0.f, 0.f, 0.f};
                const h8 none = {};
#pragma unroll
                for (int d = 0; d < VT; ++d)
#pragma unroll
                    for (int w = 0; w < 2; ++w) z = mfma_f16(__builtin_bit_cast(h8, value_word(d, w)), none, z);
                reload();
                odd = z[0] != z[0] || z[1] != z[1] || z[2] != z[2] || z[3] != z[3];
                r.new_unit(1.f);
            }
            odd = __any(odd);
            // (by the words and numbers that are taken: in ordinary tiles they are not looked at)
            auto sums_f32 = [&](auto value_of) {
#pragma unroll
                for (int d4 = 0; d4 < VT; d4 += 4)
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        u4 y[4];
#pragma unroll
                        for (int d = d4; d < VT && d < d4 + 4; ++d) y[d - d4] = value_word(d, w);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
#pragma unroll
                            for (int d = d4; d < VT && d < d4 + 4; ++d)
#pragma unroll
                                for (int n = 0; n < NT; ++n)
                                    r.o[d][n] = mfma_f32(value_of(y[d - d4][e]), s[w][n][e], r.o[d][n]);
                    }
            };
            auto sums_f16 = [&](auto word_of) {
                h8 p[NT][2];
                r.weights(s, p);
#pragma unroll
                for (int d = 0; d < VT; ++d) {
                    const h8 g0 = __builtin_bit_cast(h8, word_of(value_word(d, 0)));
                    const h8 g1 = __builtin_bit_cast(h8, word_of(value_word(d, 1)));
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        r.o[d][n] = mfma_f16(g0, p[n][0], r.o[d][n]);
                        r.o[d][n] = mfma_f16(g1, p[n][1], r.o[d][n]);
                    }
                }
            };
            if (__builtin_expect(odd, 0)) {
                if constexpr (kF32) {
                    uint32_t from = 0, to = limit;
                    float by = 1.f;
#pragma unroll 1
                    for (;;) {
                        feature = lane_here() % 16;       // (no address is kept over the turns)
                        sums_f32([&](uint32_t bits) {
                            const uint32_t b = bits & 0x7fffffffu;
                            return b >= from && b < to ? __uint_as_float(bits) * by : 0.f;
                        });
                        if (from) break;
                        // the larger ones and their weights
                        from = limit;
                        to = 0x7f800000u;
                        by = __builtin_ldexpf(1.f, 1 - kLarge);
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                const float y = scores[(n * 16 + x) * kScores + 16 * c + e] - (r.m[n] == kMinusInf ? 0.f : r.m[n]);
                                s[e / 4][n][e % 4] = y == y ? weight_at(y, shift + kLarge - 1) : 0.f;
                            }
                    }
                } else {
                    sums_f16([](u4 y) { return finite_word(y); });
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    h8 w[2];
#pragma unroll
                    for (int e = 0; e < 16; ++e) w[e / 8][e % 8] = odd_weight(scores[(n * 16 + x) * kScores + 16 * c + e]);
                    odd_values<kF32>(r.o, n, w, value_word);
                }
            } else if constexpr (kF32) {
                sums_f32([](uint32_t bits) { return __uint_as_float(bits); });
            } else {
                sums_f16([](u4 y) { return y; });
            }
        }
        if (end > kt.paged) __syncthreads();     // (the waves' parts of LDS are free again)

        // ---- the wave's sums over its totals, then the four waves'
        Result<kF32, VT, NT> mine;
        r.finish(mine, shift);
        if (end - begin > 1) join_waves(mine, lds);
        return wave == 0 && store_result<T, 16 * NT>(a, t, 0, mine, again);
    };
    // (twice in the code: a loop around it kept registers from turn to turn, and spilled them)
    const bool odd = pass(false);
    if constexpr (kF32)
        if (__builtin_expect(__syncthreads_or(odd), 0)) pass(true);
}

// ------------------------------------------------- many rows (binary16)

// Barrier of a workgroup whose waves share LDS; loads from memory go on
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// The same pass where a (sequence, key head) has many rows: a wave has rows of its own, all four
// go through the same key tiles.  Each decodes a quarter of a tile -- the decoding is most of a
// tile's vector work -- and leaves it in LDS as the matrix instructions take it, 16 bytes a
// lane, so that neither side has a bank conflict.  Two buffers: while tile i is multiplied,
// tile i + 1 is decoded and tile i + 2 on its way.  Against the waves with keys of their own, 32
// rows each: 75 us in place of 88 for the 63 drafted tokens above, whose (sequence, key head) have 252
// rows each (when both were measured; 474 vector instructions a tile and wave now).
template <int VT, int NT, bool kInt8>
__global__ __launch_bounds__(256, VT == 16 ? 1 : 2) void k_cache_attention_shared(CacheAttnArgs a) {
    using T = _Float16;
    constexpr int KC = (VT + 3) / 4, W = 64 * NT, kFragments = 8 * KC + 2 * VT, VQ = (VT + 3) / 4;
    __shared__ __align__(16) h8 frag[2][kFragments][64];
    __shared__ int odd_of[4];
    const int lane = threadIdx.x & 63, x = lane % 16, c = lane / 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const CacheView &v = a.c;
    const int D = v.D, D16 = v.D16, room = v.room;

    RowTile t;
    if (!row_tile<W, false>(a, blockIdx.x, t)) return;
    const int head = t.head;
    const KeyTiles kt = key_tiles(a, t.n, t.T);
    int begin, end;
    kt.range(t.part, t.parts, &begin, &end);
    if (begin >= end) return;
    end = seen_end<W>(a, t, kt, end);               // (then the part's result is that of no keys)
    const int first_row = t.first + 16 * NT * wave;
    const bool rows = first_row < t.rows;            // the wave has some

    const int two = v.block == 128, paged_end = min(end, kt.paged);
    const int64_t heads = v.heads;
    Ahead pages;                                     // of the tile that is loaded next
    const uint32_t k_bytes = v.block * D16, v_bytes = D * v.block, past = 0x7fffffffu;
    const uint32_t k_at = (16 * (x / 4) + x % 4) * D16 + 16 * c, v_at = x * v.block + 16 * c;
    uint32_t k_off[KC];
#pragma unroll
    for (int k = 0; k < KC; ++k) k_off[k] = 64 * k + 16 * c < D16 ? k_at + 64 * k : past;
    // the wave's quarter of a tile: keys 16 (.) + 4 wave + (.), features of 16 d, d % 4 == wave
    u4 kk[KC], vv[VQ];
    float ks[3], vs[3];                              // of the tile at hand and the next two
    auto load = [&](int tile, int to) {
        const int i = (tile - begin) & 63;
        if (i == 0) pages.look(a, t, tile, 1, paged_end);
        const int64_t of = pages.place(i);
        ks[to] = pages.scale(pages.ks, i);
        vs[to] = pages.scale(pages.vs, i);
        const buf_rsrc_t from_k = buf_rsrc(v.k_pages + of * k_bytes, k_bytes);
        const buf_rsrc_t from_v = buf_rsrc(v.v_pages + of * v_bytes, v_bytes);
#pragma unroll
        for (int k = 0; k < KC; ++k) kk[k] = buf_load16(from_k, k_off[k], ((tile & two) * 64 + 4 * wave) * D16);
#pragma unroll
        for (int i = 0; i < VQ; ++i)
            vv[i] = buf_load16(from_v, v_at + (tile & two) * 64 + 16 * (wave + 4 * i) * v.block, 0);
    };
    auto decode = [&](int to) {
#pragma unroll
        for (int k = 0; k < KC; ++k) {
            frag[to][(wave * KC + k) * 2][lane] = decode8<kInt8>(kk[k][0], kk[k][1]);
            frag[to][(wave * KC + k) * 2 + 1][lane] = decode8<kInt8>(kk[k][2], kk[k][3]);
        }
#pragma unroll
        for (int i = 0; i < VQ; ++i) {
            const int d = wave + 4 * i;
            if (VT % 4 && d >= VT) continue;
            frag[to][8 * KC + 2 * d][lane] = decode8<kInt8>(vv[i][0], vv[i][1]);
            frag[to][8 * KC + 2 * d + 1][lane] = decode8<kInt8>(vv[i][2], vv[i][3]);
        }
    };
    if (begin < paged_end) load(begin, 0);

    h8 q[NT][KC][2];
    int token[NT];
    {
        const T *Q = static_cast<const T *>(a.Q);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int row = min(first_row + 16 * n + x, t.rows - 1);
            token[n] = row % t.T;
            const T *from = Q + ((int64_t)(head * a.share + row / t.T) * D + 16 * c) * a.ldq + t.q0 + token[n];
#pragma unroll
            for (int k = 0; k < KC; ++k)
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    q[n][k][j / 8][j % 8] = 64 * k + 16 * c + j < D ? *from : (T)0.f;
                    from += j < 15 ? a.ldq : 49 * a.ldq;
                }
        }
    }
    Pass<false, VT, NT> r;
    r.clear();
    const float factor = a.scale * kLog2e;

    // (products that follow one another are of different sums: none waits for the last)
    auto scores = [&](int from, v4f (&s)[4][NT]) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int n = 0; n < NT; ++n) s[i][n] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KC; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const h8 f = frag[from][(i * KC + k) * 2 + h][lane];
#pragma unroll
                    for (int n = 0; n < NT; ++n) s[i][n] = mfma_f16(f, q[n][k][h], s[i][n]);
                }
    };
    auto sums = [&](int from, const v4f (&s)[4][NT]) {
        h8 p[NT][2];
        r.weights(s, p);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int d = 0; d < VT; ++d) {
                const h8 g = frag[from][8 * KC + 2 * d + h][lane];
#pragma unroll
                for (int n = 0; n < NT; ++n) r.o[d][n] = mfma_f16(g, p[n][h], r.o[d][n]);
            }
    };

    // ---- whole pages
    if (begin < paged_end) {
        decode(0);
        if (begin + 1 < paged_end) load(begin + 1, 1);
        lds_barrier();
    }
    for (int tile = begin, buffer = 0; tile < paged_end; ++tile, buffer ^= 1) {
        const float tile_ks = ks[0], tile_vs = value_unit(vs[0]);
        if (tile + 1 < paged_end) decode(buffer ^ 1);
        if (tile + 2 < paged_end) load(tile + 2, 2);
        ks[0] = ks[1];
        vs[0] = vs[1];
        ks[1] = ks[2];
        vs[1] = vs[2];
        if (rows) {
            v4f s[4][NT];
            scores(buffer, s);
            r.softmax(s, factor * tile_ks);
            r.new_unit(tile_vs);
            sums(buffer, s);
        }
        lds_barrier();
    }

    // ---- open tokens: the next tile is on its way while one is multiplied
    const int64_t ring = ((int64_t)a.layer * v.sequences + t.b) * heads + head;
    auto first_slot = [&](int tile) {
        return (int)((uint32_t)(t.n - kt.kept + 64 * (tile - kt.paged)) % (uint32_t)room);
    };
    // 8 values of feature d, h of the lane's two words; what lies behind the open tokens is anything
    auto raw_word = [&](int tile, int d, int h) {
        const T *vf = static_cast<const T *>(v.v_open) + ring * D * room + first_slot(tile);
        return d < D && kt.open - 64 * (tile - kt.paged) - 16 * c > 8 * h
                   ? *reinterpret_cast<const u4 *>(vf + (int64_t)d * room + 16 * c + 8 * h)
                   : u4{0, 0, 0, 0};
    };
    auto cut_word = [&](int tile, u4 y, int h) {
        const int valid = kt.open - 64 * (tile - kt.paged) - 16 * c;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (8 * h + 2 * e >= valid) y[e] = 0;
            if (8 * h + 2 * e + 1 >= valid) y[e] &= 0xffffu;
        }
        return y;
    };
    auto open_word = [&](int tile, int d, int h) { return cut_word(tile, raw_word(tile, d, h), h); };
    u4 ko[KC][2], vo[VQ][2];
    uint32_t seen[NT];
    auto load_open = [&](int tile) {
        const int at_slot = first_slot(tile);
        const buf_rsrc_t key_tile = buf_rsrc(static_cast<const T *>(v.k_open) + (ring * room + at_slot) * D16,
                                             64 * D16 * sizeof(T));
#pragma unroll
        for (int k = 0; k < KC; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t from = k_off[k] == past ? past : k_off[k] * (uint32_t)sizeof(T);
                ko[k][h] = buf_load16(key_tile, from, (4 * wave * D16 + 8 * h) * sizeof(T));
            }
#pragma unroll
        for (int i = 0; i < VQ; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) vo[i][h] = raw_word(tile, 16 * (wave + 4 * i) + x, h);
    };
    int tile = max(begin, kt.paged);
    if (tile < end) load_open(tile);
    for (; tile < end; ++tile) {
        const int first = 64 * (tile - kt.paged);
#pragma unroll
        for (int k = 0; k < KC; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                frag[0][(wave * KC + k) * 2 + h][lane] = __builtin_bit_cast(h8, ko[k][h]);
        v4f z = {0.f, 0.f, 0.f, 0.f};
        auto put_values = [&](auto clean) {
#pragma unroll
            for (int i = 0; i < VQ; ++i) {
                const int d = wave + 4 * i;
                if (VT % 4 && d >= VT) continue;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const u4 y = cut_word(tile, vo[i][h], h);
                    const h8 g = __builtin_bit_cast(h8, decltype(clean)::value ? finite_word(y) : y), none = {};
                    frag[0][8 * KC + 2 * d + h][lane] = g;
                    if constexpr (!decltype(clean)::value) z = mfma_f16(g, none, z);   // NaN where a value is not finite
                }
            }
        };
        put_values(std::false_type{});
        const bool mine = __any(z[0] != z[0] || z[1] != z[1] || z[2] != z[2] || z[3] != z[3]);
        if (__builtin_expect(mine, 0)) put_values(std::true_type{});
        if (rows)
#pragma unroll
            for (int n = 0; n < NT; ++n) seen[n] = seen_of(a, t, kt, token[n], first + 16 * c);
        if (tile + 1 < end) load_open(tile + 1);
        if (lane == 0) odd_of[wave] = mine;
        lds_barrier();
        if (rows) {
            v4f s[4][NT];
            scores(0, s);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (!(seen[n] >> (4 * i + e) & 1)) s[i][n][e] = kMinusInf;
            const bool odd = odd_of[0] | odd_of[1] | odd_of[2] | odd_of[3];
            uint32_t dead[NT] = {};          // (seen keys whose weight is 0: only scores tell)
            if (__builtin_expect(odd, 0))
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 16; ++e) dead[n] |= (uint32_t)(s[e / 4][n][e % 4] == kMinusInf) << e;
            r.softmax(s, factor);
            r.new_unit(1.f);
            sums(0, s);
            if (__builtin_expect(odd, 0))
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    h8 w[2];
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        w[e / 8][e % 8] = odd_weight(!(seen[n] >> e & 1) ? __builtin_nanf("") : dead[n] >> e & 1 ? kMinusInf : 0.f);
                    odd_values<false>(r.o, n, w, [&](int d, int i) { return open_word(tile, 16 * d + x, i); });
                }
        }
        lds_barrier();
    }
    if (!rows) return;
    Result<false, VT, NT> mine;
    r.finish(mine);
    store_result<T, W>(a, t, 16 * NT * wave, mine);
}

// Parts of a row tile's keys joined.  A thread takes a row of the tile and every 256 / W-th
// feature of its workgroup's; the parts' weights are made once, in LDS.  34 MB of parts of 128 rows:
// 14 us, 16 parts of 16 rows of 32 (sequence, head): 6 us.
template <typename T, int W>
__global__ __launch_bounds__(256) void k_cache_join(CacheAttnArgs a) {
    __shared__ float root[max_parts(W)][W], weight[max_parts(W)][W];   // (maxima, totals at first)
    RowTile t;
    if (!row_tile<W, true>(a, blockIdx.x, t) || t.parts == 1) return;
    const int used = t.parts;
    const KeyTiles kt = key_tiles(a, t.n, t.T);
    constexpr int kGroups = 256 / W;
    const int row = threadIdx.x % W, g = threadIdx.x / W, D = a.c.D;
    const int64_t size = part_floats(D, W);
    const float *from = a.part + t.place * size + row;
    for (int p = g; p < used; p += kGroups) {
        int begin, end;
        kt.range(p, used, &begin, &end);             // (a part without tiles has left nothing: -1)
        root[p][row] = begin < end ? from[p * size + D * W] : kMinusInf;
        weight[p][row] = begin < end ? from[p * size + (D + 1) * W] : -1.f;
    }
    __syncthreads();
    float top = kMinusInf, all = 0.f;
    for (int p = 0; p < used; ++p) top = fmaxf(top, root[p][row]);
    const float base = top == kMinusInf ? 0.f : top;
    // binary32: of a part's factor the root and the rest (root_weight)
    constexpr bool kF32 = std::is_same<T, float>::value;
    auto root_of = [&](int p) { return kF32 ? root_weight(root[p][row], base) : exp2_fast(root[p][row] - base); };
    for (int p = 0; p < used; ++p) {
        const float l = weight[p][row], r = root_of(p);
        all += l < 0.f ? 0.f : l * r * (kF32 ? r : 1.f);
    }
    const float inv = all == 0.f ? 0.f : 1.f / all;
    __syncthreads();
    for (int p = g; p < used; p += kGroups) {
        const float l = weight[p][row], r = root_of(p);
        if (kF32) root[p][row] = r;
        weight[p][row] = l < 0.f ? -1.f : not_zero(l * inv * r);
    }
    __syncthreads();
    if (t.first + row >= t.rows) return;
    const int64_t h = t.head * a.share + (t.first + row) / t.T;
    T *to = static_cast<T *>(a.O) + h * D * a.ldo + t.q0 + (t.first + row) % t.T;
    // two features of eight parts at a time, so that many loads are on their way whatever the number of parts
    const int each = (D + gridDim.y - 1) / gridDim.y, end = min(D, ((int)blockIdx.y + 1) * each);
    for (int d = blockIdx.y * each + g; d < end; d += 2 * kGroups) {
        float o[2] = {};
        for (int p0 = 0; p0 < used; p0 += 8) {
            float v[8][2];
#pragma unroll
            for (int p = 0; p < 8; ++p)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    v[p][i] = from[min(p0 + p, used - 1) * size + min(d + i * kGroups, D - 1) * W];
#pragma unroll
            for (int p = 0; p < 8; ++p)
#pragma unroll
                for (int i = 0; i < 2; ++i) asm volatile("" : "+v"(v[p][i]));   // (loaded, whatever the weight)
#pragma unroll
            for (int p = 0; p < 8; ++p) {
                const float w = p0 + p < used ? weight[p0 + p][row] : -1.f;
                const float r = kF32 ? root[min(p0 + p, used - 1)][row] : 1.f;
#pragma unroll
                for (int i = 0; i < 2; ++i) o[i] += w < 0.f ? 0.f : v[p][i] * r * w;   // (what is not there may be anything)
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (d + i * kGroups < end) to[(d + i * kGroups) * a.ldo] = all == 0.f ? (T)0.f : (T)o[i];
    }
}

// kShared: the waves of a workgroup have rows of their own
template <typename T, int VT, int NT, bool kShared = false>
nmg_status run_cache_attention(nmg_cache_format format, const CacheAttnArgs &a, hipStream_t stream) {
    // as many as there may be: row tiles, and what they are split into
    const int64_t total = (int64_t)a.slots * a.c.heads + a.target;
    if (total > INT32_MAX / 256) return NMG_ERR_UNSUPPORTED;
    if constexpr (kShared) {
        if (format == NMG_CACHE_INT8)
            k_cache_attention_shared<VT, NT, true><<<(int)total, 256, 0, stream>>>(a);
        else
            k_cache_attention_shared<VT, NT, false><<<(int)total, 256, 0, stream>>>(a);
    } else {
        if (format == NMG_CACHE_INT8)
            k_cache_attention<T, VT, NT, true><<<(int)total, 256, 0, stream>>>(a);
        else
            k_cache_attention<T, VT, NT, false><<<(int)total, 256, 0, stream>>>(a);
    }
    nmg_status st = launched();
    if (st == NMG_OK && a.target > 0) {
        constexpr int W = (kShared ? 64 : 16) * NT;
        // workgroups for every compute unit, as far as a feature for every thread goes
        const int64_t tiles = (int64_t)a.slots * a.c.heads, most = std::max(1, a.c.D * W / 256);
        const int y = (int)std::min<int64_t>(most, std::max<int64_t>(1, 1024 / tiles));
        k_cache_join<T, W><<<dim3((int)tiles, y), 256, 0, stream>>>(a);
        st = launched();
    }
    return st;
}

}  // namespace

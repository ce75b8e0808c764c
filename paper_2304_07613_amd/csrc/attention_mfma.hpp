// attention_mfma.hpp -- attention on the matrix cores, features x tokens, one
// pass over the keys with a running maximum and sum.
//
// Orientation.  With a head's K as D x keys and Q as D x rows, both products
// have the rows as their columns:
//     S^T = K^T Q   (keys x rows),     O^T = V P^T   (D x rows)
// on 32 x 32 tiles.  A lane then holds, of one row (lane % 32), half of the
// keys of every 32 (half h = lane / 32), so maxima and sums over keys are sums
// over its own registers and one exchange between the halves, and O^T is
// stored as rows of tokens.
//
// P never moves.  The lane holds S^T[key][row] for some keys, and the second
// product wants P^T's keys of a contraction step in the lane.  Which key of a
// tile stands at which place of the contraction is free, as long as both
// operands agree:
//   binary16 (32 x 32 x 16): the places of S^T's rows are permuted by where the
//     transposing LDS read of K fetches its 4-key segments, so that half h
//     holds keys 16 c + 8 h + 0..7 of step c: 16 consecutive bytes of V's row.
//   binary32 (32 x 32 x 2): register i of half h is key 8 (i/4) + 4 h + i%4;
//     step i takes that key from each half: also 16 consecutive bytes of V.
//
// Key tiles are rows of 128 bytes (64 binary16 or 32 binary32 keys) of K and of
// V in LDS, in the matrices' own layout.  16-byte chunks of a row are permuted
// (chunk ^ swizzle(row)) so that the reads of both operands touch every bank
// once: V's reads take one chunk of 16 consecutive rows, K's (binary16) four
// chunks of 4 rows.  Tiles come with buffer loads that write LDS, which take
// any address that is a multiple of 4 bytes; binary16 rows that start between go
// through registers.
//
// Two kernels:
//   k_attn_shared  4 waves of 32 rows share key tiles: two LDS buffers, one
//                  barrier per tile, the next tile in flight.
//   k_attn_split   for few rows: the waves of a workgroup hold the same 32 rows
//                  and each walks its own key tiles, without barriers; their
//                  results are joined in LDS.
// Either may take a part of every key range (splits > 1); k_attn_join adds the
// parts.
#pragma once

#include "attention.hpp"

namespace {

typedef float f16v __attribute__((ext_vector_type(16)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;

constexpr int kRowBytes = 128;  // of a staged row
constexpr float kLog2e = 1.4426950408889634f;

// What differs between the element types.  kLift: weights are 2^kLift times
// exp(s - m), and m may lag kSlack (in powers of 2) behind the true maximum: the
// largest binary16 weight is 2^15, and weights stay normal numbers down to
// 2^-21 of the largest.  Binary16 weights are rounded to binary16, the type of the
// other operand of their product; the total that divides it is of the rounded ones.
// With the output's own rounding that is 2.3 to 2.9e-4 off (2-norm) where binary32
// weights are 2.1e-4; a second part for the lost bits would double that product.
template <typename T> struct Elem;
template <> struct Elem<_Float16> {
    static constexpr int keys = 64, per_chunk = 8;
    static constexpr float lift = 7.f, slack = 8.f;
};
template <> struct Elem<float> {
    static constexpr int keys = 32, per_chunk = 4;
    static constexpr float lift = 0.f, slack = 16.f;
};

template <typename T, bool V>
__device__ __forceinline__ int chunk_swizzle(int row) {
    if (V) return (row >> 1) & 7;
    return sizeof(T) == 2 ? ((row >> 1) & 1) * 4 : 0;
}

// One row tile and the keys its sequence has
struct RowTile {
    int q0, n;        // first query column, query columns
    int begin, end;   // keys
    int64_t row0;     // first row
};

// The sum of v over the lanes up to each, by data-parallel moves (row shifts of 1,
// 2, 4, 8 lanes, then the last lane of a row of 16 and of 32 to those after it)
__device__ __forceinline__ int sum_upto(int v) {
#if defined(__HIP_DEVICE_COMPILE__)
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
#endif
    return v;
}

// 64 sequences from b0 on, one a lane: their query columns, keys, row tiles, and
// the tiles of those up to each
template <int TR>
struct Sequences64 {
    int lo, hi, begin, end, tiles, upto;
    __device__ __forceinline__ void read(const AttnArgs &a, int b0) {
        const int lane = threadIdx.x & 63, b = b0 + lane;
        lo = hi = begin = end = 0;
        if (b < a.sequences) {
            lo = a.q_offsets[b];
            hi = a.q_offsets[b + 1];
            begin = a.kv_begin[b];
            end = a.kv_end[b];
        }
        lo = min(max(lo, 0), a.Nq);
        hi = min(max(hi, lo), a.Nq);
        begin = min(max(begin, 0), a.Nk);
        end = max(min(end, a.Nk), begin);
        tiles = (int)(((int64_t)(hi - lo) * a.share + TR - 1) / TR);
        upto = sum_upto(tiles);
    }
    __device__ __forceinline__ int total() const { return __builtin_amdgcn_readlane(upto, 63); }
};

// A workgroup's row tile of a key head, and its part of the keys
struct Place {
    int tile, part, head;
    RowTile rows;
};

// Workgroup `id` of the launch -> its place, wave-uniform; false when there is
// none (the launch has room for the most tiles that sequences of any lengths
// have).  The tiles there are go to the XCDs in equal shares, those of one
// (head, part) adjacent on one XCD: they read the same keys.
template <int TR>
__device__ __forceinline__ bool find_place(const AttnArgs &a, int id, Place &p) {
    Sequences64<TR> s;
    s.read(a, 0);
    int total = s.total();
    for (int b0 = 64; b0 < a.sequences; b0 += 64) {
        s.read(a, b0);
        total += s.total();
    }
    total = min(total, a.tiles);
    const int groups = a.splits * a.kv_heads;
    if (id >= total * groups) return false;
    id = xcd_tile(id, total * groups);
    p.tile = id % total;
    id /= total;
    p.part = id % a.splits;
    p.head = id / a.splits;
    int t = p.tile;
    for (int b0 = 0; b0 < a.sequences; b0 += 64) {
        if (a.sequences > 64) s.read(a, b0);
        const uint64_t hit = __ballot(s.upto > t);
        if (hit) {
            const int w = __builtin_ctzll(hit);
            RowTile &r = p.rows;
            r.q0 = __builtin_amdgcn_readlane(s.lo, w);
            r.n = __builtin_amdgcn_readlane(s.hi, w) - r.q0;
            r.row0 = (int64_t)(t - __builtin_amdgcn_readlane(s.upto - s.tiles, w)) * TR;
            r.begin = __builtin_amdgcn_readlane(s.begin, w);
            r.end = __builtin_amdgcn_readlane(s.end, w);
            return true;
        }
        t -= s.total();
    }
    return false;
}

// The lane's row of a tile: which query column and head.  Rows past the last
// are read as the first.
struct RowAt {
    bool valid;
    int g, column;
};
template <int TR>
__device__ __forceinline__ RowAt row_at(const AttnArgs &a, const RowTile &r, int i) {
    const int64_t row = r.row0 + i;
    RowAt x;
    x.valid = row >= 0 && row < (int64_t)r.n * a.share;
    x.g = 0;
    int t = x.valid ? (int)row : 0;
    if (a.share > 1) {  // (64-bit division is slow, and rows that need it rare)
        if ((int64_t)r.n * a.share <= INT32_MAX) {
            x.g = (int)((uint32_t)t / (uint32_t)r.n);
            t -= x.g * r.n;
        } else if (x.valid) {
            x.g = (int)(row / r.n);
            t = (int)(row - (int64_t)x.g * r.n);
        }
    }
    x.column = r.q0 + t;
    return x;
}

// v, for code that few tiles run: what is computed from it is computed there, not
// kept in registers over the whole loop
__device__ __forceinline__ int rarely(int v) {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("" : "+v"(v));
#endif
    return v;
}

// The kernel's arguments, read again: what rarely run code needs of them takes no
// registers in the loop around it.  (They are the kernel's only parameter.)
__device__ __forceinline__ AttnArgs args_again() {
#if defined(__HIP_DEVICE_COMPILE__)
    auto p = (const __attribute__((address_space(4))) AttnArgs *)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    AttnArgs a;
    __builtin_memcpy(&a, (const void *)p, sizeof a);
    return a;
#else
    return AttnArgs{};
#endif
}

// Over a row's two lanes, lane and lane ^ 32
__device__ __forceinline__ float larger_of_halves(float v) {
#if defined(__HIP_DEVICE_COMPILE__)
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                    false);
    return fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
#else
    return v;
#endif
}
__device__ __forceinline__ float sum_of_halves(float v) { return v + __shfl_xor(v, 32); }

__device__ __forceinline__ float exp2_fast(float v) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_exp2f(v);
#else
    return v;
#endif
}

__device__ __forceinline__ float log2_fast(float v) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_logf(v);
#else
    return v;
#endif
}

__device__ __forceinline__ f16v mfma(h8 a, h8 b, f16v c) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
#else
    return c;
#endif
}
__device__ __forceinline__ f16v mfma(float a, float b, f16v c) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
#else
    return c;
#endif
}
__device__ __forceinline__ s4 read_tr(lds_char *p) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4 *)p);
#else
    return s4{};
#endif
}
__device__ __forceinline__ u4 read16(lds_char *p) {
    return *(__attribute__((address_space(3))) u4 *)p;
}
__device__ __forceinline__ float read4(lds_char *p) {
    return *(__attribute__((address_space(3))) float *)p;
}
__device__ __forceinline__ void write16(lds_char *p, u4 v) {
    *(__attribute__((address_space(3))) u4 *)p = v;
}

template <int n>
__device__ __forceinline__ void wave_priority() {
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_s_setprio(n);
#endif
}

// 16 or 4 bytes at byte offset `off` (a multiple of 4) of a buffer, 0 past its end
__device__ __forceinline__ u4 load16_buf(buf_rsrc_t r, uint32_t off) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_bit_cast(u4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, 0, 0));
#else
    return u4{};
#endif
}
__device__ __forceinline__ uint32_t load4_buf(buf_rsrc_t r, uint32_t off) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_raw_buffer_load_b32(r, (int)off, 0, 0);
#else
    return 0;
#endif
}

// Wait until at most n vector-memory operations of this wave are in flight
template <int n>
__device__ __forceinline__ void wait_vm() {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((n & 0xf) | (n >> 4) << 14 | 0x7 << 4 | 0xf << 8);
    asm volatile("" ::: "memory");
#endif
}
// ... and until its LDS operations are done
__device__ __forceinline__ void wait_lds() {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xf | 0x3 << 14 | 0x7 << 4);
    asm volatile("" ::: "memory");
#endif
}

// All but the last n of this wave's copies into LDS have landed and its LDS
// accesses are done, then the workgroup barrier.  The wait is spelled out: the one
// the compiler puts before __syncthreads() counts copies into LDS among other memory
// operations, and at the head of a loop that count can leave copies of the loop's end
// in flight.
template <int n = 0>
__device__ __forceinline__ void landed_barrier() {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((n & 0xf) | (n >> 4) << 14 | 0x7 << 4);  // vmcnt(n) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
#endif
}

// One head of K or V from column `first` on, read through buffers: what lies past
// its last row or element is read as 0.  (A word that holds any byte of the head
// counts as inside.)  A head that spans less than 2^31 bytes is one buffer; WIDE:
// every 8 rows of a tile are (64-bit addresses, 32-bit offsets among the 8 rows).
template <bool WIDE>
struct HeadRows {
    const char *base;       // on 4 bytes
    int64_t end, ld;        // bytes to the end of the last row, and from row to row
    buf_rsrc_t whole;
    __device__ __forceinline__ int init(const AttnArgs &a, const void *matrix, int64_t ld_,
                                        int head, int first, int es) {
        ld = ld_ * es;
        base = (const char *)matrix + head * (int64_t)a.D * ld + (int64_t)first * es;
        const int odd = (int)((uintptr_t)base & 3);  // bytes past a multiple of 4
        base -= odd;
        end = (a.D - 1) * ld + (int64_t)(a.Nk - first) * es + odd;
        whole = part(0);
        return odd;
    }
    // from byte `from` on
    __device__ __forceinline__ buf_rsrc_t part(int64_t from) const {
        const int64_t left = min(max(end - from, (int64_t)0), (int64_t)0x7ffffff0);
        return buf_rsrc(base + from, ((uint32_t)left + 3) & ~3u);
    }
    // f(i, buffer, offset of its first row, bytes) for a wave's groups of 8 rows of
    // the tile at byte `at`: the first is `wave`, then every STEP-th
    template <int N, int STEP, typename F>
    __device__ __forceinline__ void groups(int64_t at, int wave, F f) const {
        if constexpr (!WIDE) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                // one scalar for the group and tile, not an offset register for every group
                f(i, whole, __builtin_amdgcn_readfirstlane(
                                (uint32_t)(8 * (STEP * i + wave)) * (uint32_t)ld + (uint32_t)at));
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) f(i, part(8 * (STEP * i + wave) * ld + at), 0u);
        }
    }
};

// Rows of one matrix of keys or values on their way into LDS.  STEP waves share
// a tile, this one takes every STEP-th group of 8 rows (1024 bytes).  HOW: see
// AttnRows; kAttnShift: words into registers, shifted
// by an element where the row's start is odd, and from there into LDS.
template <typename T, int DP, bool V, AttnRows HOW, int STEP>
struct Stager {
    static constexpr bool SHIFT = HOW == kAttnShift;
    static constexpr int kGroups = DP / 8 / STEP;
    // SHIFT: with few enough words to hold, a tile waits in registers from ask to
    // put; else ask takes it into LDS, 4 groups at a time
    static constexpr bool kHolds = SHIFT && DP <= 128;
    HeadRows<HOW != kAttnNarrow> rows;
    uint32_t off[STEP % 2 ? 2 : 1];  // of the lane's chunk in the wave's even and odd groups
                                     // (groups of one parity: one)
    uint32_t shift;                  // bits
    u4 hold[kHolds ? kGroups : 4];
    uint32_t next[kHolds ? kGroups : 4];

    __device__ __forceinline__ void init(const AttnArgs &a, const void *matrix, int64_t ld,
                                         int head, int first, int wave) {
        const int odd = rows.init(a, matrix, ld, head, first, sizeof(T));
        const int lane = threadIdx.x & 63, row = lane >> 3;
        const uint32_t at = (uint32_t)(row * rows.ld) + odd;
        shift = SHIFT ? (at & 2) * 8 : 0;
#pragma unroll
        for (int i = 0; i < (STEP % 2 ? 2 : 1); ++i)
            off[i] = (at & ~3u) + 16 * ((lane & 7) ^ chunk_swizzle<T, V>(8 * (STEP * i + wave) + row));
    }

    // Ask for the tile that starts `at` columns behind `first`; !kHolds: into `lds`
    __device__ __forceinline__ void ask(int at, lds_char *lds, int wave) {
        rows.template groups<kGroups, STEP>(
            (int64_t)at * (int64_t)sizeof(T), wave, [&](int i, buf_rsrc_t r, uint32_t row) {
                const uint32_t o = off[STEP % 2 ? i & 1 : 0] + row;
                if constexpr (!SHIFT) {
                    lds_copy16_buf(r, o, (void *)(lds + 1024 * (STEP * i + wave)));
                } else {
                    const int j = kHolds ? i : i % 4;
                    hold[j] = load16_buf(r, o);
                    next[j] = load4_buf(r, o + 16);
                    if (!kHolds && j == 3) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) put_group(lds, i - 3 + k, k, wave);
                        asm volatile("" ::: "memory");
                    }
                }
            });
        // waits count copies, so their order stays as written
        asm volatile("" ::: "memory");
    }
    __device__ __forceinline__ void put_group(lds_char *lds, int i, int j, int wave) {
        const int lane = threadIdx.x & 63;
        const u4 x = hold[j];
        const u4 y = {__builtin_amdgcn_alignbit(x[1], x[0], shift),
                      __builtin_amdgcn_alignbit(x[2], x[1], shift),
                      __builtin_amdgcn_alignbit(x[3], x[2], shift),
                      __builtin_amdgcn_alignbit(next[j], x[3], shift)};
        write16(lds + 1024 * (STEP * i + wave) + 16 * lane, y);
    }
    // kHolds: what was asked for, into `lds`
    __device__ __forceinline__ void put(lds_char *lds, int wave) {
        if constexpr (kHolds) {
#pragma unroll
            for (int i = 0; i < kGroups; ++i) put_group(lds, i, i, wave);
        }
    }
};

// The running sums of 32 rows in one wave, and one tile's scores: KB blocks of 32
// keys.  WIDE: the places of keys that contraction steps of 16 want.
template <int DP, int KB, bool WIDE>
struct RowSums {
    struct Scores {
        f16v s[KB];
    };
    static constexpr bool wide = WIDE;
    f16v o[DP / 32];
    float m, l;        // running maximum (of scores times log2 e), sum of the lane's weights
    float scale2;      // scale * log2 e

    __device__ __forceinline__ void clear(const AttnArgs &a) {
#pragma unroll
        for (int i = 0; i < DP / 32; ++i) o[i] = f16v{};
        m = -INFINITY;
        l = 0.f;
        scale2 = a.scale * kLog2e;
    }

    // The tile's place of register i of block kb
    static __device__ __forceinline__ int key_of(int kb, int i, int h) {
        return WIDE ? 32 * kb + 16 * (i >> 3) + 8 * h + (i & 7) : 8 * (i >> 2) + 4 * h + (i & 3);
    }

    // Leave keys out: bit j of `valid` (the lane's own) is key j of the tile
    __device__ __forceinline__ void mask(Scores &x, uint64_t valid) const {
        const int h = (threadIdx.x & 63) >> 5;
        const uint64_t mine = valid >> (WIDE ? 8 * h : 4 * h);
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                x.s[b][i] = (mine >> key_of(b, i, 0)) & 1 ? x.s[b][i] : -INFINITY;
    }

    // The running maximum of a row moves when it grew by more than `slack` powers of 2
    // (its own alone: what it is rounded by does not depend on the wave's other rows)
    __device__ __forceinline__ void raise(const Scores &x, float slack) {
        float top = x.s[0][0];
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, x.s[b][i]);
        top = larger_of_halves(top) * scale2;
        if (__any(top - m > slack)) {  // (nothing seen yet: m is -inf)
            const float next = top - m > slack ? top : m;
            const float keep = m == next ? 1.f : exp2_fast(m - next);
            l *= keep;
#pragma unroll
            for (int i = 0; i < DP / 32; ++i) o[i] *= keep;
            m = next;
        }
    }

    // Sums of binary32 values near the end of the range pass it before they are divided:
    // they are of weights up to 2^slack, and of as many as there are keys.  The loop over
    // the keys does not look; where it ends with a sum that is not finite, though the
    // row's weights are, leveled_rows takes the keys again, with the running maximum
    // raised before each tile's weights until all so far sum to 1/4: no sum passes the
    // largest value.
    __device__ __forceinline__ bool overflowed() const {
        float sum = 0.f;  // NaN if one of them is not finite
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) sum = fmaf(o[d][i], 0.f, sum);
        const float total = sum_of_halves(l);
        return !(sum == 0.f) && total - total == 0.f;
    }
    __device__ __forceinline__ void level(const Scores &x) {
        const float base = m == -INFINITY ? 0.f : m;
        float sum = l;
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) sum += exp2_fast(fmaf(x.s[b][i], scale2, -base));
        sum = sum_of_halves(sum);
        const float next = sum > 0.25f ? m + log2_fast(4.f * sum) : m;
        const float keep = m == next ? 1.f : exp2_fast(m - next);
        l *= keep;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) o[d] *= keep;
        m = next;
    }

    // exp2(score - m + lift); 0 for a row that has seen nothing
    __device__ __forceinline__ void exponentials(Scores &x, float lift) const {
        const float base = m == -INFINITY ? 0.f : m - lift;
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) x.s[b][i] = exp2_fast(fmaf(x.s[b][i], scale2, -base));
    }
};

// 32 rows of a tile in one wave
template <typename T, int DP>
struct Rows : RowSums<DP, Elem<T>::keys / 32, sizeof(T) == 2> {
    static constexpr int KT = Elem<T>::keys, KB = KT / 32;
    static constexpr int QF = sizeof(T) == 2 ? DP / 16 : DP / 2;
    typedef typename std::conditional<sizeof(T) == 2, h8, float>::type QFrag;
    typedef RowSums<DP, KB, sizeof(T) == 2> Sums;
    using Sums::l;
    using Sums::o;
    using typename Sums::Scores;
    struct Weights {
        h8 p[KT / 16];
    };
    QFrag q[QF];

    __device__ __forceinline__ void init(const AttnArgs &a, int kv_head, const RowAt &r) {
        const int h = (threadIdx.x & 63) >> 5;
        const T *src = (const T *)a.Q + (int64_t)(kv_head * a.share + r.g) * a.D * a.ldq + r.column;
        auto at = [&](int d) {
            const T v = src[min(d, a.D - 1) * a.ldq];
            return d < a.D ? v : (T)0;
        };
#pragma unroll
        for (int c = 0; c < QF; ++c) {
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int e = 0; e < 8; ++e) q[c][e] = at(16 * c + 8 * h + e);
            } else {
                q[c] = at(2 * c + h);
            }
        }
    }

    // S^T of the tile at k
    __device__ __forceinline__ void scores(Scores &x, lds_char *k) const {
        const int lane = threadIdx.x & 63, h = lane >> 5;
#pragma unroll
        for (int b = 0; b < KB; ++b) x.s[b] = f16v{};
        if constexpr (sizeof(T) == 2) {
            // segment lane % 4 of its 16 keys: 0, 8, 4, 12 (see the file's comment)
            const int row = 8 * h + ((lane & 15) >> 2), odd = (lane >> 3) & 1;
            const int at = row * kRowBytes + 16 * (2 * ((lane >> 4) & 1) + (lane & 1)) + 64 * odd +
                           8 * ((lane >> 1) & 1);
            lds_char *p0 = k + at, *p1 = k + (at ^ 64);
#pragma unroll
            for (int c = 0; c < QF; ++c) {
#pragma unroll
                for (int b = 0; b < KB; ++b) {
                    lds_char *p = (b ? p1 : p0) + 16 * kRowBytes * c;
                    struct { s4 x, y; } f = {read_tr(p), read_tr(p + 4 * kRowBytes)};
                    x.s[b] = mfma(__builtin_bit_cast(h8, f), q[c], x.s[b]);
                }
            }
        } else {
            lds_char *p = k + h * kRowBytes + 4 * (lane & 31);
#pragma unroll
            for (int c = 0; c < QF; ++c) x.s[0] = mfma(read4(p + 2 * kRowBytes * c), q[c], x.s[0]);
        }
    }

    // Scores to weights, and their sum
    __device__ __forceinline__ void weigh(Scores &x, Weights &w) {
        this->exponentials(x, Elem<T>::lift);
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int c = 0; c < KT / 16; ++c) {
#pragma unroll
                for (int e = 0; e < 8; ++e) w.p[c][e] = (_Float16)x.s[c >> 1][8 * (c & 1) + e];
                // the sum of the rounded weights: what the product divides by
#pragma unroll
                for (int e = 0; e < 8; e += 2)
                    l = __builtin_amdgcn_fdot2(h2{w.p[c][e], w.p[c][e + 1]},
                                               h2{(_Float16)1, (_Float16)1}, l, false);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) l += x.s[0][i];
        }
    }

    // O^T += V P^T
    __device__ __forceinline__ void values(const Scores &x, const Weights &w, lds_char *v) {
        const int lane = threadIdx.x & 63, h = lane >> 5, row = lane & 31;
        const int swz = chunk_swizzle<T, true>(row);
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int c = 0; c < KT / 16; ++c) {
                lds_char *at = v + row * kRowBytes + 16 * ((2 * c + h) ^ swz);
#pragma unroll
                for (int d = 0; d < DP / 32; ++d)
                    o[d] = mfma(__builtin_bit_cast(h8, read16(at + 32 * kRowBytes * d)), w.p[c], o[d]);
            }
        } else {
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                lds_char *at = v + row * kRowBytes + 16 * ((2 * b + h) ^ swz);
#pragma unroll
                for (int d = 0; d < DP / 32; ++d) {
                    const v4f y = __builtin_bit_cast(v4f, read16(at + 32 * kRowBytes * d));
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[d] = mfma(y[r], x.s[0][4 * b + r], o[d]);
                }
            }
        }
    }
};

// Which keys of the tile at column t0 take part (bit j: column t0 + j);
// `mask_byte`: the lane's key's
template <typename T>
__device__ __forceinline__ uint64_t valid_keys(const AttnArgs &a, int64_t t0, const RowTile &r,
                                               uint8_t mask_byte) {
    constexpr int KT = Elem<T>::keys;
    const int from = (int)max((int64_t)r.begin - t0, (int64_t)0);  // t0 is within KT of the range
    const int upto = (int)min((int64_t)r.end - t0, (int64_t)KT);
    const uint64_t in = (~0ull >> (64 - upto)) & (~0ull << from);
    return a.key_mask ? in & __ballot(mask_byte != 0) : in;
}

// Whether the tile's values in LDS hold an infinity or NaN: an exponent of ones and its
// least bit carry into the bit above
template <typename T, int DP>
__device__ __forceinline__ bool values_not_finite(lds_char *v) {
    constexpr uint32_t exponent = sizeof(T) == 2 ? 0x7c007c00u : 0x7f800000u;
    constexpr uint32_t least = sizeof(T) == 2 ? 0x04000400u : 0x00800000u;
    constexpr uint32_t above = sizeof(T) == 2 ? 0x80008000u : 0x80000000u;
    lds_char *at = v + 16 * rarely(threadIdx.x & 63);
    uint32_t any = 0;
#pragma unroll 4
    for (int i = 0; i < DP / 8; ++i) {
        const u4 x = read16(at + 1024 * i);
#pragma unroll
        for (int e = 0; e < 4; ++e) any |= (x[e] & exponent) + least;
    }
    return __any((any & above) != 0);
}

// Values of keys left out become 0 in LDS, whatever they hold (their weight is 0,
// but 0 x NaN is not).  Every wave that reads the tile does it for itself: they
// write the same bytes.
// A drafted key is left out by some rows and not by others: where a tile with such keys
// holds a value that is not finite (SPOILED), it becomes 0 for every row, and goes to
// the rows that see it at the end (add_not_finite).  All in one go: a wave that finds
// none any more finds the tile as the others leave it.
template <typename T, int DP, bool SPOILED>
__device__ __forceinline__ void clear_values(lds_char *v, uint64_t valid) {
    const int lane = rarely(threadIdx.x & 63);
#pragma unroll SPOILED ? 1 : DP / 8
    for (int i = 0; i < DP / 8; ++i) {
        const int row = 8 * i + (lane >> 3);
        const int key = Elem<T>::per_chunk * ((lane & 7) ^ chunk_swizzle<T, true>(row));
        const uint32_t bits = (uint32_t)(valid >> key);
        lds_char *at = v + 1024 * i + 16 * lane;
        u4 x = read16(at);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (sizeof(T) == 2) {
                const bool lo = SPOILED && (x[e] & 0x7c00u) == 0x7c00u;
                const bool hi = SPOILED && (x[e] & 0x7c000000u) == 0x7c000000u;
                x[e] &= ((bits >> (2 * e)) & 1 && !lo ? 0xffffu : 0u) |
                        ((bits >> (2 * e + 1)) & 1 && !hi ? 0xffff0000u : 0u);
            } else {
                const bool odd = SPOILED && (x[e] & 0x7f800000u) == 0x7f800000u;
                x[e] = (bits >> e) & 1 && !odd ? x[e] : 0u;
            }
        }
        write16(at, x);
    }
}

// The keys of the tile at t0 that the lane's row sees of the draft (bit j: key j;
// keys before the draft: 1).  A lane loads its key's byte of every row's line of
// the tree, a ballot makes the row's bits; AT_ONCE rows' loads are in flight
// together.  Called before the tile's copies are waited for: its waits take in
// what was asked for earlier, and must not take in the next tile's copies.
struct Draft {
    bool here;      // the tile holds drafted tokens
    uint64_t seen;
};
template <typename T, int AT_ONCE>
__device__ __forceinline__ Draft draft_at(const AttnArgs &a, const RowTile &r, const RowAt &mine,
                                          int64_t t0) {
    const int64_t drafted = (int64_t)r.end - r.n - t0;  // the draft's first key of the tile
    Draft x = {a.tree && drafted < Elem<T>::keys, ~0ull};
    if (!x.here) return x;
    const int lane = rarely(threadIdx.x & 63);
    const int at = lane - (int)max(drafted, (int64_t)(64 - INT32_MAX));
    const int from = min(max(at, 0), a.width - 1);
    const int line = mine.column * (int)a.ldtree;  // (a tree of 2^31 bytes or more is refused)
#pragma unroll 1
    for (int i0 = 0; i0 < 32; i0 += AT_ONCE) {
        int seen[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i)
            seen[i] = a.tree[(uint32_t)(__builtin_amdgcn_readlane(line, i0 + i) + from)] |
                      (at < 0 ? 1 : 0);
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const uint64_t bits = __ballot((seen[i] != 0) & (at < a.width));
            if ((lane & 31) == i0 + i) x.seen = bits;
        }
    }
    return x;
}

// Infinities and NaN as numbers whose sums over some keys tell which were among them:
// 1 for infinity, 128 for minus infinity, both for NaN, 0 for what is finite
__device__ __forceinline__ float code_of(float v) {
    return v - v == 0.f ? 0.f : v == INFINITY ? 1.f : v == -INFINITY ? 128.f : 129.f;
}

// What is not finite of the draft's values in the tiles lo, lo + STEP .. below hi
// (from column `first` on), to the sums of the rows that see its key: a product of 1
// for a key that is seen and the value's code.  From memory, after the last tile: it
// is rare, and in the loop its registers cost a workgroup a compute unit (32 sequences
// of 1024 columns, 12 heads x 64: 135 -> 146 us).
template <typename T, int DP, int STEP>
__device__ __forceinline__ void add_not_finite(const AttnArgs &a, const RowTile &r, const RowAt &mine,
                                               int head, int first, int lo, int hi,
                                               f16v (&o)[DP / 32]) {
    constexpr int KT = Elem<T>::keys;
    const int lane = rarely(threadIdx.x & 63), h = lane >> 5;
    const int64_t draft = (int64_t)r.end - r.n;  // its first column
    const uint8_t *line = a.tree + rarely(mine.column) * a.ldtree;
    const int64_t from = max((int64_t)lo * KT, (max(draft - first, (int64_t)0)) & ~15ll);
    for (int64_t k = from; k < (int64_t)hi * KT; k += 16) {
        if (STEP > 1 && ((int)(k / KT) - lo) % STEP) continue;
        const int64_t key = first + k + 8 * h;
        const int64_t i0 = key - draft;
        h8 one;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int64_t i = i0 + e;
            one[e] = i >= 0 && i < a.width && key + e >= r.begin && key + e < r.end && line[i]
                         ? (_Float16)1 : (_Float16)0;
        }
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) {
            const int row = 32 * d + (lane & 31);
            const T *src = (const T *)a.V + ((int64_t)head * a.D + row) * a.ldv + key;
            h8 code;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                code[e] = (_Float16)(row < a.D && key + e < r.end ? code_of((float)src[e]) : 0.f);
            const f16v codes = mfma(code, one, f16v{});
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int n = (int)codes[i];
                if (n & 127) o[d][i] += INFINITY;
                if (n >> 7) o[d][i] -= INFINITY;
            }
            asm volatile("" ::: "memory");  // one block at a time: registers are short here
        }
    }
}

// Scores of keys that take no part in a tile become -inf; true when there are
// keys whose values have to be cleared
template <typename T, typename W>
__device__ __forceinline__ bool settle(const W &w, typename W::Scores &x, uint64_t valid,
                                       const Draft &draft) {
    const bool full = valid == (Elem<T>::keys == 64 ? ~0ull : 0xffffffffull);
    if (!full || draft.here) w.mask(x, valid & draft.seen);
    return !full;
}

// The mask byte of the lane's key of the tile at t0 (1 without a mask)
__device__ __forceinline__ uint8_t mask_at(const AttnArgs &a, int64_t t0) {
    if (!a.key_mask) return 1;
    const int64_t c = t0 + (threadIdx.x & 63);
    return c < a.Nk ? a.key_mask[c] : 0;
}

// Scores of the 32 keys at column c0 from memory, by the binary32 instructions
template <bool WIDE>
__device__ __forceinline__ void scores_from_memory(const AttnArgs &a, f16v &x, int head,
                                                   const RowAt &mine, int64_t c0) {
    const int lane = rarely(threadIdx.x & 63), h = lane >> 5, row = lane & 31;
    // the key of S^T's row lane % 32
    const int key =
        WIDE ? 16 * (row >> 4) + 8 * ((row >> 2) & 1) + 4 * ((row >> 3) & 1) + (row & 3) : row;
    const float *k = (const float *)a.K + (int64_t)head * a.D * a.ldk + c0;
    const float *q = (const float *)a.Q + (int64_t)(head * a.share + mine.g) * a.D * a.ldq + mine.column;
    x = f16v{};
    for (int d = h; d < a.D + h; d += 2) {
        const bool in = d < a.D;
        const float y = in && key < a.Nk - c0 ? k[d * a.ldk + key] : 0.f;
        const float z = in ? q[d * a.ldq] : 0.f;
        x = mfma(y, z, x);
    }
}

// Sums of the values of the 32 keys at column c0 (those in `valid`) from memory, by the
// same instructions; `finite`: infinities and NaN left out (see clear_values)
template <int DP, typename Sums>
__device__ __forceinline__ void values_from_memory(const AttnArgs &a, Sums &w,
                                                   const typename Sums::Scores &x, int head,
                                                   int64_t c0, uint64_t valid, bool finite) {
    const int lane = rarely(threadIdx.x & 63), h = lane >> 5;
    const float *v = (const float *)a.V + (int64_t)head * a.D * a.ldv + c0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int key = Sums::key_of(0, i, h);
        const bool in = (valid >> key) & 1;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) {
            const int row = 32 * d + (lane & 31);
            float y = in && row < a.D ? v[row * a.ldv + key] : 0.f;
            if (finite && y - y != 0.f) y = 0.f;
            w.o[d] = mfma(y, x.s[0][i], w.o[d]);
        }
        asm volatile("" ::: "memory");  // few loads at once: registers are short here
    }
}

// The wave's rows over the tiles lo, lo + step .. below hi once more, from memory, for
// sums that passed the largest number (RowSums::level)
template <int DP, typename Sums>
__device__ __forceinline__ void leveled_rows(const AttnArgs &a, const RowTile &r, const RowAt &mine,
                                             int head, int first, int lo, int hi, int step, Sums &w) {
    w.clear(a);
#pragma unroll 1
    for (int t = lo; t < hi; t += step) {
        const int64_t t0 = (int64_t)first + (int64_t)t * Elem<float>::keys;
        const uint64_t valid = valid_keys<float>(a, t0, r, mask_at(a, t0));
        const Draft draft = draft_at<float, 8>(a, r, mine, t0);
        typename Sums::Scores x;
        scores_from_memory<Sums::wide>(a, x.s[0], head, mine, t0);
        settle<float>(w, x, valid, draft);
        w.raise(x, Elem<float>::slack);
        w.level(x);
        w.exponentials(x, Elem<float>::lift);
#pragma unroll
        for (int i = 0; i < 16; ++i) w.l += x.s[0][i];
        values_from_memory<DP>(a, w, x, head, t0, valid, draft.here);
    }
}

// The order of a step's instructions: the next scores' matrix instructions
// between the weights' vector instructions, LDS reads ahead of their use, then
// the product with V (4096 x 16384 at 64: 340 -> 323 us)
template <typename T, int DP>
__device__ __forceinline__ void interleave() {
#if defined(__HIP_DEVICE_COMPILE__)
    if constexpr (sizeof(T) == 2) {
        constexpr int kScores = DP / 16 * 2, kValues = DP / 32 * 4, kVector = 96 / kScores;
        __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
        for (int i = 0; i < kScores; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x002, kVector, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
#pragma unroll
        for (int i = 0; i < kValues; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
    }
#endif
}

// Parts in the workspace: means (padded D x rows), then maxima and totals, of every
// (part, head, tile).  (Sums of parts could pass the largest number, means do not.)
template <int DP, int TR>
__device__ __forceinline__ float *part_at(const AttnArgs &a, int part, int head, int tile) {
    return a.part + (((int64_t)part * a.kv_heads + head) * a.tiles + tile) * ((DP + 2) * TR);
}

// The end of a wave of 32 rows: its outputs, or its part of them
template <typename T, int DP, typename W>
__device__ __forceinline__ void finish(const AttnArgs &a, const Place &at, const RowAt &mine,
                                       const W &w, int wave) {
    constexpr int TR = kAttnSharedRows;
    const int lane = threadIdx.x & 63;
    const int h = lane >> 5;
    const float total = sum_of_halves(w.l);
    const float inv = total == 0.f ? 0.f : 1.f / total;
    if (a.splits > 1) {
        float *part = part_at<DP, TR>(a, at.part, at.head, at.tile) + 32 * wave + (lane & 31);
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                part[(32 * d + 8 * (i >> 2) + 4 * h + (i & 3)) * TR] = w.o[d][i] * inv;
        if (h == 0) {
            part[DP * TR] = w.m;
            part[(DP + 1) * TR] = total;
        }
        return;
    }
    if (!mine.valid) return;
    T *out = (T *)a.O + (int64_t)(at.head * a.share + mine.g) * a.D * a.ldo + mine.column;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int row = 32 * d + 8 * (i >> 2) + 4 * h + (i & 3);
            if (row < a.D) out[row * a.ldo] = (T)(w.o[d][i] * inv);
        }
}

// 4 waves of 32 rows over shared key tiles.  128 rows read a key tile once: 64
// multiplications a byte of K and V in binary16 (8 TB/s from the L2s at the rate below,
// where the workgroups of a head on one XCD find each other's tiles), so the matrix
// pipe is the bound where there are workgroups enough: 16 / 4 heads x 128, 4096 columns
// over 16384 keys, 520 us = 1060 TFLOP/s (a large library product 1330), matrix
// instructions in 64% of the cycles, the rest the softmax's vector instructions that
// find no matrix instruction beside them.  2 workgroups on a compute unit: one's barriers and first tiles lie
// under the other's steps (a third: 515 -> 543 us); heads up to 64 have room for a
// third (32 sequences of 1024 columns, 12 heads x 64: 158 us with two, 143 with three).
template <typename T, int DP, AttnRows HOW>
__global__ __launch_bounds__(256, DP <= 64 && HOW != kAttnShift ? 3 : DP <= (HOW == kAttnShift ? 96 : 128) ? 2 : 1) void k_attn_shared(AttnArgs a) {
    constexpr int TR = kAttnSharedRows, KT = Elem<T>::keys, kTile = DP * kRowBytes;
    constexpr bool SHIFT = HOW == kAttnShift;
    // variables of their own: the compiler sees that reads of one do not touch
    // copies into another still in flight
    __shared__ __attribute__((aligned(1024))) char lds_k0[kTile];
    __shared__ __attribute__((aligned(1024))) char lds_k1[kTile];
    __shared__ __attribute__((aligned(1024))) char lds_v0[kTile];
    __shared__ __attribute__((aligned(1024))) char lds_v1[kTile];
    __shared__ int odd;  // a wave found a drafted value that is not finite
    Place at;
    if (!find_place<TR>(a, blockIdx.x, at)) return;
    const RowTile &r = at.rows;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const RowAt mine = row_at<TR>(a, r, 32 * wave + (lane & 31));
    Rows<T, DP> w;
    w.clear(a);

    const int first = r.begin - r.begin % a.align;
    const int tiles = r.end > r.begin ? (r.end - first + KT - 1) / KT : 0;
    const int lo = (int)((int64_t)tiles * at.part / a.splits);
    const int hi = (int)((int64_t)tiles * (at.part + 1) / a.splits);
    if (lo < hi) {
        if (threadIdx.x == 0) odd = 0;
        Stager<T, DP, false, HOW, 4> ks;
        Stager<T, DP, true, HOW, 4> vs;
        ks.init(a, a.K, a.ldk, at.head, first, wave);
        vs.init(a, a.V, a.ldv, at.head, first, wave);
        uint8_t byte;
        // The scores of tile t + 1 are taken while tile t's become weights: matrix
        // and vector instructions of one wave side by side.
        typename Rows<T, DP>::Scores s0, s1;
        typename Rows<T, DP>::Weights p;
        auto valid_at = [&](int t, uint8_t b) {
            return valid_keys<T>(a, (int64_t)first + (int64_t)t * KT, r, b);
        };
        // K of tile t + 1 and V of tile t are under way
        auto step = [&](auto more, int t, typename Rows<T, DP>::Scores &cur,
                        typename Rows<T, DP>::Scores &nxt, lds_char *k_cur, lds_char *k_nxt,
                        lds_char *v_cur, lds_char *v_nxt) {
            const Draft draft =
                draft_at<T, 8>(a, r, mine, (int64_t)first + (int64_t)t * KT);
            landed_barrier();  // they have landed; the buffers of K of tile t, V of t - 1 are free
            const uint64_t valid = valid_at(t, byte);
            if (more) {
                byte = mask_at(a, (int64_t)first + (int64_t)(t + 1) * KT);
                if (t + 2 < hi) ks.ask((t + 2) * KT, k_cur, wave);
                vs.ask((t + 1) * KT, v_nxt, wave);
            }
            const bool clear = settle<T>(w, cur, valid, draft);
            const bool spoiled = draft.here && values_not_finite<T, DP>(v_cur);
            if (spoiled) {
                odd = 1;
                clear_values<T, DP, true>(v_cur, valid);
            } else if (clear) {
                clear_values<T, DP, false>(v_cur, valid);
            }
            w.raise(cur, Elem<T>::slack);
            // before the other wave of the SIMD while the matrix pipe has work for
            // this one (4096 x 16384 at 128: 546 -> 515 us)
            wave_priority<1>();
            if (more) w.scores(nxt, k_nxt);
            w.weigh(cur, p);
            w.values(cur, p, v_cur);
            if (more) interleave<T, DP>();
            wave_priority<0>();
            if (SHIFT && more) {
                if (t + 2 < hi) ks.put(k_cur, wave);
                vs.put(v_nxt, wave);
            }
        };
        lds_char *k0 = (lds_char *)lds_k0, *k1 = (lds_char *)lds_k1;
        lds_char *v0 = (lds_char *)lds_v0, *v1 = (lds_char *)lds_v1;
        // K of the first tile and Q on the way together, then the copies that the
        // first step waits for
        ks.ask(lo * KT, k0, wave);
        w.init(a, at.head, mine);
        byte = mask_at(a, (int64_t)first + (int64_t)lo * KT);
        ks.put(k0, wave);
        vs.ask(lo * KT, v0, wave);
        if (!SHIFT && lo + 1 < hi) {
            ks.ask((lo + 1) * KT, k1, wave);
            landed_barrier<2 * decltype(ks)::kGroups>();
        } else {
            landed_barrier<SHIFT ? 0 : decltype(vs)::kGroups>();
        }
        w.scores(s0, k0);
        if (SHIFT) {
            vs.put(v0, wave);
            if (lo + 1 < hi) ks.ask((lo + 1) * KT, k1, wave);
            if (lo + 1 < hi) ks.put(k1, wave);
        }
        constexpr std::true_type on{};
        constexpr std::false_type off{};
        int t = lo;
        lds_char *last = v0;
        while (t + 1 < hi) {
            step(on, t++, s0, s1, k0, k1, v0, v1);
            if (t + 1 == hi) {
                s0 = s1;
                last = v1;
                break;
            }
            step(on, t++, s1, s0, k1, k0, v1, v0);
        }
        step(off, t, s0, s1, k0, k1, last, v0);
        if constexpr (sizeof(T) == 4)
            if (__any(w.overflowed())) leveled_rows<DP>(args_again(), r, mine, at.head, first, lo, hi, 1, w);
        if (a.tree) {
            __syncthreads();
            if (__builtin_amdgcn_readfirstlane(odd))
                add_not_finite<T, DP, 1>(args_again(), r, mine, at.head, first, lo, hi, w.o);
        }
    }

    finish<T, DP>(a, at, mine, w, wave);
}

// The waves of a workgroup split the keys of 32 rows, and join over LDS at the end.
// For few rows: what counts are the bytes of K and V, and before them the chain of
// loads a workgroup starts with.  32 / 8 heads x 128, 16 sequences of 1 column over 8192
// keys: 127 us = 4.2 TB/s (a large copy 4.9); 12 heads x 64, 8 of 1 over 512: 7.4 us,
// most of it the launch, the places and the join.  No barriers before the join: the
// waves' copies run apart, two tiles a wave on the way.
template <typename T, int DP, AttnRows HOW>
__global__ __launch_bounds__(64 * attn_split_waves(DP), 1) void k_attn_split(AttnArgs a) {
    constexpr int TR = kAttnSplitRows, KT = Elem<T>::keys, kTile = DP * kRowBytes;
    constexpr bool SHIFT = HOW == kAttnShift;
    constexpr int W = attn_split_waves(DP);
    __shared__ __attribute__((aligned(1024))) char lds_k[W * kTile];
    __shared__ __attribute__((aligned(1024))) char lds_v[W * kTile];
    __shared__ float tops[W][TR], totals[W][TR];
    Place at;
    if (!find_place<TR>(a, blockIdx.x, at)) return;
    const RowTile &r = at.rows;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const RowAt mine = row_at<TR>(a, r, lane & 31);
    Rows<T, DP> w;
    w.clear(a);

    const int first = r.begin - r.begin % a.align;
    const int tiles = r.end > r.begin ? (r.end - first + KT - 1) / KT : 0;
    const int lo = (int)((int64_t)tiles * at.part / a.splits) + wave;
    const int hi = (int)((int64_t)tiles * (at.part + 1) / a.splits);
    lds_char *k = (lds_char *)lds_k + wave * kTile, *v = (lds_char *)lds_v + wave * kTile;
    if (lo < hi) {
        Stager<T, DP, false, HOW, 1> ks;
        Stager<T, DP, true, HOW, 1> vs;
        constexpr int kCopies = DP / 8;
        ks.init(a, a.K, a.ldk, at.head, first, 0);
        vs.init(a, a.V, a.ldv, at.head, first, 0);
        bool odd = false;  // the wave found a drafted value that is not finite
        ks.ask(lo * KT, k, 0);
        w.init(a, at.head, mine);
        uint8_t byte = mask_at(a, (int64_t)first + (int64_t)lo * KT);
        ks.put(k, 0);
        vs.ask(lo * KT, v, 0);
        for (int t = lo; t < hi; t += W) {
            const int64_t t0 = (int64_t)first + (int64_t)t * KT;
            const bool more = t + W < hi;
            const uint8_t now = byte;
            const Draft draft = draft_at<T, 32>(a, r, mine, t0);
            if (!SHIFT) wait_vm<kCopies>();  // K has landed; V may still be in flight
            typename Rows<T, DP>::Scores x;
            typename Rows<T, DP>::Weights p;
            w.scores(x, k);
            wait_lds();  // K's tile has been read
            vs.put(v, 0);
            if (more) {
                byte = mask_at(a, t0 + (int64_t)W * KT);
                ks.ask((t + W) * KT, k, 0);
            }
            const uint64_t valid = valid_keys<T>(a, t0, r, now);
            const bool clear = settle<T>(w, x, valid, draft);
            w.raise(x, Elem<T>::slack);
            w.weigh(x, p);
            if (!SHIFT) {
                if (more)
                    wait_vm<kCopies>();
                else
                    wait_vm<0>();
            }
            const bool spoiled = draft.here && values_not_finite<T, DP>(v);
            if (spoiled) {
                odd = true;
                clear_values<T, DP, true>(v, valid);
            } else if (clear) {
                clear_values<T, DP, false>(v, valid);
            }
            w.values(x, p, v);
            wait_lds();  // V's too
            if (more) {
                ks.put(k, 0);
                vs.ask((t + W) * KT, v, 0);
            }
        }
        if constexpr (sizeof(T) == 4)
            if (__any(w.overflowed())) leveled_rows<DP>(args_again(), r, mine, at.head, first, lo, hi, W, w);
        if (odd) add_not_finite<T, DP, W>(a, r, mine, at.head, first, lo, hi, w.o);
    }

    // join the waves: maxima and totals, then sums at the common maximum, divided by the
    // total of all first (sums of finite sums could pass the largest number)
    const int h = lane >> 5, row = lane & 31;
    const float total = sum_of_halves(w.l);
    if (h == 0) {
        tops[wave][row] = w.m;
        totals[wave][row] = total;
    }
    __syncthreads();
    float top = tops[0][row];
#pragma unroll
    for (int i = 1; i < W; ++i) top = fmaxf(top, tops[i][row]);
    auto weight_of = [&](float m) { return m == -INFINITY ? 0.f : exp2_fast(m - top); };
    float all = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) all += weight_of(tops[i][row]) * totals[i][row];
    const float f = all == 0.f ? 0.f : weight_of(w.m) / all;
    static_assert(DP * TR * 4 == kTile, "a wave's sums take the place of its keys");
    float *sums = (float *)(lds_k + wave * kTile);
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i)
            sums[(32 * d + 8 * (i >> 2) + 4 * h + (i & 3)) * TR + row] = f * w.o[d][i];
    __syncthreads();
    float *part = part_at<DP, TR>(a, at.part, at.head, at.tile) + row;
    if (a.splits > 1 && threadIdx.x < TR) {
        part[DP * TR] = top;
        part[(DP + 1) * TR] = all;
    }
    T *out = (T *)a.O + (int64_t)(at.head * a.share + mine.g) * a.D * a.ldo + mine.column;
    for (int d = threadIdx.x / TR; d < DP; d += 2 * W) {
        float x = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) x += ((const float *)(lds_k + i * kTile))[d * TR + row];
        if (a.splits > 1)
            part[d * TR] = x;
        else if (mine.valid && d < a.D)
            out[d * a.ldo] = (T)x;
    }
}

// Parts of every key range, in their order, to outputs: a workgroup per (tile,
// head, a.join_rows rows of the head).  Reads every part once (32 heads x 128, 252
// columns in 8 parts: 34 MB, 11 us); few rows wait for two chains of loads, maxima and
// sums, 3-4 us with the launch.
template <typename T, int DP, int TR>
__global__ __launch_bounds__(kBlock) void k_attn_join(AttnArgs a) {
    AttnArgs one = a;
    one.splits = 1;
    Place at;
    if (!find_place<TR>(one, blockIdx.x, at)) return;
    const RowTile &r = at.rows;
    const int tile = at.tile, head = at.head;
    // of every part and row (as much LDS as there are parts: 2 workgroups fewer a
    // compute unit cost the join of 8 parts 5 us)
    extern __shared__ float join_lds[];
    float(*weights)[TR] = (float(*)[TR])join_lds;
    float(*totals)[TR] = weights + a.splits;
    const int64_t step = (int64_t)a.kv_heads * a.tiles * ((DP + 2) * TR);
    const float *part = part_at<DP, TR>(a, 0, head, tile);
    // every part's maxima and totals at once
    for (int x = threadIdx.x; x < a.splits * TR; x += kBlock) {
        weights[x / TR][x % TR] = part[(x / TR) * step + DP * TR + x % TR];
        totals[x / TR][x % TR] = part[(x / TR) * step + (DP + 1) * TR + x % TR];
    }
    __syncthreads();
    const int i = threadIdx.x % TR;
    if (threadIdx.x < TR) {
        float top = -INFINITY, all = 0.f;
        for (int s = 0; s < a.splits; ++s) top = fmaxf(top, weights[s][i]);
        for (int s = 0; s < a.splits; ++s) {
            const float m = weights[s][i];
            const float f = (m == -INFINITY ? 0.f : exp2_fast(m - top)) * totals[s][i];
            weights[s][i] = f;
            all += f;
        }
        totals[0][i] = all == 0.f ? 0.f : 1.f / all;
    }
    __syncthreads();
    const RowAt mine = row_at<TR>(a, r, i);
    if (!mine.valid) return;
    const float inverse = totals[0][i];
    T *out = (T *)a.O + (int64_t)(head * a.share + mine.g) * a.D * a.ldo + mine.column;
    const int d0 = blockIdx.y * a.join_rows;
    for (int d = d0 + threadIdx.x / TR; d < d0 + a.join_rows && d < a.D; d += kBlock / TR) {
        float x = 0.f;
#pragma unroll 8
        for (int s = 0; s < a.splits; ++s)
            x += weights[s][i] * inverse * part[s * step + d * TR + i];
        out[d * a.ldo] = (T)x;
    }
}

// The launch of a call's main kernel
template <typename T, int DP>
void launch_main(const AttnArgs &a, bool shared, AttnRows how, dim3 grid, hipStream_t stream);

template <typename T, int DP>
nmg_status launch_attn_dim(const AttnArgs &a, bool shared, AttnRows how, hipStream_t stream) {
    launch_main<T, DP>(a, shared, how, dim3((unsigned)(a.tiles * a.splits * a.kv_heads)), stream);
    if (a.splits > 1) {
        const dim3 join((unsigned)(a.tiles * a.kv_heads),
                        (unsigned)((a.D + a.join_rows - 1) / a.join_rows));
        const int tr = shared ? kAttnSharedRows : kAttnSplitRows;
        const size_t lds = (size_t)a.splits * tr * 2 * sizeof(float);  // 64 KB at most
        if (shared)
            hipLaunchKernelGGL((k_attn_join<T, DP, kAttnSharedRows>), join, dim3(kBlock), lds,
                               stream, a);
        else
            hipLaunchKernelGGL((k_attn_join<T, DP, kAttnSplitRows>), join, dim3(kBlock), lds,
                               stream, a);
    }
    return launched();
}

template <typename T>
nmg_status launch_attn(const AttnArgs &a, bool shared, AttnRows how, hipStream_t stream) {
    switch (attn_padded_dim(a.D)) {
        case 32: return launch_attn_dim<T, 32>(a, shared, how, stream);
        case 64: return launch_attn_dim<T, 64>(a, shared, how, stream);
        case 96: return launch_attn_dim<T, 96>(a, shared, how, stream);
        case 128: return launch_attn_dim<T, 128>(a, shared, how, stream);
        default: return launch_attn_dim<T, 256>(a, shared, how, stream);
    }
}

}  // namespace

// attention_parts.hpp -- binary32 attention on the bfloat16 matrix instructions.
//
// A binary32 number is the sum of three bfloat16 numbers, exactly: its leading 8
// significant bits, the next 8 and the last 8, each cut off (not rounded) by
// taking the upper half of the remainder's bits.  With x = x0 + x1 + x2 and
// y = y0 + y1 + y2 the product is taken as
//     x0 y0 + x0 y1 + x1 y0 + x1 y1 + x0 y2 + x2 y0,
// six exact products summed in binary32; what is left out is at most 2^-21 of
// |x y| and 2^-24 in the mean, of the product's sign, so that most of it goes
// with the division by the sum of the weights.  bfloat16 has binary32's range:
// no scaling.  Six products at 16 times the binary32 matrix rate are 2.7 times
// as fast.  12 heads x 64, 8 sequences of 1024 columns over 1024 keys: 153 us = 168
// TFLOP/s (a large binary32 library product 154).  The splitting of K, V and the
// weights into parts is vector work beside the matrix instructions, and the bound
// where there are many workgroups; with fewer than compute units (the same heads, 8
// sequences of up to 250 columns over up to 701 keys: 192 workgroups with a row tile,
// 51 us) it is each one's own chain of tiles, with matrix instructions in 18% of the
// cycles.
//
// Infinities and NaN have no such parts (infinity x 0 among the six products is
// NaN), and the instructions take subnormal parts as 0, which the last part of a
// number below 2^-103 can be.  A tile of K or V that holds such a number
// anywhere, or a wave whose queries do, takes its product from memory by the
// binary32 instructions instead.
//
// Otherwise as k_attn_shared: 4 waves of 32 rows, scores of the next tile taken
// while this one's become weights.  Tiles are 32 keys; a staged row is 3 x 64
// bytes, the parts one after another, which puts 4 consecutive rows on distinct
// quarters of the LDS banks (the transposing reads of K); V's 16-byte chunks are
// permuted by (row / 4) % 4 for its reads of 16 rows.  Two buffers each for K and
// V; the tiles after them are in registers meanwhile.
#pragma once

#include "attention_mfma.hpp"

namespace {

typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));

constexpr int kPartBytes = 64;              // of a part of a staged row
constexpr int kPartRow = 3 * kPartBytes;
constexpr int kPartKeys = 32;

__device__ __forceinline__ f16v mfma(b8 a, b8 b, f16v c) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
#else
    return c;
#endif
}

// Upper halves of two words
__device__ __forceinline__ uint32_t upper_halves(uint32_t lo, uint32_t hi) {
    return __builtin_amdgcn_perm(hi, lo, 0x07060302);
}

// Two numbers -> their parts, packed by twos
__device__ __forceinline__ void split2(float x, float y, uint32_t (&part)[3]) {
    const uint32_t x0 = __float_as_uint(x), y0 = __float_as_uint(y);
    const float rx = x - __uint_as_float(x0 & 0xffff0000u);
    const float ry = y - __uint_as_float(y0 & 0xffff0000u);
    const uint32_t x1 = __float_as_uint(rx), y1 = __float_as_uint(ry);
    const uint32_t x2 = __float_as_uint(rx - __uint_as_float(x1 & 0xffff0000u));
    const uint32_t y2 = __float_as_uint(ry - __uint_as_float(y1 & 0xffff0000u));
    part[0] = upper_halves(x0, y0);
    part[1] = upper_halves(x1, y1);
    part[2] = upper_halves(x2, y2);
}

// Whether among some numbers one is infinite, NaN, or not 0 and below 2^-103
struct Odd {
    uint32_t least = ~0u;  // of 2 |x| - 1 as the numbers' bits, for 0 the greatest there is
    bool special = false;

    __device__ __forceinline__ void add(float x) {
        least = min(least, 2 * __float_as_uint(x) - 1);
        special |= __builtin_amdgcn_classf(x, 0x207);
    }

    // for the whole wave
    __device__ __forceinline__ bool any() const {
        return __any(special || least < (2u * (127 - 103) << 23) - 1);
    }
};

// The 6 of the 9 products of parts that are taken, the smallest first
constexpr int kPairs[6][2] = {{2, 0}, {0, 2}, {1, 1}, {1, 0}, {0, 1}, {0, 0}};

// Rows of K or V: memory -> registers -> parts in LDS; wave `wave` of 4 takes
// every fourth group of 8 rows
template <int DP, bool V, bool WIDE>
struct PartStager {
    static constexpr int kGroups = DP / 32;
    HeadRows<WIDE> rows;
    uint32_t off;  // of the lane's 4 keys
    v4f hold[kGroups];

    __device__ __forceinline__ void init(const AttnArgs &a, const void *matrix, int64_t ld,
                                         int head, int first) {
        const int lane = threadIdx.x & 63;
        (void)rows.init(a, matrix, ld, head, first, 4);  // binary32 rows start on 4 bytes
        off = (uint32_t)((lane >> 3) * rows.ld) + 16 * (lane & 7);
    }
    __device__ __forceinline__ void ask(int at, int wave) {
        rows.template groups<kGroups, 4>(
            4 * (int64_t)at, wave, [&](int i, buf_rsrc_t r, uint32_t row) {
                hold[i] = __builtin_bit_cast(v4f, load16_buf(r, off + row));
            });
    }
    // true if one of this wave's numbers has no parts
    __device__ __forceinline__ bool put(lds_char *lds, int wave) {
        const int lane = threadIdx.x & 63;
        Odd odd;
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
            const int row = 8 * (4 * i + wave) + (lane >> 3);
            const int chunk = ((lane & 7) >> 1) ^ (V ? (row >> 2) & 3 : 0);
            uint32_t a[3], b[3];
            split2(hold[i][0], hold[i][1], a);
            split2(hold[i][2], hold[i][3], b);
            lds_char *at = lds + row * kPartRow + 16 * chunk + 8 * (lane & 1);
#pragma unroll
            for (int p = 0; p < 3; ++p)
                *(__attribute__((address_space(3))) u2 *)(at + p * kPartBytes) = u2{a[p], b[p]};
#pragma unroll
            for (int k = 0; k < 4; ++k) odd.add(hold[i][k]);
        }
        return odd.any();
    }
};

template <int DP>
struct PartRows : RowSums<DP, 1, true> {
    static constexpr int QF = DP / 16;
    typedef RowSums<DP, 1, true> Sums;
    using Sums::l;
    using Sums::o;
    using typename Sums::Scores;
    struct Weights {
        b8 p[3][2];  // part, step of 16 keys
    };
    b8 q[3][QF];
    bool plain;      // all of the wave's queries have parts

    static __device__ __forceinline__ void parts8(const float (&x)[8], b8 &p0, b8 &p1, b8 &p2) {
        u4 w[3];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t part[3];
            split2(x[2 * e], x[2 * e + 1], part);
#pragma unroll
            for (int p = 0; p < 3; ++p) w[p][e] = part[p];
        }
        p0 = __builtin_bit_cast(b8, w[0]);
        p1 = __builtin_bit_cast(b8, w[1]);
        p2 = __builtin_bit_cast(b8, w[2]);
    }

    __device__ __forceinline__ void init(const AttnArgs &a, int kv_head, const RowAt &r) {
        const int h = (threadIdx.x & 63) >> 5;
        const float *src =
            (const float *)a.Q + (int64_t)(kv_head * a.share + r.g) * a.D * a.ldq + r.column;
        Odd odd;
#pragma unroll
        for (int c = 0; c < QF; ++c) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int d = 16 * c + 8 * h + e;
                const float v = src[min(d, a.D - 1) * a.ldq];
                x[e] = d < a.D ? v : 0.f;
                odd.add(x[e]);
            }
            parts8(x, q[0][c], q[1][c], q[2][c]);
        }
        plain = !odd.any();
    }

    __device__ __forceinline__ void scores(Scores &x, lds_char *k) const {
        const int lane = threadIdx.x & 63, h = lane >> 5;
        x.s[0] = f16v{};
        // segment lane % 4 of its 16 keys: 0, 8, 4, 12
        lds_char *at = k + (8 * h + ((lane & 15) >> 2)) * kPartRow +
                       16 * (2 * ((lane >> 4) & 1) + (lane & 1)) + 8 * ((lane >> 1) & 1);
#pragma unroll
        for (int c = 0; c < QF; ++c) {
            b8 f[3];
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                lds_char *y = at + 16 * kPartRow * c + kPartBytes * p;
                struct { s4 x, y; } g = {read_tr(y), read_tr(y + 4 * kPartRow)};
                f[p] = __builtin_bit_cast(b8, g);
            }
#pragma unroll
            for (int i = 0; i < 6; ++i)
                x.s[0] = mfma(f[kPairs[i][0]], q[kPairs[i][1]][c], x.s[0]);
        }
    }

    // Scores to weights, their parts and sum; x keeps the weights
    __device__ __forceinline__ void weigh(Scores &x, Weights &w) {
        this->exponentials(x, Elem<float>::lift);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                y[e] = x.s[0][8 * c + e];
                l += y[e];
            }
            parts8(y, w.p[0][c], w.p[1][c], w.p[2][c]);
        }
    }

    __device__ __forceinline__ void values(const Weights &w, lds_char *v) {
        const int lane = threadIdx.x & 63, h = lane >> 5, row = lane & 31;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            lds_char *at = v + row * kPartRow + 16 * ((2 * c + h) ^ ((row >> 2) & 3));
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) {
                b8 f[3];
#pragma unroll
                for (int p = 0; p < 3; ++p)
                    f[p] = __builtin_bit_cast(b8, read16(at + 32 * kPartRow * d + kPartBytes * p));
#pragma unroll
                for (int i = 0; i < 6; ++i) o[d] = mfma(f[kPairs[i][0]], w.p[kPairs[i][1]][c], o[d]);
            }
        }
    }
};

template <int DP, bool WIDE>
__global__ __launch_bounds__(256, DP <= 64 && !WIDE ? 2 : 1) void k_attn_parts(AttnArgs a) {
    constexpr int TR = kAttnSharedRows, KT = kPartKeys;
    constexpr int kTile = DP * kPartRow;
    __shared__ __attribute__((aligned(1024))) char lds_k[2 * kTile];
    __shared__ __attribute__((aligned(1024))) char lds_v[2 * kTile];
    // the last even, odd tile of K, of V, that holds a number without parts
    __shared__ int odd[2][2];
    __shared__ int any_odd;  // there was one of V
    Place at;
    if (!find_place<TR>(a, blockIdx.x, at)) return;
    const RowTile &r = at.rows;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const RowAt mine = row_at<TR>(a, r, 32 * wave + (lane & 31));
    PartRows<DP> w;
    w.clear(a);

    const int first = r.begin - r.begin % a.align;
    const int tiles = r.end > r.begin ? (r.end - first + KT - 1) / KT : 0;
    const int lo = (int)((int64_t)tiles * at.part / a.splits);
    const int hi = (int)((int64_t)tiles * (at.part + 1) / a.splits);
    if (lo < hi) {
        PartStager<DP, false, WIDE> ks;
        PartStager<DP, true, WIDE> vs;
        ks.init(a, a.K, a.ldk, at.head, first);
        vs.init(a, a.V, a.ldv, at.head, first);
        auto k_at = [&](int t) { return (lds_char *)lds_k + (t & 1) * kTile; };
        auto v_at = [&](int t) { return (lds_char *)lds_v + (t & 1) * kTile; };
        auto put_k = [&](int t) {
            if (ks.put(k_at(t), wave)) odd[0][t & 1] = t;
        };
        auto put_v = [&](int t) {
            if (vs.put(v_at(t), wave)) odd[1][t & 1] = t, any_odd = 1;
        };
        auto k_plain = [&](int t) {
            return w.plain && __builtin_amdgcn_readfirstlane(odd[0][t & 1]) != t;
        };
        auto v_plain = [&](int t) { return __builtin_amdgcn_readfirstlane(odd[1][t & 1]) != t; };
        auto scores_at = [&](int t, typename PartRows<DP>::Scores &x) {
            if (k_plain(t))
                w.scores(x, k_at(t));
            else
                scores_from_memory<true>(args_again(), x.s[0], at.head, mine, (int64_t)first + (int64_t)t * KT);
        };
        ks.ask(lo * KT, wave);
        w.init(a, at.head, mine);
        uint8_t byte = mask_at(a, (int64_t)first + (int64_t)lo * KT);
        if (threadIdx.x < 4) odd[threadIdx.x >> 1][threadIdx.x & 1] = -1;
        if (threadIdx.x == 4) any_odd = 0;
        __syncthreads();
        put_k(lo);
        vs.ask(lo * KT, wave);
        if (lo + 1 < hi) ks.ask((lo + 1) * KT, wave);
        __syncthreads();
        typename PartRows<DP>::Scores cur, nxt;
        typename PartRows<DP>::Weights p;
        scores_at(lo, cur);
        for (int t = lo; t < hi; ++t) {
            const int64_t t0 = (int64_t)first + (int64_t)t * KT;
            const uint64_t valid = valid_keys<float>(a, t0, r, byte);
            const bool more = t + 1 < hi;
            const Draft draft = draft_at<float, 8>(a, r, mine, t0);
            // V of this tile and K of the next, in registers since the last step, into
            // the buffers that the step before it read; the ones after them asked for
            put_v(t);
            if (more) {
                put_k(t + 1);
                byte = mask_at(a, t0 + KT);
                vs.ask((t + 1) * KT, wave);
                if (t + 2 < hi) ks.ask((t + 2) * KT, wave);
            }
            settle<float>(w, cur, valid, draft);
            w.raise(cur, Elem<float>::slack);
            __syncthreads();
            if (more && k_plain(t + 1) && v_plain(t)) {
                w.scores(nxt, k_at(t + 1));
                w.weigh(cur, p);
                w.values(p, v_at(t));  // (a key left out is finite here: 0 times it is 0)
            } else {
                w.weigh(cur, p);
                if (v_plain(t))
                    w.values(p, v_at(t));
                else
                    values_from_memory<DP>(args_again(), w, cur, at.head, t0, valid,
                                           a.tree && r.end - r.n - t0 < KT);
                if (more) scores_at(t + 1, nxt);
            }
            cur = nxt;
        }
        if (__any(w.overflowed())) leveled_rows<DP>(args_again(), r, mine, at.head, first, lo, hi, 1, w);
        if (a.tree) {
            __syncthreads();
            if (__builtin_amdgcn_readfirstlane(any_odd))
                add_not_finite<float, DP, 1>(args_again(), r, mine, at.head, first, lo, hi, w.o);
        }
    }
    finish<float, DP>(a, at, mine, w, wave);
}

}  // namespace

// k_norm.hip -- H = R + scale G after(A), Y = before(H), norms over the features of
// every token, in one pass over features x tokens.
//
// A workgroup takes a tile of tokens with all their features and holds it in registers
// from the first read to the last store: every matrix is read or written once.  A
// thread has kVec neighbouring tokens of every (threads / lanes)-th row, so that the
// tile's part of a row is one run; the sums of a token go over lanes, then over
// waves through LDS.  Rows may start on any element: the loads of kVec tokens do not
// ask for more.
//
// 768 x 8: 7.6 us, one workgroup's chain of loads, two sums and stores.  768 x 4096
// (residual, LayerNorm, 25 MB): 11.5 us, 256 workgroups, one a compute unit, so that a
// chain stands beside no other.  Binary32 4096 x 4095, norms on both sides, gate and residual
// (335 MB): 122 us, 2.7 TB/s: 8 tokens are all that fit the registers, 32 bytes a row, and
// one workgroup a compute unit holds them, so reading, summing and writing alternate.
// Measured there: 16 tokens of 1024 threads 227 us and of 512 threads with 128 values each
// 156, 4 tokens 238 (runs of 16 bytes), two workgroups of 128 registers 170 to 207 (spills),
// half of the values in LDS 136.  Rows of 4128 values in place of 4096 take 109 us.
#include "norm.hpp"

namespace {

constexpr int kThreads = 512;    // of a workgroup; 1024 were slower at every size (128 registers each)
constexpr int kHold = 64;        // values a thread holds, at most

template <typename T, int kVec>
struct Pack {
    T v[kVec];
    // kWhole: all kVec are inside, else the first `valid`
    template <bool kWhole>
    __device__ __forceinline__ static Pack load(const T *from, int valid) {
        Pack p = {};
        if constexpr (kWhole)
            __builtin_memcpy(&p, from, sizeof p);
        else
#pragma unroll
            for (int e = 0; e < kVec; ++e)
                if (e < valid) p.v[e] = from[e];
        return p;
    }
    template <bool kWhole>
    __device__ __forceinline__ void store(T *to, int valid) const {
        if constexpr (kWhole)
            __builtin_memcpy(to, this, sizeof *this);
        else
#pragma unroll
            for (int e = 0; e < kVec; ++e)
                if (e < valid) to[e] = v[e];
    }
};

// Sums (kMax: largest) of v over the threads of the same tokens.  Two buffers in turn, so that
// one barrier a call is enough.  kRare: in a few registers.
template <int kVec>
struct Reducer {
    static constexpr int kWaves = kThreads / 64;
    double *lds;
    int lanes, turn = 0;

    template <bool kMax, bool kRare = false, typename V>
    __device__ __forceinline__ void operator()(V (&v)[kVec]) {
        auto both = [](V a, V b) { return kMax ? (a > b ? a : b) : a + b; };
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tokens = lanes * kVec;
        V *here = reinterpret_cast<V *>(lds + turn * kWaves * tokens);
        turn ^= 1;
        if (kVec > 1 && lanes * kVec <= 64) {
            // halves are exchanged first: a lane ends up with one of its tokens, after 10
            // moves in place of 6 kVec
            int token = 0;
#pragma unroll
            for (int c = kVec / 2, d = 32; c >= 1; c /= 2, d /= 2) {
                const bool up = lane & d;
#pragma unroll
                for (int e = 0; e < c; ++e) {
                    const V a = v[e], b = v[e + c], send = up ? a : b, keep = up ? b : a;
                    v[e] = both(keep, __shfl_xor(send, d));
                }
                token += up ? c : 0;
            }
            for (int d = 32 / kVec; d >= lanes; d /= 2) v[0] = both(v[0], __shfl_xor(v[0], d));
            if (lane % (64 / kVec) < lanes) here[wave * tokens + lane % lanes * kVec + token] = v[0];
        } else {
#pragma unroll
            for (int e = 0; e < kVec; ++e)
                for (int d = 32; d >= lanes; d /= 2) v[e] = both(v[e], __shfl_xor(v[e], d));
            if (lane < lanes)
#pragma unroll
                for (int e = 0; e < kVec; ++e) here[wave * tokens + lane * kVec + e] = v[e];
        }
        __syncthreads();
        const V *mine = here + threadIdx.x % lanes * kVec;
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[e] = mine[e];
#pragma unroll kRare ? 1 : kWaves
        for (int w = 1; w < kWaves; ++w)
#pragma unroll
            for (int e = 0; e < kVec; ++e) v[e] = both(v[e], mine[w * tokens + e]);
    }
};

// What the values of a norm may be: kSmall, binary16, whose squares and sums are in binary32's range.  kWide, what becomes
// binary16 only afterwards (scale, weights and biases are binary32, so a sum with the residual may be of any size): sums of
// squares in binary64.  kAll, binary32: sums in binary32, and made once more where that range does not do.
// (kWide as kAll would cost calls of 4096 rows a workgroup a compute unit, 8192 tokens 191 us in place of 147.)
enum Range { kSmall, kWide, kAll };

// x becomes its norm, without weight and bias
template <Range kRange, int kVec, int kPer>
__device__ __forceinline__ void normed(float (&x)[kPer][kVec], const nmg_norm &norm, int M,
                                       Reducer<kVec> &reduce) {
    if (norm.kind == NMG_NORM_NONE) return;
    const int step = kThreads / reduce.lanes, r0 = threadIdx.x / reduce.lanes;
    const float inv_m = 1.f / (float)M;
    using Sum = std::conditional_t<kRange == kWide, double, float>;
    float mean[kVec], by[kVec];      // by: what a token is multiplied by first
    Sum ss[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) by[e] = 1.f;
    auto sums = [&](auto rare) __attribute__((always_inline)) {
        constexpr bool kRare = decltype(rare)::value;
#pragma unroll
        for (int e = 0; e < kVec; ++e) mean[e] = 0.f;
        if (norm.kind == NMG_NORM_LAYER) {
            // (kWide: 2^15 values of any size times 2^-16 stay in the range; rows past M hold 0)
            constexpr float down = kRange == kWide ? 0x1p-16f : 1.f;
#pragma unroll
            for (int i = 0; i < kPer; ++i)
#pragma unroll
                for (int e = 0; e < kVec; ++e) mean[e] = __builtin_fmaf(x[i][e], down * by[e], mean[e]);
            reduce.template operator()<false, kRare>(mean);
#pragma unroll
            for (int e = 0; e < kVec; ++e) mean[e] *= inv_m * (1.f / down);
        }
#pragma unroll
        for (int e = 0; e < kVec; ++e) ss[e] = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i)
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                const Sum d = r0 + i * step < M ? __builtin_fmaf(x[i][e], by[e], -mean[e]) : 0.f;
                ss[e] += d * d;
            }
        reduce.template operator()<false, kRare>(ss);
    };
    sums(std::false_type{});
    // Squares or sums past the range, or below it where eps does not cover what is lost: once more, of tokens
    // times a power of two each that brings them to about 1
    bool scaled = false;
    if constexpr (kRange == kAll) {
#pragma unroll
        for (int e = 0; e < kVec; ++e)
            scaled |= !(ss[e] < __builtin_inff()) || (ss[e] < 0x1p-80f && norm.eps < 0x1p-60f);
        // (every wave has all tokens of the tile, with the same sums: all agree without a barrier)
        scaled = __any(scaled);
    }
    float *factors = reinterpret_cast<float *>(reduce.lds + 2 * Reducer<kVec>::kWaves * reduce.lanes * kVec);
    float *scales = factors + reduce.lanes * kVec;
    const int at = threadIdx.x % reduce.lanes * kVec;
    if (__builtin_expect(scaled, 0)) {
        float top[kVec];
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            top[e] = 0.f;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const float v = fabsf(x[i][e]);
                if (v < __builtin_inff()) top[e] = fmaxf(top[e], v);
            }
        }
        reduce.template operator()<true, true>(top);
#pragma unroll
        for (int e = 0; e < kVec; ++e)
            by[e] = top[e] == 0.f ? 1.f : __builtin_ldexpf(1.f, min(max(1 - __builtin_amdgcn_frexp_expf(top[e]), -126), 126));
        sums(std::true_type{});
        // the factors of the differences: 1 / sqrt(mean square + eps by^2), by a thread each
        if ((int)threadIdx.x < reduce.lanes)
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                factors[at + e] = ss[e];
                scales[at + e] = by[e];
            }
        __syncthreads();
        if (const int t = threadIdx.x; t < reduce.lanes * kVec)
            factors[t] = (float)(1.0 / sqrt((double)factors[t] / M + (double)norm.eps * scales[t] * scales[t]));
        __syncthreads();
    }
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
        const float inv = scaled             ? factors[at + e]
                          : kRange == kWide ? (float)(1.0 / sqrt(ss[e] * inv_m + norm.eps))
                                            : 1.f / sqrtf(ss[e] * inv_m + norm.eps);
#pragma unroll
        for (int i = 0; i < kPer; ++i) x[i][e] = __builtin_fmaf(x[i][e], by[e], -mean[e]) * inv;
    }
}

// kWhole: every token of the tile is inside
template <typename T, int kVec, int kPer, bool kWhole>
__device__ __forceinline__ void residual_norm(const NormArgs &a, int tile, double *lds) {
    using P = Pack<T, kVec>;
    // The gate and the residual are asked for with A where they are 64 bytes a thread at most:
    // more of them beside A cost registers that the loads of A lack (binary16 768 x 32768 101 us
    // with a limit of 128 bytes, 82 with 64).
    constexpr bool kEarly = kPer * kVec * (int)sizeof(T) <= 64, kWeights = kEarly && kPer <= 4;
    constexpr int kE = kEarly ? kPer : 1, kW = kWeights ? kPer : 1;
    const int lanes = a.lanes, step = kThreads / lanes, r0 = threadIdx.x / lanes;
    const int64_t n = (int64_t)tile * lanes * kVec + threadIdx.x % lanes * kVec;
    const int valid = kWhole ? kVec : (int)max((int64_t)0, min((int64_t)kVec, a.N - n));
    float x[kPer][kVec];
    // row r of a matrix at the thread's tokens: what a thread's rows differ by is the same for all
    auto at_row = [&](const void *from, int64_t ld, int i) {
        return static_cast<const T *>(from) + ((int64_t)r0 * ld + n) + (int64_t)(i * step) * ld;
    };
    auto load = [&](const void *from, int64_t ld, int i) {
        return P::template load<kWhole>(at_row(from, ld, i), valid);
    };
    P gate[kE], residual[kE];
    float w1[kW], b1[kW], w2[kW], b2[kW];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int r = r0 + i * step;
        P p = {};
        if (valid && r < a.M) p = load(a.A, a.lda, i);
#pragma unroll
        for (int e = 0; e < kVec; ++e) x[i][e] = (float)p.v[e];
    }
    auto others = [&](int i, int to) {
        if (a.G) gate[to] = load(a.G, a.ldg, i);
        if (a.R) residual[to] = load(a.R, a.ldr, i);
    };
    auto firsts = [&](int r, int i) {
        w1[i] = a.after.weight ? a.after.weight[r] : 1.f;
        b1[i] = a.after.bias ? a.after.bias[r] : 0.f;
    };
    auto lasts = [&](int r, int i) {
        w2[i] = a.before.weight ? a.before.weight[r] : 1.f;
        b2[i] = a.before.bias ? a.before.bias[r] : 0.f;
    };
    if constexpr (kEarly)
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int r = r0 + i * step;
            if (!valid || r >= a.M) continue;
            others(i, i);
            if constexpr (kWeights) {
                firsts(r, i);
                lasts(r, i);
            }
        }
    Reducer<kVec> reduce{lds, lanes};
    normed<std::is_same<T, float>::value ? kAll : kSmall, kVec, kPer>(x, a.after, a.M, reduce);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int r = r0 + i * step;
        if (!valid || r >= a.M) {
#pragma unroll
            for (int e = 0; e < kVec; ++e) x[i][e] = 0.f;
            continue;
        }
        const int at = kEarly ? i : 0, w = kWeights ? i : 0;
        if constexpr (!kEarly) others(i, at);
        if constexpr (!kWeights) firsts(r, w);
        P h;
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            float y = x[i][e] * w1[w] + b1[w];
            if (a.G) y *= (float)gate[at].v[e];
            y *= a.scale;
            if (a.R) y += (float)residual[at].v[e];
            x[i][e] = y;
            h.v[e] = (T)y;
        }
        if (a.H) h.template store<kWhole>(const_cast<T *>(at_row(a.H, a.ldh, i)), valid);
    }
    if (!a.Y) return;
    normed<std::is_same<T, float>::value ? kAll : kWide, kVec, kPer>(x, a.before, a.M, reduce);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int r = r0 + i * step;
        if (!valid || r >= a.M) continue;
        const int at = kWeights ? i : 0;
        if constexpr (!kWeights) lasts(r, at);
        P y;
#pragma unroll
        for (int e = 0; e < kVec; ++e) y.v[e] = (T)(x[i][e] * w2[at] + b2[at]);
        y.template store<kWhole>(const_cast<T *>(at_row(a.Y, a.ldy, i)), valid);
    }
}

// (binary16 of up to 4096 rows: two workgroups a compute unit, 128 registers.  147 us for 8192 tokens; one
// workgroup of 134 registers, 188.)
template <typename T, int kVec, int kPer>
__global__ __launch_bounds__(kThreads, (kVec == 8 && kPer == 8 ? 4 : 2)) void k_residual_norm(NormArgs a, int tiles) {
    extern __shared__ double lds[];
    const int tile = xcd_tile(blockIdx.x, tiles);
    if (((int64_t)tile + 1) * a.lanes * kVec <= a.N)
        residual_norm<T, kVec, kPer, true>(a, tile, lds);
    else
        residual_norm<T, kVec, kPer, false>(a, tile, lds);
}

template <typename T, int kVec>
nmg_status run(NormArgs a, int tokens, hipStream_t stream) {
    a.lanes = tokens / kVec;
    const int tiles = (int)(((int64_t)a.N + tokens - 1) / tokens);
    if ((int64_t)tiles * kThreads >= ((int64_t)1 << 32)) return NMG_ERR_UNSUPPORTED;
    const int step = kThreads / a.lanes, per = (a.M + step - 1) / step;
    const size_t room = (2 * (kThreads / 64) + 1) * tokens * sizeof(double);
    auto go = [&](auto k) {
        constexpr int kPer = decltype(k)::value;
        k_residual_norm<T, kVec, kPer><<<tiles, kThreads, room, stream>>>(a, tiles);
        return launched();
    };
    if (per <= kHold / kVec / 8) return go(std::integral_constant<int, kHold / kVec / 8>{});
    if (per <= kHold / kVec / 4) return go(std::integral_constant<int, kHold / kVec / 4>{});
    if (per <= kHold / kVec / 2) return go(std::integral_constant<int, kHold / kVec / 2>{});
    return go(std::integral_constant<int, kHold / kVec>{});
}

template <typename T>
nmg_status plan(const NormArgs &a, hipStream_t stream) {
    constexpr int kVec = 16 / sizeof(T);
    // The most tokens whose features a workgroup can hold, fewer while compute units stand
    // idle.
    int tokens = 64;
    while (tokens > 1 && (int64_t)tokens * a.M > (int64_t)kThreads * kHold) tokens /= 2;
    while (tokens > kVec && ((int64_t)a.N + tokens - 1) / tokens < device_cus()) tokens /= 2;
    return tokens < kVec ? run<T, 1>(a, tokens, stream) : run<T, kVec>(a, tokens, stream);
}

}  // namespace

namespace nmg_internal {

nmg_status launch_residual_norm(nmg_dtype dtype, NormArgs a, hipStream_t stream) {
    if (a.M > kThreads * kHold) return NMG_ERR_UNSUPPORTED;
    return dtype == NMG_F32 ? plan<float>(a, stream) : plan<_Float16>(a, stream);
}

}  // namespace nmg_internal

// k_norm.hip -- H = R + scale G after(A), Y = before(H), norms over the features of
// every token, in one pass over features x tokens.
//
// A workgroup takes a tile of tokens with all their features and holds it in registers
// from the first read to the last store: every matrix is read or written once.  A
// thread has kVec neighbouring tokens of every (512 / lanes)-th row, so that the
// tile's part of a row is one run; the sums of a token go over lanes, then over
// waves through LDS.
#include "norm.hpp"

namespace {

constexpr int kThreads = 512;
constexpr int kHold = 64;        // values a thread holds, at most

template <typename T, int kVec>
struct __align__(sizeof(T) * kVec) Pack {
    T v[kVec];
};

// Sums (kMax: largest) of v over the threads of the same tokens
template <int kVec, bool kMax>
__device__ __forceinline__ void over_rows(float (&v)[kVec], int lanes, float *lds) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tokens = lanes * kVec;
#pragma unroll
    for (int e = 0; e < kVec; ++e)
        for (int d = 32; d >= lanes; d /= 2) {
            const float o = __shfl_xor(v[e], d);
            v[e] = kMax ? fmaxf(v[e], o) : v[e] + o;
        }
    float *total = lds + kThreads / 64 * 64 * kVec;
    __syncthreads();                             // (the last call's totals have been read)
    if (lane < lanes)
#pragma unroll
        for (int e = 0; e < kVec; ++e) lds[wave * tokens + lane * kVec + e] = v[e];
    __syncthreads();
    if ((int)threadIdx.x < tokens) {
        float s = lds[threadIdx.x];
        for (int w = 1; w < kThreads / 64; ++w) {
            const float o = lds[w * tokens + threadIdx.x];
            s = kMax ? fmaxf(s, o) : s + o;
        }
        total[threadIdx.x] = s;
    }
    __syncthreads();
    const int first = threadIdx.x % lanes * kVec;
#pragma unroll
    for (int e = 0; e < kVec; ++e) v[e] = total[first + e];
}
template <int kVec>
constexpr int over_rows_floats() { return (kThreads / 64 + 1) * 64 * kVec; }

// x becomes its norm, without weight and bias
template <typename T, int kVec, int kPer>
__device__ __forceinline__ void normed(float (&x)[kPer][kVec], const nmg_norm &norm, int M, int lanes,
                                       float *lds) {
    if (norm.kind == NMG_NORM_NONE) return;
    const int step = kThreads / lanes, r0 = threadIdx.x / lanes;
    const float inv_m = 1.f / (float)M;
    float mean[kVec], ss[kVec];
    auto statistics = [&]() {
#pragma unroll
        for (int e = 0; e < kVec; ++e) mean[e] = 0.f;
        if (norm.kind == NMG_NORM_LAYER) {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
#pragma unroll
                for (int e = 0; e < kVec; ++e) mean[e] += x[i][e];   // (rows past M hold 0)
            over_rows<kVec, false>(mean, lanes, lds);
#pragma unroll
            for (int e = 0; e < kVec; ++e) mean[e] *= inv_m;
        }
#pragma unroll
        for (int e = 0; e < kVec; ++e) ss[e] = 0.f;
#pragma unroll
        for (int i = 0; i < kPer; ++i)
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                const float d = r0 + i * step < M ? x[i][e] - mean[e] : 0.f;
                ss[e] += d * d;
            }
        over_rows<kVec, false>(ss, lanes, lds);
    };
    statistics();
    if constexpr (std::is_same<T, float>::value) {
        // Squares or sums past the range, or below it where eps does not cover what is
        // lost: the tokens are scaled by a power of two each to below 2 and summed again.
        bool again = false;
#pragma unroll
        for (int e = 0; e < kVec; ++e)
            again |= !(ss[e] < __builtin_inff()) || (ss[e] < 0x1p-80f && norm.eps < 0x1p-60f);
        if (__syncthreads_or(again)) {
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
            over_rows<kVec, true>(top, lanes, lds);
            int ex[kVec];
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                ex[e] = top[e] == 0.f ? 0 : __builtin_amdgcn_frexp_expf(top[e]) - 1;
#pragma unroll
                for (int i = 0; i < kPer; ++i) x[i][e] = __builtin_ldexpf(x[i][e], -ex[e]);
            }
            statistics();
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                // x / sqrt(mean square + eps) with both over 2^ex
                const double var = (double)ss[e] / M + __builtin_ldexp((double)norm.eps, -2 * ex[e]);
                const float inv = (float)(1.0 / sqrt(var));
#pragma unroll
                for (int i = 0; i < kPer; ++i) x[i][e] = (x[i][e] - mean[e]) * inv;
            }
            return;
        }
    }
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
        const float inv = 1.f / sqrtf(ss[e] * inv_m + norm.eps);
#pragma unroll
        for (int i = 0; i < kPer; ++i) x[i][e] = (x[i][e] - mean[e]) * inv;
    }
}

template <typename T, int kVec, int kPer>
__global__ __launch_bounds__(kThreads) void k_residual_norm(NormArgs a, int tiles) {
    __shared__ float lds[over_rows_floats<kVec>()];
    using P = Pack<T, kVec>;
    const int lanes = a.lanes, step = kThreads / lanes, r0 = threadIdx.x / lanes;
    const int64_t n = (int64_t)xcd_tile(blockIdx.x, tiles) * lanes * kVec + threadIdx.x % lanes * kVec;
    const bool in = n < a.N;     // (kVec tokens are inside together: N and the tiles are multiples)
    float x[kPer][kVec];
    auto load = [&](const void *from, int64_t ld, int r) {
        return *reinterpret_cast<const P *>(static_cast<const T *>(from) + (int64_t)r * ld + n);
    };
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int r = r0 + i * step;
        P p = {};
        if (in && r < a.M) p = load(a.A, a.lda, r);
#pragma unroll
        for (int e = 0; e < kVec; ++e) x[i][e] = (float)p.v[e];
    }
    normed<T, kVec, kPer>(x, a.after, a.M, lanes, lds);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int r = r0 + i * step;
        if (!in || r >= a.M) {
#pragma unroll
            for (int e = 0; e < kVec; ++e) x[i][e] = 0.f;
            continue;
        }
        const float w = a.after.weight ? a.after.weight[r] : 1.f, b = a.after.bias ? a.after.bias[r] : 0.f;
        P g, res;
        if (a.G) g = load(a.G, a.ldg, r);
        if (a.R) res = load(a.R, a.ldr, r);
        P h;
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            float y = x[i][e] * w + b;
            if (a.G) y *= (float)g.v[e];
            y *= a.scale;
            if (a.R) y += (float)res.v[e];
            x[i][e] = y;
            h.v[e] = (T)y;
        }
        if (a.H) *reinterpret_cast<P *>(static_cast<T *>(a.H) + (int64_t)r * a.ldh + n) = h;
    }
    if (!a.Y) return;
    normed<T, kVec, kPer>(x, a.before, a.M, lanes, lds);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int r = r0 + i * step;
        if (!in || r >= a.M) continue;
        const float w = a.before.weight ? a.before.weight[r] : 1.f,
                    b = a.before.bias ? a.before.bias[r] : 0.f;
        P y;
#pragma unroll
        for (int e = 0; e < kVec; ++e) y.v[e] = (T)(x[i][e] * w + b);
        *reinterpret_cast<P *>(static_cast<T *>(a.Y) + (int64_t)r * a.ldy + n) = y;
    }
}

template <typename T, int kVec>
nmg_status run(NormArgs a, int tokens, hipStream_t stream) {
    a.lanes = tokens / kVec;
    const int tiles = (int)(((int64_t)a.N + tokens - 1) / tokens);
    if ((int64_t)tiles * kThreads >= ((int64_t)1 << 32)) return NMG_ERR_UNSUPPORTED;
    const int step = kThreads / a.lanes, per = (a.M + step - 1) / step;
    auto go = [&](auto k) {
        constexpr int kPer = decltype(k)::value;
        k_residual_norm<T, kVec, kPer><<<tiles, kThreads, 0, stream>>>(a, tiles);
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
    bool vec = a.N % kVec == 0;
    auto fits = [&](const void *p, int64_t ld) {
        if (p) vec = vec && aligned(p, 16) && ld % kVec == 0;
    };
    fits(a.A, a.lda);
    fits(a.G, a.ldg);
    fits(a.R, a.ldr);
    fits(a.H, a.ldh);
    fits(a.Y, a.ldy);
    // the most tokens whose features the workgroup can hold
    int most = 64 * (vec ? kVec : 1);
    while (most > 1 && (int64_t)most * a.M > (int64_t)kThreads * kHold) most /= 2;
    // fewer while compute units stand idle
    int tokens = most;
    while (tokens > kVec && ((int64_t)a.N + tokens - 1) / tokens < device_cus()) tokens /= 2;
    if (vec && tokens >= kVec) return run<T, kVec>(a, tokens, stream);
    return run<T, 1>(a, std::min(tokens, 64), stream);
}

}  // namespace

namespace nmg_internal {

nmg_status launch_residual_norm(nmg_dtype dtype, NormArgs a, hipStream_t stream) {
    if (a.M > kThreads * kHold) return NMG_ERR_UNSUPPORTED;
    return dtype == NMG_F32 ? plan<float>(a, stream) : plan<_Float16>(a, stream);
}

}  // namespace nmg_internal

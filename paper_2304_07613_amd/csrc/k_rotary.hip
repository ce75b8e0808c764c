// k_rotary.hip -- position rotation of heads, alone or behind the norm of
// queries and keys (features x tokens), and its tables.
//
// k_rotary.  A head's rows come in units: the R / 2 pairs that turn, then the
// other rows by twos.  A workgroup covers a run of tokens (lanes, so every load
// and store is a run of a row) and all units of a head, dealt over its
// slices; a thread keeps its units of `tokens` tokens in registers from the
// load to the store, so a head is read once and written once, whether the sum
// of squares (added over the slices by lane exchanges and LDS) comes between
// or not.  Cosines and sines are the same for every head: a workgroup keeps
// them in registers for a run of heads, as many as leave about four workgroups
// for every compute unit.  One read and one write are all there is to it: 16 heads
// x 128, 16384 tokens of binary32 in 51-60 us = 4.6-5.4 TB/s (a large copy 4.9); a few
// tokens take a launch and two chained loads, positions and table (3 us).
//
// k_rotary_table  cosines and sines in binary64.
#include "rotary.hpp"

namespace {

// Whether squares passed an end of binary32's range (below it only where eps is too)
__device__ __forceinline__ bool squares_far(float sum, float eps) {
    return sum == INFINITY || (sum < 0x1p-90f && eps < 0x1p-90f);
}

// One head of a workgroup's tokens with such squares: summed once more, of the values
// times a power of two.  From memory and token by token, in few registers: it is rare.
template <int N>
__device__ __forceinline__ void norm_far(const RotaryArgs &a, const RotaryRows &r, int h, int64_t t,
                                         int x, int slice, int slices, float *sums) {
    const int lanes = a.lanes, half = a.R / 2, units = half + (a.D - a.R + 1) / 2;
    const float *src = (const float *)r.X + (int64_t)h * a.D * r.ldx;
    float *dst = (float *)r.Y + (int64_t)h * a.D * r.ldy;
#pragma unroll 1
    for (int n = 0; n < N; ++n) {
        const int64_t c = t + n;
        const bool here = c < a.N;
        auto rows_of = [&](int u, int &f, int &g) {  // of unit u; g may be none: -1
            f = u >= half ? a.R + 2 * (u - half) : a.interleaved ? 2 * u : u;
            g = u < half ? (a.interleaved ? f + 1 : f + half) : f + 1 < a.D ? f + 1 : -1;
        };
        float scale = 1.f, sum = 0.f;
#pragma unroll 1
        for (int pass = 0; pass < 2; ++pass) {
            float part = 0.f;
            for (int u = slice; u < units && here; u += slices) {
                int f, g;
                rows_of(u, f, g);
                const float p = scale * src[f * r.ldx + c], q = g < 0 ? 0.f : scale * src[g * r.ldx + c];
                part = fmaf(p, p, fmaf(q, q, part));
            }
            for (int d = lanes; d < 64; d *= 2) part += __shfl_xor(part, d);
            __syncthreads();  // the sums before have been read
            if ((threadIdx.x & 63) < lanes) sums[threadIdx.x / 64 * 64 + x] = part;
            __syncthreads();
            sum = 0.f;
            for (int i = 0; i < kBlock / 64; ++i) sum += sums[i * 64 + x];
            if (pass == 0 && squares_far(sum, a.eps)) scale = sum == INFINITY ? 0x1p-100f : 0x1p100f;
        }
        if (!here) continue;
        // scale / rms may pass the range, where the values are below it
        const float first = fmaxf(scale, 1.f);
        const float second = fminf(scale, 1.f) / sqrtf(sum / (float)a.D + a.eps * scale * scale);
        for (int u = slice; u < units; u += slices) {
            int f, g;
            rows_of(u, f, g);
            float p = first * src[f * r.ldx + c], q = g < 0 ? 0.f : first * src[g * r.ldx + c];
            p = p * second * (r.weight ? r.weight[f] : 1.f);
            q = q * second * (r.weight && g >= 0 ? r.weight[g] : 1.f);
            if (u < half) {
                const int64_t at = min(max((int64_t)a.positions[c], (int64_t)0), a.length - 1);
                const float cs = a.table[u * a.length + at], sn = a.table[(half + u) * a.length + at];
                const float y = p * cs - q * sn;
                q = p * sn + q * cs;
                p = y;
            }
            dst[f * r.ldy + c] = p;
            if (g >= 0) dst[g * r.ldy + c] = q;
        }
    }
}

// N: tokens a thread, U: units a thread
template <typename T, bool NORM, int N, int U>
__global__ __launch_bounds__(kBlock, N == 4 && U <= 4 ? 3 : 1) void k_rotary(RotaryArgs a) {
    __shared__ float sums[2][kBlock / 64][64 * N];
    const int lanes = a.lanes, slices = kBlock / lanes;  // of tokens
    const int x = threadIdx.x % lanes, slice = threadIdx.x / lanes;
    // neighbouring runs of tokens on one XCD: rows rarely start on a cache line,
    // and the line two workgroups share is put together in its L2
    const int id = xcd_tile(blockIdx.x, gridDim.x), run = id / a.blocks;
    const int64_t t = ((int64_t)(id - run * a.blocks) * lanes + x) * N;
    const bool here = t < a.N, whole = t + N <= a.N;
    const int which = run >= a.groups0;
    const RotaryRows r = a.part[which];
    const int h0 = (run - (which ? a.groups0 : 0)) * a.run;
    const int h1 = min(h0 + a.run, r.heads);

    const int half = a.R / 2, units = half + (a.D - a.R + 1) / 2;
    int row[U][2];       // of unit i; -1: none
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int u = slice + i * slices;
        row[i][0] = row[i][1] = -1;
        if (u < half) {
            row[i][0] = a.interleaved ? 2 * u : u;
            row[i][1] = a.interleaved ? 2 * u + 1 : u + half;
        } else if (u < units) {
            row[i][0] = a.R + 2 * (u - half);
            row[i][1] = row[i][0] + 1 < a.D ? row[i][0] + 1 : -1;
        }
    }
    typedef T TN __attribute__((ext_vector_type(N)));
    TN in[U][2];         // of the head to come
    auto load = [&](int h) {
        const T *src = (const T *)r.X + (int64_t)h * a.D * r.ldx + t;
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                TN y = {};
                if (row[i][e] >= 0 && here) {
                    const T *q = src + row[i][e] * r.ldx;
                    if (whole) {
                        __builtin_memcpy(&y, q, sizeof y);
                    } else {
#pragma unroll
                        for (int n = 0; n < N; ++n)
                            if (t + n < a.N) y[n] = q[n];
                    }
                }
                in[i][e] = y;
            }
    };
    // the first head is on its way while positions, then cosines, sines and weights come
    load(h0);
    float c[U][N], s[U][N], w[U][2];
    int64_t p[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        p[n] = 0;
        if (a.R && t + n < a.N) p[n] = min(max((int64_t)a.positions[t + n], (int64_t)0), a.length - 1);
    }
    // tokens mostly follow one another in their sequence: one load then gives their
    // cosines, one their sines (16 heads x 128, 16384 tokens binary32: 53.4 -> 51.3 us)
    bool follow = p[0] + N <= a.length;
#pragma unroll
    for (int n = 1; n < N; ++n) follow &= t + n >= a.N || p[n] == p[0] + n;
    const bool runs = N > 1 && __all(follow || !here);
    typedef float FN __attribute__((ext_vector_type(N)));
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int u = slice + i * slices;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            c[i][n] = 1.f;
            s[i][n] = 0.f;
        }
        if (u < half && here) {
            const float *cs = a.table + u * a.length, *sn = a.table + (half + u) * a.length;
            if (runs) {
                FN x, y;
                __builtin_memcpy(&x, cs + p[0], sizeof x);
                __builtin_memcpy(&y, sn + p[0], sizeof y);
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    c[i][n] = x[n];
                    s[i][n] = y[n];
                }
            } else {
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    c[i][n] = cs[p[n]];
                    s[i][n] = sn[p[n]];
                }
            }
        }
#pragma unroll
        for (int e = 0; e < 2; ++e)
            w[i][e] = NORM && r.weight && row[i][e] >= 0 ? r.weight[row[i][e]] : 1.f;
    }

    int far = 0;             // bit h - h0: head h's squares passed the range
    for (int h = h0; h < h1; ++h) {
        T *dst = (T *)r.Y + (int64_t)h * a.D * r.ldy + t;
        float v[U][2][N];
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int n = 0; n < N; ++n) v[i][e][n] = (float)in[i][e][n];
        if (h + 1 < h1) load(h + 1);
        float scale[N];
        if constexpr (NORM) {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < U; ++i)
                    sum = fmaf(v[i][0][n], v[i][0][n], fmaf(v[i][1][n], v[i][1][n], sum));
                for (int d = lanes; d < 64; d *= 2) sum += __shfl_xor(sum, d);
                scale[n] = sum;
            }
            // two sets of sums: a wave may be a head ahead of another's reads
            auto &mine = sums[(h - h0) & 1];
            if ((threadIdx.x & 63) < lanes)
#pragma unroll
                for (int n = 0; n < N; ++n) mine[threadIdx.x / 64][x * N + n] = scale[n];
            __syncthreads();
            bool out = false;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < kBlock / 64; ++i) sum += mine[i][x * N + n];
                scale[n] = 1.f / sqrtf(sum / (float)a.D + a.eps);
                out |= squares_far(sum, a.eps);
            }
            // binary32: a wave holds lanes of every token of the workgroup and all have the
            // same sums, so all of them leave such a head for the end
            if (sizeof(T) == 4 && __any(out)) {
                far |= 1 << (h - h0);
                continue;
            }
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            TN out[2];
#pragma unroll
            for (int n = 0; n < N; ++n) {
                float f = v[i][0][n], g = v[i][1][n];
                if (NORM) {
                    f = f * scale[n] * w[i][0];
                    g = g * scale[n] * w[i][1];
                }
                const bool turns = slice + i * slices < half;
                out[0][n] = (T)(turns ? f * c[i][n] - g * s[i][n] : f);
                out[1][n] = (T)(turns ? f * s[i][n] + g * c[i][n] : g);
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if (row[i][e] < 0 || !here) continue;
                T *q = dst + row[i][e] * r.ldy;
                if (whole) {
                    __builtin_memcpy(q, &out[e], sizeof(TN));
                } else {
#pragma unroll
                    for (int n = 0; n < N; ++n)
                        if (t + n < a.N) q[n] = out[e][n];
                }
            }
        }
    }
    if constexpr (NORM && sizeof(T) == 4)
        for (; far; far &= far - 1)
            norm_far<N>(a, r, h0 + __builtin_ctz(far), t, x, slice, slices, &sums[0][0][0]);
}

__global__ __launch_bounds__(kBlock) void k_rotary_table(RotaryTableArgs a) {
    const int64_t p = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    const int i = blockIdx.y;
    if (p >= a.length) return;
    double f = exp(-(double)i / (double)a.half * a.log_base);
    if (a.scaling == NMG_ROTARY_LINEAR) f /= a.factor;
    if (a.scaling == NMG_ROTARY_PARTS) {
        const double turns = a.original * f / 6.283185307179586476925;
        const double keep = fmin(fmax((turns - a.slow) / (a.fast - a.slow), 0.0), 1.0);
        f *= keep + (1.0 - keep) / a.factor;
    }
    double sn, cs;
    sincos((double)p * f, &sn, &cs);
    a.table[i * a.length + p] = (float)(a.magnitude * cs);
    a.table[(a.half + i) * a.length + p] = (float)(a.magnitude * sn);
}

}  // namespace

namespace nmg_internal {

namespace {

template <typename T, bool NORM>
void launch(const RotaryArgs &a, int tokens, int units, dim3 grid, hipStream_t stream) {
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kBlock), 0, stream, a); };
    if (tokens == 1 && units <= 1)
        go(k_rotary<T, NORM, 1, 1>);
    else if (tokens == 1 && units <= 4)
        go(k_rotary<T, NORM, 1, 4>);
    else if (tokens == 1)
        go(k_rotary<T, NORM, 1, 16>);
    else if (tokens == 2) {
        if constexpr (sizeof(T) == 2) {
            if (units <= 4)
                go(k_rotary<T, NORM, 2, 4>);
            else
                go(k_rotary<T, NORM, 2, 8>);
        }
    } else if (units <= 2)
        go(k_rotary<T, NORM, 4, 2>);
    else if (units <= 4)
        go(k_rotary<T, NORM, 4, 4>);
    else
        go(k_rotary<T, NORM, 4, 8>);
}

}  // namespace

nmg_status launch_rotary(nmg_dtype dtype, const RotaryArgs &args, bool norm, hipStream_t stream) {
    RotaryArgs a = args;
    const int units = a.R / 2 + (a.D - a.R + 1) / 2;
    auto per_thread = [&] { return (units * a.lanes + kBlock - 1) / kBlock; };
    const int64_t heads = (int64_t)a.part[0].heads + a.part[1].heads;
    // 4 tokens a thread for 128 or more: 256 bytes of a row at a time (at any
    // alignment); 2 where that leaves binary16 fewer than 4 workgroups for every compute
    // unit (12 + 12 heads x 64 with norms: 4096 tokens 14.9 -> 13.1 us, 32768 52 -> 54)
    int tokens = a.N >= 128 ? 4 : 1;
    if (tokens == 4 && dtype == NMG_F16 && (a.N + 127) / 128 * heads < 4 * device_cus()) tokens = 2;
    const int most_lanes = tokens == 1 ? 64 : dtype == NMG_F16 ? 32 : 16;
    a.lanes = 1;
    while (a.lanes < most_lanes && (int64_t)a.lanes * tokens < a.N) a.lanes *= 2;
    while (a.lanes > 1 && per_thread() > (tokens == 1 ? 16 : 8)) a.lanes /= 2;
    if (per_thread() > 8) tokens = 1;
    if (per_thread() > 16) return NMG_ERR_UNSUPPORTED;
    const int64_t width = (int64_t)a.lanes * tokens, blocks = (a.N + width - 1) / width;
    a.run = (int)std::max<int64_t>(1, std::min<int64_t>(8, blocks * heads / (4 * device_cus())));
    a.groups0 = (a.part[0].heads + a.run - 1) / a.run;
    const int64_t groups = a.groups0 + (a.part[1].heads + a.run - 1) / a.run;
    if (!launchable(blocks * groups, kBlock)) return NMG_ERR_UNSUPPORTED;
    a.blocks = (int)blocks;
    const dim3 grid((unsigned)(blocks * groups));
    const int u = per_thread();
    if (dtype == NMG_F32)
        norm ? launch<float, true>(a, tokens, u, grid, stream)
             : launch<float, false>(a, tokens, u, grid, stream);
    else
        norm ? launch<_Float16, true>(a, tokens, u, grid, stream)
             : launch<_Float16, false>(a, tokens, u, grid, stream);
    return launched();
}

nmg_status launch_rotary_table(const RotaryTableArgs &a, hipStream_t stream) {
    const dim3 grid((unsigned)((a.length + kBlock - 1) / kBlock), (unsigned)a.half);
    hipLaunchKernelGGL(k_rotary_table, grid, dim3(kBlock), 0, stream, a);
    return launched();
}

}  // namespace nmg_internal

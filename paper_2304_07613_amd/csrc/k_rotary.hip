// k_rotary.hip -- position rotation of heads, alone or behind the norm of
// queries and keys (features x tokens), and its tables.
//
//   k_rotary        a thread per (token, head): the column's sum of squares,
//                   then its pairs.
//   k_rotary_table  cosines and sines in binary64.
#include "rotary.hpp"

namespace {

template <typename T, bool NORM>
__global__ __launch_bounds__(kBlock) void k_rotary(RotaryArgs a) {
    const int64_t t = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (t >= a.N) return;
    const int which = (int)blockIdx.y >= a.part[0].heads;
    const RotaryRows &r = a.part[which];
    const int h = (int)blockIdx.y - (which ? a.part[0].heads : 0);
    const T *x = (const T *)r.X + (int64_t)h * a.D * r.ldx + t;
    T *y = (T *)r.Y + (int64_t)h * a.D * r.ldy + t;
    float s = 1.f;
    if (NORM) {
        float sum = 0.f;
        for (int d = 0; d < a.D; ++d) {
            const float v = (float)x[d * r.ldx];
            sum = fmaf(v, v, sum);
        }
        s = 1.f / sqrtf(sum / (float)a.D + a.eps);
    }
    auto at = [&](int d) {
        const float v = (float)x[d * r.ldx];
        return NORM ? v * s * (r.weight ? r.weight[d] : 1.f) : v;
    };
    int64_t p = 0;
    if (a.R) p = min(max((int64_t)a.positions[t], (int64_t)0), a.length - 1);
    for (int i = 0; i < a.R / 2; ++i) {
        const int da = a.interleaved ? 2 * i : i, db = a.interleaved ? 2 * i + 1 : i + a.R / 2;
        const float c = a.table[i * a.length + p], n = a.table[(a.R / 2 + i) * a.length + p];
        const float u = at(da), v = at(db);
        y[da * r.ldy] = (T)(u * c - v * n);
        y[db * r.ldy] = (T)(u * n + v * c);
    }
    for (int d = a.R; d < a.D; ++d) y[d * r.ldy] = (T)at(d);
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

nmg_status launch_rotary(nmg_dtype dtype, const RotaryArgs &a, bool norm, hipStream_t stream) {
    const int64_t heads = (int64_t)a.part[0].heads + a.part[1].heads;
    if (heads > 65535) return NMG_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)((a.N + kBlock - 1) / kBlock), (unsigned)heads);
    if (dtype == NMG_F32 && norm)
        hipLaunchKernelGGL((k_rotary<float, true>), grid, dim3(kBlock), 0, stream, a);
    else if (dtype == NMG_F32)
        hipLaunchKernelGGL((k_rotary<float, false>), grid, dim3(kBlock), 0, stream, a);
    else if (norm)
        hipLaunchKernelGGL((k_rotary<_Float16, true>), grid, dim3(kBlock), 0, stream, a);
    else
        hipLaunchKernelGGL((k_rotary<_Float16, false>), grid, dim3(kBlock), 0, stream, a);
    return launched();
}

nmg_status launch_rotary_table(const RotaryTableArgs &a, hipStream_t stream) {
    const dim3 grid((unsigned)((a.length + kBlock - 1) / kBlock), (unsigned)a.half);
    hipLaunchKernelGGL(k_rotary_table, grid, dim3(kBlock), 0, stream, a);
    return launched();
}

}  // namespace nmg_internal

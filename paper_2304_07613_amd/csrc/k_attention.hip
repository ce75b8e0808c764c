// k_attention.hip -- attention of ranges of query columns to ranges of key
// columns, features x tokens.
//
//   k_attention  one workgroup per (query column, query head): keys 256 at a
//                time, a lane per key for the scores (every read of K is a run
//                of columns), one online softmax step per 256 keys, then a
//                lane per 8 rows of V for the weighted sum.
#include "attention.hpp"

namespace {

constexpr int kAttnKeys = kBlock;  // keys per step, one a thread

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_attention(AttnArgs a) {
    __shared__ float q[256], o[256], p[kAttnKeys], red[4];
    const int c = blockIdx.x, h = blockIdx.y, tid = threadIdx.x, D = a.D;
    int b = 0;
    while (b < a.sequences && !(a.q_offsets[b] <= c && c < a.q_offsets[b + 1])) ++b;
    if (b == a.sequences) return;
    const int q0 = a.q_offsets[b], n = a.q_offsets[b + 1] - q0;
    const int end = min(max(a.kv_end[b], 0), a.Nk), begin = max(a.kv_begin[b], 0);
    const T *Q = (const T *)a.Q + (int64_t)h * D * a.ldq + c;
    const T *K = (const T *)a.K + (int64_t)(h / a.share) * D * a.ldk;
    const T *V = (const T *)a.V + (int64_t)(h / a.share) * D * a.ldv;
    if (tid < D) {
        q[tid] = (float)Q[tid * a.ldq];
        o[tid] = 0.f;
    }
    float m = -INFINITY, l = 0.f;
    __syncthreads();
    for (int64_t k0 = begin; k0 < end; k0 += kAttnKeys) {
        const int64_t j = k0 + tid;
        bool see = j < end && (!a.key_mask || a.key_mask[j]);
        if (see && a.tree && j >= end - n) {
            const int64_t i = j - (end - n);
            see = i < a.width && a.tree[c * a.ldtree + i];
        }
        float s = -INFINITY;
        if (see) {
            float acc = 0.f;
            for (int d = 0; d < D; ++d) acc = fmaf(q[d], (float)K[d * a.ldk + j], acc);
            s = acc * a.scale;
        }
        const float wm = wave_max(s);
        if (tid % 64 == 0) red[tid / 64] = wm;
        __syncthreads();
        const float top = fmaxf(m, fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
        const float base = top == -INFINITY ? 0.f : top;  // nothing seen yet: every weight 0
        const float w = see ? expf(s - base) : 0.f;
        p[tid] = w;
        const float ws = wave_sum(w);
        __syncthreads();
        if (tid % 64 == 0) red[tid / 64] = ws;
        __syncthreads();
        const float keep = m == top ? 1.f : expf(m - base);
        l = l * keep + (red[0] + red[1] + red[2] + red[3]);
        m = top;
        for (int d = tid / 64; d < D; d += kBlock / 64) {
            float acc = 0.f;
            for (int i = tid % 64; i < kAttnKeys; i += 64)
                if (p[i] != 0.f) acc = fmaf(p[i], (float)V[d * a.ldv + k0 + i], acc);
            acc = wave_sum(acc);
            if (tid % 64 == 0) o[d] = o[d] * keep + acc;
        }
        __syncthreads();
    }
    if (tid < D)
        ((T *)a.O)[((int64_t)h * D + tid) * a.ldo + c] = (T)(l == 0.f ? 0.f : o[tid] / l);
}

}  // namespace

namespace nmg_internal {

int64_t attention_workspace_bytes(nmg_dtype, const AttnArgs &) { return 0; }

nmg_status launch_attention(nmg_dtype dtype, const AttnArgs &a, void *, int64_t,
                            hipStream_t stream) {
    const dim3 grid((unsigned)a.Nq, (unsigned)(a.kv_heads * a.share));
    if (grid.y > 65535) return NMG_ERR_UNSUPPORTED;
    if (dtype == NMG_F32)
        hipLaunchKernelGGL((k_attention<float>), grid, dim3(kBlock), 0, stream, a);
    else
        hipLaunchKernelGGL((k_attention<_Float16>), grid, dim3(kBlock), 0, stream, a);
    return launched();
}

}  // namespace nmg_internal

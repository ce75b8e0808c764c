// k_attention_f32.hip -- binary32 attention: many rows on bfloat16 parts
// (attention_parts.hpp), few rows and heads over 128 on the binary32 matrix
// instructions (attention_mfma.hpp).
#include "attention_parts.hpp"

namespace {

template <int DP, bool WIDE>
void launch_how(const AttnArgs &a, bool shared, dim3 grid, hipStream_t stream) {
    constexpr AttnRows how = WIDE ? kAttnWide : kAttnNarrow;
    if (!shared) {
        hipLaunchKernelGGL((k_attn_split<float, DP, how>), grid, dim3(64 * attn_split_waves(DP)), 0,
                           stream, a);
    } else {
        if constexpr (DP <= 128)
            hipLaunchKernelGGL((k_attn_parts<DP, WIDE>), grid, dim3(256), 0, stream, a);
        else
            hipLaunchKernelGGL((k_attn_shared<float, DP, how>), grid, dim3(256), 0, stream, a);
    }
}

template <typename T, int DP>
void launch_main(const AttnArgs &a, bool shared, AttnRows how, dim3 grid, hipStream_t stream) {
    if (how == kAttnNarrow)
        launch_how<DP, false>(a, shared, grid, stream);
    else
        launch_how<DP, true>(a, shared, grid, stream);
}

}  // namespace

namespace nmg_internal {
nmg_status launch_attention_f32(const AttnArgs &a, bool shared, AttnRows how, hipStream_t stream) {
    return launch_attn<float>(a, shared, how, stream);
}
}  // namespace nmg_internal

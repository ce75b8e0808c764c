// k_attention_f16.hip -- binary16 attention (attention_mfma.hpp).
#include "attention_mfma.hpp"

namespace {

template <int DP, AttnRows HOW>
void launch_how(const AttnArgs &a, bool shared, dim3 grid, hipStream_t stream) {
    if (shared)
        hipLaunchKernelGGL((k_attn_shared<_Float16, DP, HOW>), grid, dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL((k_attn_split<_Float16, DP, HOW>), grid, dim3(64 * attn_split_waves(DP)), 0,
                           stream, a);
}

template <typename T, int DP>
void launch_main(const AttnArgs &a, bool shared, AttnRows how, dim3 grid, hipStream_t stream) {
    if (how == kAttnNarrow)
        launch_how<DP, kAttnNarrow>(a, shared, grid, stream);
    else if (how == kAttnWide)
        launch_how<DP, kAttnWide>(a, shared, grid, stream);
    else
        launch_how<DP, kAttnShift>(a, shared, grid, stream);
}

}  // namespace

namespace nmg_internal {
nmg_status launch_attention_f16(const AttnArgs &a, bool shared, AttnRows how, hipStream_t stream) {
    return launch_attn<_Float16>(a, shared, how, stream);
}
}  // namespace nmg_internal

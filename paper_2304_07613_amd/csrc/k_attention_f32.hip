// k_attention_f32.hip -- binary32 attention (attention_mfma.hpp).
#include "attention_mfma.hpp"

namespace nmg_internal {
nmg_status launch_attention_f32(const AttnArgs &a, bool shared, bool regs, hipStream_t stream) {
    return launch_attn<float>(a, shared, regs, stream);
}
}  // namespace nmg_internal

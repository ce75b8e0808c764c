// k_attention_f16.hip -- binary16 attention (attention_mfma.hpp).
#include "attention_mfma.hpp"

namespace nmg_internal {
nmg_status launch_attention_f16(const AttnArgs &a, bool shared, bool regs, hipStream_t stream) {
    return launch_attn<_Float16>(a, shared, regs, stream);
}
}  // namespace nmg_internal

// k_cache_attention_f32.hip -- cache_attention.hpp for binary32 activations.
#include "cache_attention.hpp"

namespace nmg_internal {

nmg_status cache_attention_f32(nmg_cache_format format, const CacheAttnArgs &a, CacheAttnRows rows,
                               hipStream_t stream) {
    const int tiles = (a.c.D + 15) / 16;
    if (rows == kRows16)
        return tiles > 8   ? run_cache_attention<float, 16, 1>(format, a, stream)
               : tiles > 6 ? run_cache_attention<float, 8, 1>(format, a, stream)
               : tiles > 4 ? run_cache_attention<float, 6, 1>(format, a, stream)
                           : run_cache_attention<float, 4, 1>(format, a, stream);
    return tiles > 4 ? run_cache_attention<float, 8, 2>(format, a, stream)
                     : run_cache_attention<float, 4, 2>(format, a, stream);
}

}  // namespace nmg_internal

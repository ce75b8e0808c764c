// k_cache_attention_f16.hip -- cache_attention.hpp for binary16 activations.
#include "cache_attention.hpp"

namespace nmg_internal {

nmg_status cache_attention_f16(nmg_cache_format format, const CacheAttnArgs &a, CacheAttnRows rows,
                               hipStream_t stream) {
    const int tiles = (a.c.D + 15) / 16;
    switch (rows) {
    case kRows16:
        return tiles > 8   ? run_cache_attention<_Float16, 16, 1>(format, a, stream)
               : tiles > 6 ? run_cache_attention<_Float16, 8, 1>(format, a, stream)
               : tiles > 4 ? run_cache_attention<_Float16, 6, 1>(format, a, stream)
                           : run_cache_attention<_Float16, 4, 1>(format, a, stream);
    case kRows32:
        return tiles > 6   ? run_cache_attention<_Float16, 8, 2>(format, a, stream)
               : tiles > 4 ? run_cache_attention<_Float16, 6, 2>(format, a, stream)
                           : run_cache_attention<_Float16, 4, 2>(format, a, stream);
    case kRows64:
        return run_cache_attention<_Float16, 16, 1, true>(format, a, stream);
    default:
        return tiles > 6   ? run_cache_attention<_Float16, 8, 2, true>(format, a, stream)
               : tiles > 4 ? run_cache_attention<_Float16, 6, 2, true>(format, a, stream)
                           : run_cache_attention<_Float16, 4, 2, true>(format, a, stream);
    }
}

}  // namespace nmg_internal

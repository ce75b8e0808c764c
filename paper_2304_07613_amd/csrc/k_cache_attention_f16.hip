// k_cache_attention_f16.hip -- cache_attention.hpp for binary16 activations.
#include "cache_attention.hpp"

namespace nmg_internal {

nmg_status cache_attention_f16(nmg_cache_format format, const CacheAttnArgs &a, int nt,
                               hipStream_t stream) {
    const int tiles = (a.c.D + 15) / 16;
    if (tiles > 8) return nt == 1 ? run_cache_attention<_Float16, 16, 1>(format, a, stream)
                                  : run_cache_attention<_Float16, 16, 2>(format, a, stream);
    if (tiles > 6) return nt == 1   ? run_cache_attention<_Float16, 8, 1>(format, a, stream)
                          : nt == 2 ? run_cache_attention<_Float16, 8, 2>(format, a, stream)
                                    : run_cache_attention<_Float16, 8, 4>(format, a, stream);
    if (tiles > 4) return nt == 1   ? run_cache_attention<_Float16, 6, 1>(format, a, stream)
                          : nt == 2 ? run_cache_attention<_Float16, 6, 2>(format, a, stream)
                                    : run_cache_attention<_Float16, 6, 4>(format, a, stream);
    return nt == 1   ? run_cache_attention<_Float16, 4, 1>(format, a, stream)
           : nt == 2 ? run_cache_attention<_Float16, 4, 2>(format, a, stream)
                     : run_cache_attention<_Float16, 4, 4>(format, a, stream);
}

}  // namespace nmg_internal

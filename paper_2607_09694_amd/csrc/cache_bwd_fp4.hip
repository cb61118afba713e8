// The backward over a source stack in 4 bits (e2m1).
#include "cache_bwd.h"

namespace lrar {

hipError_t launch_cache_bwd_fp4(const CacheProblem &p, const void *dH, void *dV, void *dK,
                                float *coef, bool deferred, float *partial, bool accumulate,
                                hipStream_t st)
{
    return p.dtype == LRAR_DTYPE_BF16
               ? launch_cache_bwd_as<LRAR_CACHE_FP4, uint16_t>(p, dH, dV, dK, coef, deferred,
                                                               partial, accumulate, st)
               : launch_cache_bwd_as<LRAR_CACHE_FP4, float>(p, dH, dV, dK, coef, deferred,
                                                            partial, accumulate, st);
}

}  // namespace lrar

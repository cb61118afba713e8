// Host-side interface of the kernels over a source stack in 8 or 4 bits.
// Internal to the library.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <string>

#include "lr_attnres_cache.h"

namespace lrar {

constexpr int kCacheBlock = 32;  // columns that share a scale

inline int64_t cache_blocks(int64_t d) { return (d + kCacheBlock - 1) / kCacheBlock; }
inline int64_t cache_row_bytes(int64_t d, int format)
{
    return cache_blocks(d) * (format == LRAR_CACHE_FP8 ? kCacheBlock : kCacheBlock / 2);
}

// One read site over a cache (validated by the C ABI layer).
struct CacheProblem {
    const uint8_t *codes, *scales;
    const void *K;   // [S][N][r] (projected keys) or NULL
    const float *q;  // [r]
    int64_t S, N, d, r;
    int mode, format, dtype;
    float eps;
};

int check_cache_supported(const CacheProblem &p, bool bwd, std::string *why);
size_t cache_bwd_workspace_bytes(const CacheProblem &p);

int launch_cache_write(const void *O, uint8_t *codes, uint8_t *scales, int64_t rows, int64_t d,
                       int format, int dtype, hipStream_t st, std::string *err);
int launch_cache_read(const uint8_t *codes, const uint8_t *scales, void *O, int64_t rows,
                      int64_t d, int format, int dtype, hipStream_t st, std::string *err);
// o_new: NULL, or the rows that plane S-1 (codes and scales writable) takes first.
int launch_cache_fwd(const CacheProblem &p, const void *o_new, void *H, hipStream_t st,
                     std::string *err);
// coef: NULL for gradient rows (dV, dK; added to when accumulating), or the
// deferred form's coefficients.
int launch_cache_bwd(const CacheProblem &p, const void *dH, void *dV, void *dK, float *coef,
                     float *dq, void *ws, bool accumulate, hipStream_t st, std::string *err);

}  // namespace lrar

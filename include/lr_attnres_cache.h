/*
 * lr_attnres_cache.h - the source stack in 8 or 4 bits: quantising a source
 * as it is written, reading it back, and the depth routing of lr_attnres.h
 * over such a stack, forward and backward (LR-AttnRes, arXiv 2607.09694).
 *
 * The values o_0 .. o_{S-1} that every read site attends over (Sec. 3.1) are
 * the bytes of a model pass and of its activation memory (Appendix A
 * "Activation memory").  A cache holds them in blocks of 32 columns with one
 * scale byte each.  The paper states no storage below bf16; the format is
 * this library's reading:
 *   - a row of d columns is nb = ceil(d / 32) blocks, the columns past d zero;
 *   - scales [S][N][nb] bytes: e stands for 2^(e - 127), and 255 makes every
 *     value of its block NaN;
 *   - codes  LRAR_CACHE_FP8 [S][N][32 nb] bytes: e4m3 (sign, 4 exponent, 3
 *                           mantissa bits; magnitudes up to 448);
 *            LRAR_CACHE_FP4 [S][N][16 nb] bytes: e2m1 (0, 0.5, 1, 1.5, 2, 3, 4,
 *                           6), two columns a byte, the even one in the low half;
 *   - a value is its code times its block's power of two.
 * Sources are planes, so the first S' sources of a deeper cache are a cache,
 * and so is one plane.  Keys, queries, routed states and gradients keep the
 * storage `dtype` (fp32 or bf16); arithmetic is fp32.
 *
 * Execution, ownership, error codes and lr_attnres_last_error are those of
 * lr_attnres.h.  codes are 16-byte aligned; scales need no alignment.
 */
#ifndef LR_ATTNRES_CACHE_H
#define LR_ATTNRES_CACHE_H

#include "lr_attnres.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { LRAR_CACHE_FP8 = 0, LRAR_CACHE_FP4 = 1 };

/* Bytes of one row's codes and of its scales; 0 for d < 1, d > 2^20 or an
 * unknown format. */
size_t lr_attnres_cache_row_bytes(int64_t d, int format);
size_t lr_attnres_cache_row_scales(int64_t d);

/*
 * Quantises `rows` rows O [rows][d] (storage `dtype`) into codes and scales;
 * for one source of N tokens, rows = N and the pointers are its plane's.
 * Per block: e is the smallest of 1 .. 254 with max |x| <= M 2^(e - 127), M the
 * largest code (448 or 6), so nothing saturates; a code is x 2^(127 - e), an
 * exact product, rounded to nearest even.  A block that holds a NaN or an
 * infinity gets e = 255 and codes 0.  Magnitudes from (1 - 2^-5) 2^128 on (e2m1:
 * (1 - 2^-3) 2^128) round to 2^128, which fp32 does not hold: they read as
 * infinities.  O needs element alignment only.
 * EINVAL: rows < 0, d < 1, unknown format or storage, NULL or misaligned
 * pointers, overlapping buffers, a size overflowing int64.  EUNSUPPORTED:
 * rows above 2^40, d above 2^20, more than about 2^31 workgroups' worth.
 */
int lr_attnres_cache_write(const void *O, void *codes, void *scales, int64_t rows, int64_t d,
                           int format, int dtype, void *stream);

/* The values of `rows` rows into O [rows][d], storage `dtype`: exact in fp32
 * and, down to bf16's subnormals, in bf16.  Errors as for the write. */
int lr_attnres_cache_read(const void *codes, const void *scales, void *O, int64_t rows, int64_t d,
                          int format, int dtype, void *stream);

/*
 * lr_attnres_route_fwd over a cache: h = sum_i alpha_i x_i with x_i the values
 * that the cache holds, sliced keys being the last r columns of x_i and
 * full-rank keys x_i itself.
 *   K [S][N][r] storage `dtype` (projected keys, else NULL), q [r] fp32,
 *   H [N][d] storage `dtype`, overwritten.
 *   o_new: NULL, or [N][d] storage `dtype`, the newest source: plane S-1 of
 *       codes and scales is first overwritten with it as by
 *       lr_attnres_cache_write, and the site reads that plane as every later
 *       site will.  With o_new NULL codes and scales are only read.
 * Errors as for lr_attnres_route_fwd, plus EINVAL for an unknown format.
 * EUNSUPPORTED: S > 1024, N > 2^25, full-rank keys with d > 4096, d > 2^20,
 * projected keys with r > 2^20.
 */
int lr_attnres_cache_route_fwd(void *codes, void *scales, const void *K, const float *q,
                               const void *o_new, void *H, int64_t S, int64_t N, int64_t d,
                               int64_t r, int mode, int format, int dtype, float eps,
                               void *stream);

/*
 * lr_attnres_route_bwd over a cache: the gradients of L = sum_n dH[n] . h[n]
 * with respect to the values x_i that the cache holds (training hands them to
 * the sources unchanged, through the rounding), to K and to q.  codes and
 * scales are the 8- or 4-bit checkpoints of the sources, read only.
 *   dH [N][d], dV [S][N][d], dK [S][N][r] (projected keys, else NULL) storage
 *   `dtype`, dq [r] fp32; accumulate = 0 overwrites dV, dK and dq, 1 adds.
 *   workspace: lr_attnres_cache_route_bwd_workspace_bytes(...) bytes, 16-byte
 *   aligned (NULL when that is 0); what serves S sources serves fewer.
 * Results are bitwise reproducible.  Errors as for lr_attnres_route_bwd, plus
 * EINVAL for an unknown format and accumulate not 0 or 1.  EUNSUPPORTED:
 * S > 512, N > 2^25, projected or sliced keys with r > 256, d > 4096.
 */
size_t lr_attnres_cache_route_bwd_workspace_bytes(int64_t S, int64_t N, int64_t d, int64_t r,
                                                  int mode, int format, int dtype);
int lr_attnres_cache_route_bwd(const void *codes, const void *scales, const void *K,
                               const float *q, const void *dH, void *dV, void *dK, float *dq,
                               void *workspace, size_t workspace_bytes, int64_t S, int64_t N,
                               int64_t d, int64_t r, int mode, int format, int dtype, float eps,
                               int accumulate, void *stream);

/*
 * lr_attnres_route_bwd_deferred over a cache: one site of the reverse pass in
 * deferred form.  coef [S][3][N] fp32 (alpha, ds / rho, ds s / (rho r) of every
 * source and token) and dq [r] fp32, overwritten.  lr_attnres_route_gather_bwd
 * then forms a source's gradient from the sites that read it (projected keys
 * from K alone; sliced keys from the source's plane, read back by
 * lr_attnres_cache_read).  Projected or sliced keys (full rank: EUNSUPPORTED);
 * workspace, limits and errors as for lr_attnres_cache_route_bwd.
 */
int lr_attnres_cache_route_bwd_deferred(const void *codes, const void *scales, const void *K,
                                        const float *q, const void *dH, float *coef, float *dq,
                                        void *workspace, size_t workspace_bytes, int64_t S,
                                        int64_t N, int64_t d, int64_t r, int mode, int format,
                                        int dtype, float eps, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* LR_ATTNRES_CACHE_H */

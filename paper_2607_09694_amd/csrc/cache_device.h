// Device-side building blocks over a source stack in 8 or 4 bits: decoding and
// encoding of codes with their block scales, key loads and scores.
//
// gfx950 converts both formats in hardware, two values an instruction at full
// rate, with the block's power of two applied by the same instruction: the
// scale operand is the fp32 number whose exponent field is the scale byte.
// Checked over every code and every scale byte: exact, 255 gives NaN and 0
// gives 2^-127; encoding rounds to nearest even.
#pragma once

#include "cache_launch.h"
#include "route_common.h"

namespace lrar {

constexpr int kCacheVec = 16;  // columns that a lane loads at once in the row streams

// Codes of 16 and of 8 columns as one lane loads them.
template <int FMT> struct Codes;
template <> struct Codes<LRAR_CACHE_FP8> {
    typedef u32x4_t row_t;
    typedef u32x2_t key_t;
    static constexpr int per_byte = 1;  // columns a byte
};
template <> struct Codes<LRAR_CACHE_FP4> {
    typedef u32x2_t row_t;
    typedef unsigned key_t;
    static constexpr int per_byte = 2;
};

__device__ __forceinline__ float block_scale(unsigned e) { return __uint_as_float(e << 23); }

// 4 e4m3 or 8 e2m1 codes of one word to fp32, times the block's scale.
__device__ __forceinline__ void decode_fp8(unsigned w, float sc, float *x)
{
    const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, sc, false);
    const f32x2_t b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, sc, true);
    x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
}
__device__ __forceinline__ void decode_fp4(unsigned w, float sc, float *x)
{
    const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 0);
    const f32x2_t b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 1);
    const f32x2_t c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 2);
    const f32x2_t e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 3);
    x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
    x[4] = c.x; x[5] = c.y; x[6] = e.x; x[7] = e.y;
}
template <int FMT>
__device__ __forceinline__ void decode(const u32x4_t &w, float sc, float (&x)[16])
{
    static_assert(FMT == LRAR_CACHE_FP8, "16 one-byte codes");
    decode_fp8(w.x, sc, x);
    decode_fp8(w.y, sc, x + 4);
    decode_fp8(w.z, sc, x + 8);
    decode_fp8(w.w, sc, x + 12);
}
template <int FMT>
__device__ __forceinline__ void decode(const u32x2_t &w, float sc, float (&x)[16])
{
    static_assert(FMT == LRAR_CACHE_FP4, "16 half-byte codes");
    decode_fp4(w.x, sc, x);
    decode_fp4(w.y, sc, x + 8);
}
template <int FMT>
__device__ __forceinline__ void decode(const u32x2_t &w, float sc, float (&x)[8])
{
    static_assert(FMT == LRAR_CACHE_FP8, "8 one-byte codes");
    decode_fp8(w.x, sc, x);
    decode_fp8(w.y, sc, x + 4);
}
template <int FMT>
__device__ __forceinline__ void decode(const unsigned &w, float sc, float (&x)[8])
{
    static_assert(FMT == LRAR_CACHE_FP4, "8 half-byte codes");
    decode_fp4(w, sc, x);
}

// The scale byte of a block from the largest magnitude in it: the smallest e in
// 1 .. 254 with top <= M 2^(e - 127), M = 1.75 * 2^8 (e4m3) or 1.5 * 2^2 (e2m1);
// 255 where top is an infinity or NaN.
template <int FMT> __device__ __forceinline__ unsigned scale_byte(float top)
{
    const unsigned u = __float_as_uint(top);
    constexpr int shift = FMT == LRAR_CACHE_FP8 ? 8 : 2;
    constexpr unsigned over = FMT == LRAR_CACHE_FP8 ? 0x600000u : 0x400000u;
    const int e = (int)(u >> 23) - shift + ((u & 0x7fffffu) > over ? 1 : 0);
    return u >= 0x7f800000u ? 255u : (unsigned)max(e, 1);
}

// 8 values to codes, each divided by the block's scale and rounded to nearest
// even (codes 0 where the block is NaN).
template <int FMT>
__device__ __forceinline__ typename Codes<FMT>::key_t encode(const float (&x)[8], unsigned e)
{
    const float sc = block_scale(e);
    if constexpr (FMT == LRAR_CACHE_FP8) {
        typedef short s16x2_t __attribute__((ext_vector_type(2)));
        s16x2_t a = {0, 0}, b = {0, 0};
        a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(a, x[0], x[1], sc, false);
        a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(a, x[2], x[3], sc, true);
        b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, x[4], x[5], sc, false);
        b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, x[6], x[7], sc, true);
        const u32x2_t c = {__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b)};
        return e == 255u ? u32x2_t{0u, 0u} : c;
    } else {
        unsigned c = 0u;
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], sc, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], sc, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], sc, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], sc, 3);
        return e == 255u ? 0u : c;
    }
}

// Larger magnitude, NaN winning.
__device__ __forceinline__ float max_magnitude(float a, float b)
{
    // Magnitudes order as their bits do, with NaN above infinity.
    return __uint_as_float(max(__float_as_uint(a) & 0x7fffffffu, __float_as_uint(b) & 0x7fffffffu));
}

// 8 consecutive elements of a row of `width` (zeros past its end): one or two
// 16-byte accesses where the rows allow it (vec: width % 8 == 0, aligned base),
// else element by element.
template <typename T>
__device__ __forceinline__ void load8(const T *__restrict__ row, int col, int width, bool vec,
                                      float (&x)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e)
        x[e] = 0.0f;
    if (vec) {
        if (col < width) {
            if constexpr (sizeof(T) == 2) {
                widen(load_raw<T, 8>(row + col), x);
            } else {
                const f32x4_t a = load_raw<T, 4>(row + col), b = load_raw<T, 4>(row + col + 4);
                x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
                x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (col + e < width)
                x[e] = load_elem(row + col + e);
    }
}

template <typename T, bool NT>
__device__ __forceinline__ void store8(T *__restrict__ row, int col, int width, bool vec,
                                       const float (&y)[8])
{
    if (vec) {
        if (col < width) {
            if constexpr (sizeof(T) == 2) {
                store_stream<T, 8, NT>(row + col, Narrow<T, 8>::run(y));
            } else {
                store_stream<T, 4, NT>(row + col, f32x4_t{y[0], y[1], y[2], y[3]});
                store_stream<T, 4, NT>(row + col + 4, f32x4_t{y[4], y[5], y[6], y[7]});
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (col + e < width)
                store_elem(row + col + e, y[e]);
    }
}

// ---------------------------------------------------------------------------
// Keys: slots of 8 elements, the r key elements from a separate row of K
// (projected) or the columns [d - r, d) of the cache's row (sliced)
// ---------------------------------------------------------------------------

// How a wave reads the keys of a site.  Sliced keys start at slot column
// `base` = (d - r) / 8 * 8, of which the first d - r - base elements are not
// the key's; `lps` lanes (a power of two, at most 64) read one source's key.
template <int FMT, typename T, bool SLICED> struct Keys {
    const T *__restrict__ K;
    const uint8_t *__restrict__ codes, *__restrict__ scales;
    int N, d, r, nb, base, nkv, lps;
    bool vec;

    __device__ Keys(const void *K_, const uint8_t *codes_, const uint8_t *scales_, int N_, int d_,
                    int r_)
        : K(static_cast<const T *>(K_)), codes(codes_), scales(scales_), N(N_), d(d_), r(r_),
          nb((d_ + kCacheBlock - 1) / kCacheBlock), base(SLICED ? (d_ - r_) / 8 * 8 : 0),
          nkv(((SLICED ? d_ - base : r_) + 7) / 8), lps(1), vec(r_ % 8 == 0)
    {
        while (lps < nkv && lps < kWaveSize)
            lps <<= 1;
    }
    // First of the query's elements that slot v meets (below 0: not the key's).
    __device__ int first(int v) const { return v * 8 + base - (SLICED ? d - r : 0); }
    __device__ void query(const float *__restrict__ q, int v, float (&x)[8]) const
    {
        const int j = first(v);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            x[e] = v < nkv && j + e >= 0 && j + e < r ? q[j + e] : 0.0f;
    }
    struct Raw {
        typename Codes<FMT>::key_t c;
        unsigned e;
        float x[8];
    };
    // Slot v of source i and token n (both in range; slots past the key re-read
    // the last one).
    __device__ __forceinline__ void load(int i, int n, int v, Raw &w) const
    {
        v = min(v, nkv - 1);
        const size_t row = (size_t)i * N + n;
        if constexpr (SLICED) {
            const int col = base + v * 8;
            const size_t at = row * nb * (kCacheBlock / Codes<FMT>::per_byte) +
                              (unsigned)(col / Codes<FMT>::per_byte);
            w.c = *reinterpret_cast<const typename Codes<FMT>::key_t *>(codes + at);
            w.e = scales[row * nb + (unsigned)col / kCacheBlock];
        } else {
            load8(K + row * r, v * 8, r, vec, w.x);
        }
    }
    // Its values, zeros where the slot's elements are not the key's.
    __device__ __forceinline__ void values(const Raw &w, int v, float (&x)[8]) const
    {
        if constexpr (SLICED) {
            decode<FMT>(w.c, block_scale(w.e), x);
            const int j = first(v);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                x[e] = j + e >= 0 ? x[e] : 0.0f;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                x[e] = w.x[e];
        }
    }
};

// Scores s_i = q . k_i / rho_i and (rho_out) rho_i of the sources [ib, ie) of
// TW consecutive tokens (tokens past N are read as token N-1 and not written),
// into s_out[t * s_pad + i].  A group of lps lanes reads one source's key, so
// 64 / lps sources are scored together, and KP such groups' loads of every
// token go out before the first is used.  The caller waits for the LDS writes.
template <int FMT, typename T, bool SLICED, int TW>
__device__ __forceinline__ void cache_scores(const Keys<FMT, T, SLICED> &k,
                                             const float *__restrict__ q, int ib, int ie,
                                             int n0, float eps, int lane, float *s_out,
                                             float *rho_out, int s_pad)
{
    constexpr int KP = TW >= 2 ? 2 : 4;
    const int lps = k.lps, spi = kWaveSize / lps;
    const int isub = lane / lps, v = lane % lps;
    const float inv_r = 1.0f / (float)k.r;
    if (k.nkv <= lps) {
        float qv[8];
        k.query(q, v, qv);
        const bool vok = v < k.nkv;
        for (int i0 = ib; i0 < ie; i0 += KP * spi) {
            typename Keys<FMT, T, SLICED>::Raw w[TW][KP];
#pragma unroll
            for (int t = 0; t < TW; ++t)
#pragma unroll
                for (int p = 0; p < KP; ++p)
                    k.load(min(i0 + p * spi + isub, ie - 1), min(n0 + t, k.N - 1), v, w[t][p]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < TW; ++t)
#pragma unroll
                for (int p = 0; p < KP; ++p) {
                    float x[8];
                    k.values(w[t][p], v, x);
                    float ss = 0.0f, dot = 0.0f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        ss = fmaf(x[e], x[e], ss);
                        dot = fmaf(qv[e], x[e], dot);
                    }
                    if (!vok)
                        ss = dot = 0.0f;
                    butterfly_sum2<true>(ss, dot, lps);
                    const int i = i0 + p * spi + isub;
                    if (v == 0 && i < ie && n0 + t < k.N) {
                        const float rho = sqrtf(ss * inv_r + eps);
                        s_out[t * s_pad + i] = dot / rho;
                        if (rho_out)
                            rho_out[t * s_pad + i] = rho;
                    }
                }
        }
        return;
    }
    for (int t = 0; t < TW; ++t) {
        const int n = n0 + t;
        if (n >= k.N)
            break;
        for (int i = ib; i < ie; ++i) {  // keys of more than 64 slots: the wave reads one
            float ss = 0.0f, dot = 0.0f;
            for (int vv = lane; vv < k.nkv; vv += kWaveSize) {
                typename Keys<FMT, T, SLICED>::Raw w;
                float x[8], qv[8];
                k.load(i, n, vv, w);
                k.query(q, vv, qv);
                k.values(w, vv, x);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    ss = fmaf(x[e], x[e], ss);
                    dot = fmaf(qv[e], x[e], dot);
                }
            }
            butterfly_sum2<true>(ss, dot, kWaveSize);
            if (lane == 0) {
                const float rho = sqrtf(ss * inv_r + eps);
                s_out[t * s_pad + i] = dot / rho;
                if (rho_out)
                    rho_out[t * s_pad + i] = rho;
            }
        }
    }
}

// Where a lane reads its 16 columns of a chunk of 1024: bytes into the row's
// codes and the index of its scale.  Lanes past the row re-read its last 16
// columns (in range; what they compute reaches no output).
template <int FMT> struct RowAt {
    int code, scale;
    __device__ RowAt(int col, int nb)
    {
        const int c = min(col, nb * kCacheBlock - kCacheVec);
        code = c / Codes<FMT>::per_byte;
        scale = c / kCacheBlock;
    }
};

template <int FMT> struct RowRaw {
    typename Codes<FMT>::row_t c;
    unsigned e;
};

template <int FMT>
__device__ __forceinline__ void load_row(const uint8_t *__restrict__ codes,
                                         const uint8_t *__restrict__ scales, size_t row, int nb,
                                         const RowAt<FMT> &at, RowRaw<FMT> &w)
{
    typedef typename Codes<FMT>::row_t row_t;
    const row_t *p = reinterpret_cast<const row_t *>(
        codes + row * nb * (kCacheBlock / Codes<FMT>::per_byte) + at.code);
    w.c = __builtin_nontemporal_load(p);
    w.e = scales[row * nb + at.scale];
}

template <int FMT>
__device__ __forceinline__ void row_values(const RowRaw<FMT> &w, float (&x)[16])
{
    decode<FMT>(w.c, block_scale(w.e), x);
}

// Calls f(std::integral_constant<int, NCH>) for rows of up to 1024 NCH columns.
template <typename F> hipError_t dispatch_row_chunks(int64_t d, F &&f)
{
    if (d <= 1024)
        return f(std::integral_constant<int, 1>{});
    if (d <= 2048)
        return f(std::integral_constant<int, 2>{});
    return f(std::integral_constant<int, 4>{});
}

}  // namespace lrar

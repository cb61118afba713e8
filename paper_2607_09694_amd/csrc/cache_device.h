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

// Codes of 8 columns, and how they are packed.
template <int FMT> struct Codes;
template <> struct Codes<LRAR_CACHE_FP8> {
    typedef u32x2_t key_t;
    static constexpr int per_byte = 1;  // columns a byte
};
template <> struct Codes<LRAR_CACHE_FP4> {
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

// 16 bytes at an address that is aligned to its elements only.  gfx950 moves them
// in one access; rows of any width take the vector path.
typedef u32x4_t u32x4_u __attribute__((aligned(2)));
template <bool NT> __device__ __forceinline__ u32x4_t load16(const void *p)
{
    const u32x4_u *v = reinterpret_cast<const u32x4_u *>(p);
    if constexpr (NT)
        return __builtin_nontemporal_load(v);
    else
        return *v;
}
template <bool NT> __device__ __forceinline__ void store16(void *p, u32x4_t x)
{
    u32x4_u *v = reinterpret_cast<u32x4_u *>(p);
    if constexpr (NT)
        __builtin_nontemporal_store(u32x4_u(x), v);
    else
        *v = x;
}

// VO = 16 / sizeof(T) consecutive elements of a row of `width` as they are stored,
// zeros past its end.
template <typename T>
__device__ __forceinline__ u32x4_t load16_elems(const T *__restrict__ row, int col, int width)
{
    constexpr int VO = 16 / sizeof(T);
    if (col + VO <= width)
        return load16<false>(row + col);
    u32x4_t w = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < VO; ++e)
        if (col + e < width) {
            if constexpr (sizeof(T) == 2)
                w[e / 2] |= (unsigned)row[col + e] << (16 * (e % 2));
            else
                w[e] = __float_as_uint(row[col + e]);
        }
    return w;
}
template <typename T, bool NT>
__device__ __forceinline__ void store16_elems(T *__restrict__ row, int col, int width, u32x4_t w)
{
    constexpr int VO = 16 / sizeof(T);
    if (col + VO <= width) {
        store16<NT>(row + col, w);
        return;
    }
#pragma unroll
    for (int e = 0; e < VO; ++e)
        if (col + e < width) {
            if constexpr (sizeof(T) == 2)
                row[col + e] = (uint16_t)(w[e / 2] >> (16 * (e % 2)));
            else
                row[col + e] = __uint_as_float(w[e]);
        }
}

// 8 consecutive elements, stored and widened.
template <typename T> struct Raw8 {
    u32x4_t w[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ void load8_raw(const T *__restrict__ row, int col, int width, Raw8<T> &x)
{
#pragma unroll
    for (int k = 0; k < (int)sizeof(T) / 2; ++k)
        x.w[k] = load16_elems(row, col + 4 * k, width);
}
template <typename T> __device__ __forceinline__ void widen8(const Raw8<T> &r, float (&x)[8])
{
    if constexpr (sizeof(T) == 2) {
        widen(r.w[0], x);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            x[k] = __uint_as_float(r.w[k / 4][k % 4]);
    }
}
template <typename T>
__device__ __forceinline__ void load8(const T *__restrict__ row, int col, int width, float (&x)[8])
{
    Raw8<T> r;
    load8_raw(row, col, width, r);
    widen8(r, x);
}
template <typename T, bool NT>
__device__ __forceinline__ void store8(T *__restrict__ row, int col, int width, const float (&y)[8])
{
    if constexpr (sizeof(T) == 2) {
        store16_elems<T, NT>(row, col, width, Narrow<T, 8>::run(y));
    } else {
#pragma unroll
        for (int k = 0; k < 2; ++k)
            store16_elems<T, NT>(row, col + 4 * k, width,
                                 u32x4_t{__float_as_uint(y[4 * k]), __float_as_uint(y[4 * k + 1]),
                                         __float_as_uint(y[4 * k + 2]), __float_as_uint(y[4 * k + 3])});
    }
}

// ---------------------------------------------------------------------------
// Rows: a lane takes 16 bytes of codes at a time (a unit: 16 columns of e4m3, 32
// of e2m1), LG lanes (16, 32 or 64) a row
// ---------------------------------------------------------------------------

// The codes of a unit and the scale byte of its block.  Rows of LG < 64 lanes
// share a wave, so that a load instruction covers the adjacent rows of 64 / LG
// tokens of one source.  (Two loads of 16 bytes a lane, 32 bytes apart from the
// next lane's, read e4m3 rows 10% to 15% slower.)
template <int FMT> struct UnitRaw {
    static constexpr int cols = FMT == LRAR_CACHE_FP8 ? 16 : 32;
    u32x4_t c;
    unsigned e;
};
template <int FMT> constexpr int unit_cols() { return UnitRaw<FMT>::cols; }

// Unit `at` after the one that codes points to (uniform; scales to its block).
template <int FMT>
__device__ __forceinline__ void load_unit(const uint8_t *codes, const uint8_t *scales,
                                          unsigned at, UnitRaw<FMT> &w)
{
    w.c = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(codes + at * 16u));
    w.e = scales[at * (unsigned)unit_cols<FMT>() / kCacheBlock];
}

// Columns [16 h, 16 h + 16) of the unit.
template <int FMT>
__device__ __forceinline__ void unit_values(const UnitRaw<FMT> &w, int h, float (&x)[16])
{
    const float sc = block_scale(w.e);
    if constexpr (FMT == LRAR_CACHE_FP8) {
        decode<FMT>(w.c, sc, x);
    } else {
        const u32x2_t c = h == 0 ? u32x2_t{w.c.x, w.c.y} : u32x2_t{w.c.z, w.c.w};
        decode<FMT>(c, sc, x);
    }
}

// use(a, i) for i = ib, ib + step, .. < ie (at least one), where load(a, i) reads what
// it uses.  The next trip's loads are in flight over this one's arithmetic, in two
// buffers in turn; a holds trip ib already.  Without / with: full-rank forward, e2m1,
// 49 sources, d = 1024, 4096 tokens 40.9 / 36.1 us, 16384 tokens 142 / 122; sliced r =
// 64, 33 x 4099 x 1024, e2m1, 25.5 / 22.8.
template <typename B, typename L, typename U>
__device__ __forceinline__ void pipelined(int ib, int ie, int step, B &a, L &&load, U &&use)
{
    B b;
    int i = ib;
    for (; i + 2 * step < ie; i += 2 * step) {
        load(b, i + step);
        __builtin_amdgcn_sched_barrier(0);
        use(a, i);
        __builtin_amdgcn_sched_barrier(0);
        load(a, i + 2 * step);
        __builtin_amdgcn_sched_barrier(0);
        use(b, i + step);
        __builtin_amdgcn_sched_barrier(0);
    }
    if (i + step < ie) {
        load(b, i + step);
        __builtin_amdgcn_sched_barrier(0);
        use(a, i);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_memcpy(&a, &b, sizeof(B));
        i += step;
    }
    use(a, i);
}

// Lane layout of the rows of d columns: units lu, lu + LG, .. (NCH of them) of the
// rows of group g.  Lanes past the row re-read its last unit (in range; in[c] says
// which units count).
template <int FMT, int LG, int NCH> struct Lanes {
    static constexpr int groups = kWaveSize / LG;
    int nu, g, lu;
    bool in[NCH];
    unsigned at[NCH];  // unit within the row
    __device__ Lanes(int lane, int d)
        : nu((d + kCacheBlock - 1) / kCacheBlock * (kCacheBlock / unit_cols<FMT>())), g(lane / LG),
          lu(lane % LG)
    {
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            in[c] = lu + c * LG < nu;
            at[c] = (unsigned)min(lu + c * LG, nu - 1);
        }
    }
    __device__ int col(int c) const { return (lu + c * LG) * unit_cols<FMT>(); }
};

// Calls f(std::integral_constant<int, LG>, std::integral_constant<int, NCH>) with
// the fewest lanes that hold a row of d columns (up to 4096; beyond, of one of its
// column blocks).
template <int FMT, typename F> hipError_t dispatch_lanes(int64_t d, F &&f)
{
    typedef std::integral_constant<int, 64> L64;
    typedef std::integral_constant<int, 1> One;
    const int64_t nu = cache_blocks(d) * (kCacheBlock / unit_cols<FMT>());
    if (nu <= 16)
        return f(std::integral_constant<int, 16>{}, One{});
    if (nu <= 32)
        return f(std::integral_constant<int, 32>{}, One{});
    if (nu <= 64)
        return f(L64{}, One{});
    if constexpr (FMT == LRAR_CACHE_FP8) {
        if (nu > 128)
            return f(L64{}, std::integral_constant<int, 4>{});
    }
    return f(L64{}, std::integral_constant<int, 2>{});
}

// Encodes a unit of a row (zeros past its end): e4m3 blocks are two neighbouring
// lanes', e2m1 blocks one lane's.
template <int FMT>
__device__ __forceinline__ void encode_unit(const float (&x)[UnitRaw<FMT>::cols], UnitRaw<FMT> &w)
{
    constexpr int CW = unit_cols<FMT>();
    float top = 0.0f;
#pragma unroll
    for (int e = 0; e < CW; ++e)
        top = max_magnitude(top, x[e]);
    if constexpr (FMT == LRAR_CACHE_FP8)
        top = max_magnitude(top, dpp_move<kDppXor1>(top));
    w.e = scale_byte<FMT>(top);
    unsigned c[4];
#pragma unroll
    for (int h = 0; h < CW / 8; ++h) {
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            y[e] = x[8 * h + e];
        const typename Codes<FMT>::key_t k = encode<FMT>(y, w.e);
        if constexpr (FMT == LRAR_CACHE_FP8) {
            c[2 * h] = k.x;
            c[2 * h + 1] = k.y;
        } else {
            c[h] = k;
        }
    }
    w.c = u32x4_t{c[0], c[1], c[2], c[3]};
}

template <int FMT>
__device__ __forceinline__ void store_unit(uint8_t *codes, uint8_t *scales, unsigned at,
                                           const UnitRaw<FMT> &w)
{
    *reinterpret_cast<u32x4_t *>(codes + at * 16u) = w.c;
    scales[at * (unsigned)unit_cols<FMT>() / kCacheBlock] = (uint8_t)w.e;
}

// a and b, each summed over the two halves of the wave (or of each pair of rows
// of 16 lanes): the lower half receives a's sum, the upper half b's.  One gfx950
// lane swap and one addition.
__device__ __forceinline__ float halve32(float a, float b)
{
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}
__device__ __forceinline__ float halve16(float a, float b)
{
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}
constexpr int kDppRor8 = 0x128;  // row_ror:8, lane i + 8 within each 16
__device__ __forceinline__ float halve8(float a, float b, int lane)
{
    const bool up = (lane & 8) != 0;
    return (up ? b : a) + dpp_move<kDppRor8>(up ? a : b);
}

// Four values, each summed over every group of LG lanes: a lane receives the sum
// of value four_index<LG>(lane) over its own group.
template <int LG> __device__ __forceinline__ float four_sums(const float (&v)[4], int lane)
{
    float a, b, s;
    if constexpr (LG == 64) {
        a = halve32(v[0], v[2]);
        b = halve32(v[1], v[3]);
        s = halve16(a, b);
        s += dpp_move<kDppRor8>(s);
    } else if constexpr (LG == 32) {
        a = halve16(v[0], v[2]);
        b = halve16(v[1], v[3]);
        s = halve8(a, b, lane);
    } else {
        a = halve8(v[0], v[2], lane);
        b = halve8(v[1], v[3], lane);
        const bool up = (lane & 4) != 0;
        s = (up ? b : a) + __shfl_xor(up ? a : b, 4, kWaveSize);
    }
    if constexpr (LG != 16)
        s += __shfl_xor(s, 4, kWaveSize);
    s += dpp_move<kDppXor2>(s);
    return s + dpp_move<kDppXor1>(s);
}
// The lane of the group of `lane` that holds value u.
template <int LG> __device__ __forceinline__ int four_lane(int lane, int u)
{
    constexpr int hi = LG / 2, lo = LG / 4;
    return (lane & ~(LG - 1)) + (u & 2 ? hi : 0) + (u & 1 ? lo : 0);
}
template <int LG> __device__ __forceinline__ int four_index(int lane)
{
    constexpr int hi = LG / 2, lo = LG / 4;
    return (lane & hi ? 2 : 0) + (lane & lo ? 1 : 0);
}
// Value u of a lane's group, from the lane that holds it.
template <int LG> __device__ __forceinline__ float four_value(float s, int lane, int u)
{
    if constexpr (LG == 64)
        return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(s), four_lane<LG>(0, u)));
    else
        return __shfl(s, four_lane<LG>(lane, u), kWaveSize);
}

// Softmax over the S sources of the 64 / LG tokens of a wave, each by its own LG
// lanes: alpha[g * s_pad + i] from s (which may be alpha itself).  The caller
// orders the LDS accesses.
template <int LG>
__device__ __forceinline__ void group_softmax(const float *s, float *alpha, int s_pad, int S, int g,
                                              int lu)
{
    const float *row = s + g * s_pad;
    float *out = alpha + g * s_pad;
    float m = -INFINITY;
    for (int i = lu; i < S; i += LG)
        m = fmaxf(m, row[i]);
    m = group_max(m, LG);
    float z = 0.0f;
    for (int i = lu; i < S; i += LG) {
        const float e = expf(row[i] - m);
        out[i] = e;
        z += e;
    }
    const float inv = 1.0f / group_sum(z, LG);
    for (int i = lu; i < S; i += LG)
        out[i] *= inv;
}

// ---------------------------------------------------------------------------
// Keys and scores
// ---------------------------------------------------------------------------

// How a wave reads keys: slots of 8 elements, of a row of K (projected) or of the
// columns [d - r, d) of the cache's row (sliced: slots start at column `base` =
// (d - r) / 8 * 8, whose first `off` elements are not the key's).  `lps` lanes (a
// power of two, at most 64) read one source's key.
template <int FMT, typename T, bool SLICED> struct Keys {
    const T *__restrict__ K;
    const uint8_t *codes, *scales;
    int N, d, r, nb, base, off, nkv, lps;

    __device__ Keys(const void *K_, const uint8_t *codes_, const uint8_t *scales_, int N_, int d_,
                    int r_)
        : K(static_cast<const T *>(K_)), codes(codes_), scales(scales_), N(N_), d(d_), r(r_),
          nb((d_ + kCacheBlock - 1) / kCacheBlock), base(SLICED ? (d_ - r_) / 8 * 8 : 0),
          off(SLICED ? d_ - r_ - base : 0), nkv((r_ + off + 7) / 8), lps(1)
    {
        while (lps < nkv && lps < kWaveSize)
            lps <<= 1;
    }
    // First of the key's elements that slot v holds (below 0: not the key's).
    __device__ int first(int v) const { return v * 8 - off; }
    __device__ __forceinline__ void query(const float *__restrict__ q, int v, float (&x)[8]) const
    {
        const int j = first(v);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            x[e] = v < nkv && j + e >= 0 && j + e < r ? q[max(min(j + e, r - 1), 0)] : 0.0f;
    }
    struct Raw {
        typename Codes<FMT>::key_t c;
        unsigned e;
        Raw8<T> p;
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
            load8_raw(K + row * r, v * 8, r, w.p);
        }
    }
    // Its values, zeros where the slot's elements are not the key's.
    __device__ __forceinline__ void values(const Raw &w, int v, float (&x)[8]) const
    {
        if constexpr (SLICED) {
            decode<FMT>(w.c, block_scale(w.e), x);  // zeros past the row
            if (off != 0) {                         // uniform
                const int j = first(v);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x[e] = j + e >= 0 ? x[e] : 0.0f;
            }
        } else {
            widen8(w.p, x);
        }
    }
};

// Scores s_i = q . k_i / rho_i and (ri_out) 1 / rho_i of the sources [ib, ie) of
// TW consecutive tokens (tokens past N are read as token N-1 and not written),
// into s_out[t * s_pad + i].  A group of lps lanes reads one source's key, so
// 64 / lps sources are scored together, and KP such groups' loads of every
// token go out before the first is used.  (Slots of 16 bytes, so that fewer lanes
// read a sliced key, were slower: 11% at 33 sources, 16384 tokens, r = 64, e2m1,
// the arithmetic being the same and more lanes idle.)  The caller waits for the
// LDS writes.
template <int FMT, typename T, bool SLICED, int TW, int KP>
__device__ __forceinline__ void cache_scores(const Keys<FMT, T, SLICED> &k,
                                             const float *__restrict__ q, int ib, int ie,
                                             int n0, float eps, int lane, float *s_out,
                                             float *ri_out, int s_pad)
{
    typedef Keys<FMT, T, SLICED> Key;
    const int lps = k.lps, spi = kWaveSize / lps;
    const int isub = lane / lps, v = lane % lps;
    const float inv_r = 1.0f / (float)k.r;
    if (k.nkv <= lps) {
        float qv[8];
        k.query(q, v, qv);
        const bool vok = v < k.nkv;
        for (int i0 = ib; i0 < ie; i0 += KP * spi) {
            typename Key::Raw w[TW][KP];
#pragma unroll
            for (int t = 0; t < TW; ++t)
#pragma unroll
                for (int p = 0; p < KP; ++p)
                    if (p == 0 || i0 + p * spi < ie)  // wave-uniform
                        k.load(min(i0 + p * spi + isub, ie - 1), min(n0 + t, k.N - 1), v, w[t][p]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < TW; ++t)
#pragma unroll
                for (int p = 0; p < KP; ++p) {
                    if (p > 0 && i0 + p * spi >= ie)
                        break;
                    float x[8], ss = 0.0f, dot = 0.0f;
                    k.values(w[t][p], v, x);
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
                        const float ri = rsqrtf(ss * inv_r + eps);
                        s_out[t * s_pad + i] = dot * ri;
                        if (ri_out)
                            ri_out[t * s_pad + i] = ri;
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
                typename Key::Raw w;
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
                const float ri = rsqrtf(ss * inv_r + eps);
                s_out[t * s_pad + i] = dot * ri;
                if (ri_out)
                    ri_out[t * s_pad + i] = ri;
            }
        }
    }
}

}  // namespace lrar

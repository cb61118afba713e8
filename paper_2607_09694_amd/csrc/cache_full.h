// The dots that the full-rank backward needs over a source stack in 4 bits, on the
// matrix cores (the key of source i is its whole row x_i): 16 sources of a token at
// a time, q . x_i, |x_i|^2 (the diagonal of X X^T) and dH . x_i.
//
// e2m1 rows are operands as they lie in memory: a lane of the 16 x 16 x 128 product
// holds one block of 32 columns and its scale.  q and dH enter as sums of 8 e2m1
// digits -4 .. 3 (times 1/2), each block of 32 on one power of two, 2^-3 smaller
// from digit to digit: off by at most 2^-22.5 of the block's largest magnitude, about
// what the fp32 rounding of each product and sum is.  (dH is split anew for every
// token: the digits of a column are formed together, in one integer.)  Digits times
// codes are small integers, so the products are exact.
// Not taken: e4m3 rows against such digits, because the 8-bit product of the matrix
// cores aligns its terms to about 13 bits (measured 2e-4 of the sum of magnitudes);
// e4m3 rows decoded to bf16 against three bf16 terms, exact, but slower than vector
// code where the operands' on-chip memory leaves few waves (33 sources, 8192 tokens,
// d = 2048: 672 us against 514; d = 1024, 49 x 2048: 103 against 112); and the
// forward's scores, whose vector code reads the rows once (49 x 16384 x 1024, e2m1:
// 144 us against 176).
#pragma once

#include "cache_device.h"

namespace lrar {

typedef int i32x8_t __attribute__((ext_vector_type(8)));

constexpr int kDigits = 8;      // e2m1 digits of a value
constexpr int kTileRows = 16;   // sources of a tile

// Bytes of LDS for one row operand (q or dH): the digits and an exponent of every
// block, the row padded to whole steps of the product.
constexpr int operand_bytes(int d) { return (d + 127) / 128 * 4 * (kDigits * 16 + 4); }

// Row x [d] (fp32 or storage T) as an operand in LDS, by `threads` threads (a
// multiple of 16).  The caller puts barriers around it.
template <typename T>
__device__ __forceinline__ void make_operand(const T *__restrict__ x, int d, uint8_t *__restrict__ lds,
                                             int thread, int threads)
{
    const int nb = (d + 127) / 128 * 4;
    int *scale = reinterpret_cast<int *>(lds + nb * kDigits * 16);
    // Two neighbouring columns a thread, 16 threads a block.
    for (int k = thread; k < nb * 16; k += threads) {
        const int b = k / 16, col = 2 * k;
        float y[2];
#pragma unroll
        for (int e = 0; e < 2; ++e)
            y[e] = col + e < d ? load_elem(x + col + e) : 0.0f;
        float top = max_magnitude(max_magnitude(0.0f, y[0]), y[1]);
        top = max_magnitude(top, dpp_move<kDppXor1>(top));
        top = max_magnitude(top, dpp_move<kDppXor2>(top));
        top = max_magnitude(top, dpp_move<kDppHalfMirror>(top));
        top = max_magnitude(top, dpp_move<kDppMirror>(top));
        // The smallest e >= 22 with top <= 1.5 * 2^(e - 127): every digit has a scale
        // byte of its own.  (255, above 1.5 * 2^127, reads as NaN, as infinities do.)
        const unsigned u = __float_as_uint(top);
        const int e2 = max((int)(u >> 23) + ((u & 0x7fffffu) > 0x400000u ? 1 : 0), 22);
        const bool bad = u >= 0x7f800000u;
        if (k % 16 == 0)
            scale[b] = bad ? 255 : e2;
        unsigned w[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            // In units of the last digit, |n| <= 3 * 8^7; plus 4 in every digit,
            // the octal digits are 0 .. 7.
            const int n = (int)rintf(ldexpf(bad ? 0.0f : y[e], 128 + 21 - e2));
            unsigned v = (unsigned)(n + 0x924924);
            v = (v & 0xfffu) | (v & 0xfff000u) << 4;  // a digit every 4 bits
            v = (v & 0x003f003fu) | (v & 0x0fc00fc0u) << 2;
            v = (v & 0x07070707u) | (v & 0x38383838u) << 1;
            // Digit - 4 as sign and magnitude: 4 .. 7 are 0 .. 3, and 0 .. 3 the codes 12 .. 9.
            const unsigned m = v & 0x33333333u, neg = (~v >> 2 & 0x11111111u) * 15u;
            w[e] = (m & ~neg) | ((0xccccccccu & neg) - (m & neg));
        }
        // Digit p of both columns in a byte, the largest digit first.
        const unsigned even = (w[0] & 0x0f0f0f0fu) | (w[1] & 0x0f0f0f0fu) << 4;
        const unsigned odd = (w[0] >> 4 & 0x0f0f0f0fu) | (w[1] & 0xf0f0f0f0u);
#pragma unroll
        for (int p = 0; p < kDigits; ++p)
            lds[(b * kDigits + p) * 16 + k % 16] =
                (uint8_t)(((7 - p) % 2 ? odd : even) >> 8 * ((7 - p) / 2));
    }
}

// LDS of a wave for one tile: 16 rows of 512 bytes of codes (16 bytes of padding
// after each: no bank conflict) and 32 scale bytes each (and 4).
constexpr int kTileRow = 512 + 16, kTileScales = 32 + 4;
constexpr int kTileBytes = kTileRows * (kTileRow + kTileScales);
constexpr int kTileUnits = 32;  // blocks of a row in a tile
// Chunks of a row of d columns.
constexpr int tile_chunks(int d) { return (d + kTileUnits * kCacheBlock - 1) / (kTileUnits * kCacheBlock); }

// The dots of the sources [ib, ie) of the token whose rows are `row0` rows into
// each plane, chunk by chunk of its columns: part[(3 c + 0, 1, 2) stride + i] takes
// q . x_i, |x_i|^2 and dH . x_i over chunk c.  The (tile of 16 sources, chunk) pairs
// are dealt to `waves` waves, this one being `wave`.  ql, dl: operands of q and dH;
// tile: the wave's kTileBytes.  The rows come through LDS, the next pair's loads in
// flight over this one's products: read straight into the operands' layout, a load
// touches 16 planes, and the backward took 77 us instead of 68 (49 x 2048 x 1024).
__device__ __forceinline__ void tile_dots(const uint8_t *codes, const uint8_t *scales, size_t row0,
                                          size_t plane,
                                          int ib, int ie, int d, const uint8_t *__restrict__ ql,
                                          const uint8_t *__restrict__ dl, uint8_t *tile, int wave,
                                          int waves, int lane, float *part, int stride)
{
    const int c = lane % 16, gr = lane / 16;
    const int nu = (d + kCacheBlock - 1) / kCacheBlock;
    const int chunks = tile_chunks(d), jobs = (ie - ib + kTileRows - 1) / kTileRows * chunks;
    uint8_t *tscale = tile + kTileRows * kTileRow;
    UnitRaw<LRAR_CACHE_FP4> w[kTileRows / 2];
    auto load = [&](int job) {  // two rows an access
        const int i0 = ib + job / chunks * kTileRows;
        const unsigned un = (unsigned)min(job % chunks * kTileUnits + lane % kTileUnits, nu - 1);
#pragma unroll
        for (int k = 0; k < kTileRows / 2; ++k) {
            const size_t row = (size_t)min(i0 + 2 * k + lane / kTileUnits, ie - 1) * plane + row0;
            const size_t at = row * nu + un;
            w[k].c = *reinterpret_cast<const u32x4_t *>(codes + at * 16);
            w[k].e = scales[at];
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    if (wave < jobs)
        load(wave);
    for (int job = wave; job < jobs; job += waves) {
        const int i0 = ib + job / chunks * kTileRows, chunk = job % chunks, u0 = chunk * kTileUnits;
        f32x4_t dq = {0, 0, 0, 0}, dx = {0, 0, 0, 0};
        wave_lds_sync();  // the pair before this one has been read
#pragma unroll
        for (int k = 0; k < kTileRows / 2; ++k) {
            const int r = 2 * k + lane / kTileUnits;
            const bool in = u0 + lane % kTileUnits < nu;  // units past the row are zeros
            *reinterpret_cast<u32x4_t *>(tile + r * kTileRow + lane % kTileUnits * 16) =
                in ? w[k].c : u32x4_t{0u, 0u, 0u, 0u};
            tscale[r * kTileScales + lane % kTileUnits] = (uint8_t)(in ? w[k].e : 127u);
        }
        if (job + waves < jobs)
            load(job + waves);
        wave_lds_sync();
        const int steps = (min(kTileUnits, nu - u0) + 3) / 4;  // 4 units of every row a step
        const int nbp = (nu + 3) / 4 * 4;
        // Columns 0 .. 7 of the product take q's digits, 8 .. 15 dH's.
        const uint8_t *bl = c >= kDigits ? dl : ql;
        const int *bs = reinterpret_cast<const int *>(bl + nbp * kDigits * 16);
        for (int s = 0; s < steps; ++s) {
            const u32x4_t a = *reinterpret_cast<const u32x4_t *>(tile + c * kTileRow + (4 * s + gr) * 16);
            const int ex = tscale[c * kTileScales + 4 * s + gr];
            const int b = u0 + 4 * s + gr;
            const u32x4_t qd = *reinterpret_cast<const u32x4_t *>(bl + (b * kDigits + c % kDigits) * 16);
            const int qe = bs[b];
            i32x8_t x = {0, 0, 0, 0, 0, 0, 0, 0}, y = x;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                x[k] = (int)a[k];
                y[k] = (int)qd[k];
            }
            dq = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                x, y, dq, 4, 4, 0, ex, 0, qe == 255 ? 255 : qe - 3 * (c % kDigits));
            dx = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, x, dx, 4, 4, 0, ex, 0, ex);
        }
        // Row 4 gr + k, column c of a product is element k of the lane.
        float *out = part + 3 * chunk * stride + i0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = 4 * gr + k;
            // Sums over aligned groups of 8 columns: q's in the first, dH's in the second.
            const float v = group_sum(dq[k], 8);
            if (i0 + i < ie) {
                if (c == 0)
                    out[i] = v;
                if (c == i)
                    out[stride + i] = dx[k];
                if (c == 8)
                    out[2 * stride + i] = v;
            }
        }
    }
}

// Value `which` (0, 1, 2) of source i over all chunks, in their order.
__device__ __forceinline__ float chunk_sum(const float *part, int stride, int chunks, int which, int i)
{
    float v = part[which * stride + i];
    for (int c = 1; c < chunks; ++c)
        v += part[(3 * c + which) * stride + i];
    return v;
}

}  // namespace lrar

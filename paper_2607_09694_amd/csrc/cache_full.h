// The dots that the full-rank backward needs over a source stack in 4 bits, on the
// matrix cores (the key of source i is its whole row x_i): 16 sources of a token at
// a time, q . x_i, |x_i|^2 (the diagonal of X X^T) and dH . x_i.
//
// Everything is exact before fp32 sums: an e2m1 value with its block's power of two is
// a bf16 number (checked over every code and scale byte, subnormal ones included), and
// q and fp32 dH enter as three bf16 terms, the leading 8, the next 8 and the last 8 bits
// of every element on its own (bf16 dH as it is).  No element costs another its bits,
// whatever range a block has.
// Not taken: digits of q and dH on one power of two a block, which need no decoding but
// lose what is 2^-24 of a block's largest element; e4m3 rows against the same bf16 terms,
// slower than vector code where the operands' on-chip memory leaves few waves (33
// sources, 8192 tokens, d = 2048: 672 us against 514; d = 1024, 49 x 2048: 103 against
// 112); the 8-bit product of the matrix cores, which aligns its terms to about 13 bits
// (measured 2e-4 of the sum of magnitudes); and the forward's scores, whose vector code
// reads the rows once (49 x 16384 x 1024, e2m1: 144 us against 176).  Rows of more than
// 1024 columns take vector code too.  Matrix cores / vector code, the whole backward, e2m1:
// 49 x 2048 x 1024 68.7 / 90.3 us, 33 x 4096 x 1000 120 / 142, 16 x 2048 x 1024 41.3 / 44.8,
// 8 x 4096 x 1024 67.4 / 66.4, 1 x 4096 x 1024 61.0 / 58.6, 49 x 4096 x 512 80 / 122, 4 x
// 4096 x 128 35.5 / 46.4; 33 x 4096 x 1088 260 / 189, 49 x 2048 x 1536 157 / 141, 33 x
// 8192 x 2048 570 / 427, 8 x 4096 x 2048 156 / 98 (there the tile's registers leave one
// wave a SIMD, and the operands in on-chip memory few workgroups).
#pragma once

#include "cache_device.h"

namespace lrar {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

constexpr int kTileRows = 16;   // sources of a tile

// bf16 terms of an element of fp32 or storage T.
template <typename T> constexpr int row_terms() { return sizeof(T) == 2 ? 1 : 3; }
// Bytes of LDS for one term of a row operand (q or dH), the row padded to whole steps of
// 128 columns.  (16 bytes more: the terms that a load reads together lie in other banks.)
constexpr int term_bytes(int d) { return (d + 127) / 128 * 256 + 16; }

// Row x [d] (fp32 or storage T) as row_terms<T>() rows of bf16 in LDS, zeros past d, by
// `threads` threads.  The terms are cut off, not rounded, so that none is larger than the
// element; an infinity or NaN is its first term.  The caller puts barriers around it.
template <typename T>
__device__ __forceinline__ void make_operand(const T *__restrict__ x, int d, uint8_t *__restrict__ lds,
                                             int thread, int threads)
{
    const int pairs = (d + 127) / 128 * 64, tb = term_bytes(d);
    for (int k = thread; k < pairs; k += threads) {
        float y[2];
#pragma unroll
        for (int e = 0; e < 2; ++e)
            y[e] = 2 * k + e < d ? load_elem(x + 2 * k + e) : 0.0f;
#pragma unroll
        for (int t = 0; t < row_terms<T>(); ++t) {
            unsigned w[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const unsigned u = __float_as_uint(y[e]);
                // (A NaN stays one without its last 16 bits.)
                w[e] = (u & 0x7fffffffu) > 0x7f800000u ? 0x7fc00000u : u & 0xffff0000u;
                const bool last = (u & 0x7f800000u) == 0x7f800000u;
                y[e] = last ? 0.0f : y[e] - __uint_as_float(w[e]);
            }
            *reinterpret_cast<unsigned *>(lds + t * tb + 4 * k) = w[0] >> 16 | w[1];
        }
    }
}

// 8 e2m1 codes of a word as bf16, times the block's scale.
__device__ __forceinline__ bf16x8_t decode_bf16(unsigned w, float sc)
{
    const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 0);
    const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 1);
    const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 2);
    const bf16x2_t e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 3);
    return bf16x8_t{a.x, a.y, b.x, b.y, c.x, c.y, e.x, e.y};
}

// LDS of a wave for one tile: 16 rows of 512 bytes of codes (16 bytes of padding
// after each: no bank conflict) and 32 scale bytes each (and 4).
constexpr int kTileRow = 512 + 16, kTileScales = 32 + 4;
constexpr int kTileBytes = kTileRows * (kTileRow + kTileScales);
constexpr int kTileUnits = 32;  // blocks of a row in a tile: the whole row

// The dots of the sources [ib, ie) of the token whose rows, of up to 1024 columns, are
// `row0` rows into each plane: part[i], part[stride + i] and part[2 stride + i] take
// q . x_i, |x_i|^2 and dH . x_i.  The tiles of 16 sources are dealt to `waves` waves,
// this one being `wave`.  op: the terms of q, then those of dH; tile: the wave's
// kTileBytes.  The rows come through LDS, the next tile's loads in flight over this
// one's products: read straight into the operands' layout, a load touches 16 planes, and
// the backward took 77 us instead of 68 (49 x 2048 x 1024, with rows that needed no
// decoding; with it 68.7).
template <typename T>
__device__ __forceinline__ void tile_dots(const uint8_t *codes, const uint8_t *scales, size_t row0,
                                          size_t plane, int ib, int ie, int d,
                                          const uint8_t *__restrict__ op, uint8_t *tile, int wave,
                                          int waves, int lane, float *part, int stride)
{
    const int c = lane % 16, gr = lane / 16;
    const int nu = (d + kCacheBlock - 1) / kCacheBlock;
    const int tiles = (ie - ib + kTileRows - 1) / kTileRows;
    uint8_t *tscale = tile + kTileRows * kTileRow;
    UnitRaw<LRAR_CACHE_FP4> w[kTileRows / 2];
    const unsigned un = (unsigned)min(lane % kTileUnits, nu - 1);
    auto load = [&](int k0) {  // two rows an access
        const int i0 = ib + k0 * kTileRows;
#pragma unroll
        for (int k = 0; k < kTileRows / 2; ++k) {
            const size_t row = (size_t)min(i0 + 2 * k + lane / kTileUnits, ie - 1) * plane + row0;
            const size_t at = row * nu + un;
            w[k].c = *reinterpret_cast<const u32x4_t *>(codes + at * 16);
            w[k].e = scales[at];
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    if (wave < tiles)
        load(wave);
    for (int k0 = wave; k0 < tiles; k0 += waves) {
        const int i0 = ib + k0 * kTileRows;
        f32x4_t dq = {0, 0, 0, 0}, dx = {0, 0, 0, 0};
        wave_lds_sync();  // the tile before this one has been read
#pragma unroll
        for (int k = 0; k < kTileRows / 2; ++k) {
            const int r = 2 * k + lane / kTileUnits;
            const bool in = lane % kTileUnits < nu;  // units past the row are zeros
            *reinterpret_cast<u32x4_t *>(tile + r * kTileRow + lane % kTileUnits * 16) =
                in ? w[k].c : u32x4_t{0u, 0u, 0u, 0u};
            tscale[r * kTileScales + lane % kTileUnits] = (uint8_t)(in ? w[k].e : 127u);
        }
        if (k0 + waves < tiles)
            load(k0 + waves);
        wave_lds_sync();
        const int steps = (nu + 3) / 4;  // 4 units of every row a step
        // Columns 0, 1, 2 of the product take q's terms, 8 on dH's; the others repeat q's
        // first and are not used.
        const int qt = row_terms<float>(), dt = row_terms<T>();
        const bool used = c % 8 < (c < 8 ? qt : dt);
        const uint8_t *bl = op + (used ? c % 8 + (c < 8 ? 0 : qt) : 0) * term_bytes(d);
        for (int s = 0; s < steps; ++s) {
            // Lane group gr has block 4 s + gr, 8 of its columns a product.
            const u32x4_t a = *reinterpret_cast<const u32x4_t *>(tile + c * kTileRow + (4 * s + gr) * 16);
            const float sc = block_scale(tscale[c * kTileScales + 4 * s + gr]);
            const uint8_t *b = bl + (4 * s + gr) * (2 * kCacheBlock);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const bf16x8_t x = decode_bf16(a[k], sc);
                const bf16x8_t y = *reinterpret_cast<const bf16x8_t *>(b + 16 * k);
                dq = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, dq, 0, 0, 0);
                dx = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, x, dx, 0, 0, 0);
            }
        }
        // Row 4 gr + k, column c of a product is element k of the lane.
        float *out = part + i0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = 4 * gr + k;
            // Sums over aligned groups of 8 columns: q's in the first, dH's in the second.
            const float v = group_sum(used ? dq[k] : 0.0f, 8);
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

}  // namespace lrar

// Backward of the depth routing over a source stack in 8 or 4 bits: kernels and
// launch template, instantiated per format.  Internal to the library.
//
// With x_i the stored values and dH the upstream gradient of a token,
//     g_i = dH . x_i,  ds_i = alpha_i (g_i - sum_l alpha_l g_l),
//     dV_i = alpha_i dH (+ the key gradient in sliced and full-rank keys'
//     columns),  dk_i = (ds_i / rho_i)(q - k_i s_i / (rho_i^2 r)),
//     dq = sum ds_i k_i / rho_i,
// the weights recomputed from the keys.  The stack is read once (full rank:
// twice) in the units of a lane; dV, which does not depend on it beyond the key
// columns, is written from dH alone, whole lines a store.  Bound by HBM: 64 sources,
// 16384 tokens, d = 2048, e4m3, projected r = 32 takes 1090 us: 392 for the reads (5.8
// TB/s), 664 for the 4.29 GB of dV (6.5 TB/s), 5 for dq.  The deferred form (49
// sources, 16384 tokens, d = 1024, r = 16) reads at 6.2 TB/s, 145 us.
#pragma once

#include "cache_device.h"
#include "cache_full.h"

namespace lrar {

// What the backward of one site writes per source.
enum CacheGrad { kGradWrite, kGradAdd, kGradCoef };

// dH in the units of a lane.
template <int FMT, typename T, int LG, int NCH>
__device__ __forceinline__ void load_dh(const T *__restrict__ row, const Lanes<FMT, LG, NCH> &ln, int d,
                                        float (&dh)[NCH][UnitRaw<FMT>::cols])
{
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int h = 0; h < unit_cols<FMT>() / 8; ++h) {
            float y[8];
            load8(row, ln.col(c) + 8 * h, d, y);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                dh[c][8 * h + e] = y[e];
        }
}

// A lane's share of dH . x.
template <int FMT>
__device__ __forceinline__ float dot_unit(const UnitRaw<FMT> &w, const float (&dh)[UnitRaw<FMT>::cols],
                                          float p)
{
#pragma unroll
    for (int h = 0; h < unit_cols<FMT>() / 16; ++h) {
        float x[16];
        unit_values<FMT>(w, h, x);
#pragma unroll
        for (int e = 0; e < 16; ++e)
            p = fmaf(dh[16 * h + e], x[e], p);
    }
    return p;
}

// The key gradients of sources [ib, ie) of one token, dq included: lanes over
// (source, key slot).  s, ri = 1 / rho, ds and alpha are the token's.
template <int FMT, typename T, bool SLICED, CacheGrad OUT>
__device__ __forceinline__ void key_grads(const Keys<FMT, T, SLICED> &keys, const T *__restrict__ dhrow,
                                          T *__restrict__ dV, T *__restrict__ dK, const float (&qk)[8],
                                          int ib, int ie, int n, int lane, const float *s,
                                          const float *ri, const float *ds, const float *alpha,
                                          float (&dq_acc)[8])
{
    typedef Keys<FMT, T, SLICED> Key;
    constexpr int KP = 2;
    const int lps = keys.lps, spi = kWaveSize / lps;
    const int isub = lane / lps, v = lane % lps;
    const float inv_r = 1.0f / (float)keys.r;
    float dhk[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        dhk[e] = 0.0f;
    if (SLICED && OUT != kGradCoef && v < keys.nkv)
        load8(dhrow, keys.base + v * 8, keys.d, dhk);
    for (int i0 = ib; i0 < ie; i0 += KP * spi) {
        typename Key::Raw w[KP];
#pragma unroll
        for (int p = 0; p < KP; ++p)
            if (p == 0 || i0 + p * spi < ie)  // wave-uniform
                keys.load(min(i0 + p * spi + isub, ie - 1), n, v, w[p]);
#pragma unroll
        for (int p = 0; p < KP; ++p) {
            const int i = i0 + p * spi + isub;
            if (v >= keys.nkv || i >= ie)
                continue;
            float x[8], y[8];
            keys.values(w[p], v, x);
            const size_t row = (size_t)i * keys.N + n;
            const float rv = ri[i], dsi = ds[i];
            const float cq = dsi * rv;           // ds_i / rho_i
            const float ck = cq * s[i] * inv_r;  // ds_i s_i / (rho_i r)
            const float a = SLICED ? alpha[i] : 0.0f;
            const int j = keys.first(v);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float kb = x[e] * rv;
                dq_acc[e] = fmaf(dsi, kb, dq_acc[e]);
                y[e] = a * dhk[e];
                if (!SLICED || j + e >= 0)
                    y[e] += fmaf(cq, qk[e], -ck * kb);
            }
            if constexpr (OUT != kGradCoef) {
                T *orow = SLICED ? dV + row * keys.d : dK + row * keys.r;
                const int ocol = SLICED ? keys.base + v * 8 : v * 8;
                const int width = SLICED ? keys.d : keys.r;
                if constexpr (OUT == kGradAdd) {
                    float o[8];
                    load8(orow, ocol, width, o);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        y[e] += o[e];
                }
                store8<T, false>(orow, ocol, width, y);
            }
        }
    }
}

// Chunks of 64 lanes of 16 bytes in a row of up to `cols` columns.
template <typename T> constexpr int value_chunks(int cols)
{
    return (cols * (int)sizeof(T) + 1023) / 1024;
}

// dV_i = alpha_i dH of sources [ib, ie) of TT adjacent tokens, columns [0, wend),
// in lanes of 16 bytes, whole lines a wave; alpha of source i and token t at
// alpha[i * si + t * st].
template <typename T, int NO, CacheGrad OUT, int TT>
__device__ __forceinline__ void value_grads(const T *__restrict__ dH, T *__restrict__ dV, int ib,
                                            int ie, int n0, int N, int d, int wend, int lane,
                                            const float *alpha, size_t si, int st)
{
    constexpr int VO = 16 / sizeof(T);
    u32x4_t dh[TT][NO];
    const int nt = min(TT, N - n0);  // wave-uniform
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int c = 0; c < NO; ++c)
            dh[t][c] = load16_elems(dH + (size_t)(n0 + min(t, nt - 1)) * d, (c * kWaveSize + lane) * VO, d);
    for (int i = ib; i < ie; ++i) {
        T *plane = dV + (size_t)i * N * d;
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            if (t >= nt)
                break;
            const float a = alpha[i * si + t * st];
            T *orow = plane + (size_t)(n0 + t) * d;
#pragma unroll
            for (int c = 0; c < NO; ++c) {
                const int col = (c * kWaveSize + lane) * VO;
                float y[VO];
                if constexpr (VO == 8)
                    widen(dh[t][c], y);
                else
                    widen(__builtin_bit_cast(f32x4_t, dh[t][c]), y);
#pragma unroll
                for (int e = 0; e < VO; ++e)
                    y[e] *= a;
                if constexpr (OUT == kGradAdd) {
                    const u32x4_t w = load16_elems(orow, col, wend);
                    if constexpr (VO == 8)
                        add_stored(y, w);
                    else
                        add_stored(y, __builtin_bit_cast(f32x4_t, w));
                }
                store16_elems<T, kBwdNtStore>(orow, col, wend,
                                              __builtin_bit_cast(u32x4_t, Narrow<T, VO>::run(y)));
            }
        }
    }
}

// The workgroup's dq: over the source groups of each wave (lanes of the same
// key slot), then over the waves in order, into partial[bx][r].
template <int W, int FMT, typename T, bool SLICED>
__device__ __forceinline__ void store_dq(const Keys<FMT, T, SLICED> &keys, float (&dq_acc)[8],
                                         float *stage, int r_pad, float *__restrict__ partial, int bx,
                                         int wave, int lane)
{
    const int v = lane % keys.lps, r = keys.r;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        for (int m = keys.lps; m < kWaveSize; m <<= 1)
            dq_acc[e] += __shfl_xor(dq_acc[e], m, kWaveSize);
    float *my = stage + wave * r_pad;
    if (lane / keys.lps == 0 && v < keys.nkv) {
        const int j = keys.first(v);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (j + e >= 0 && j + e < r)
                my[j + e] = dq_acc[e];
    }
    lds_barrier();
    for (int j = threadIdx.x; j < r; j += W * kWaveSize) {
        float sum = 0.0f;
        for (int w = 0; w < W; ++w)
            sum += stage[w * r_pad + j];
        partial[(size_t)bx * r + j] = sum;
    }
}

// The coefficients of P tokens from n0 on and sources [ib, ie), by `nthreads`
// threads, runs of adjacent tokens together: coef[i][0..2][n] = alpha, ds / rho,
// ds s / (rho r), or (gradient rows) coef[i][n] = alpha.  The token rows in LDS are
// s_pad apart (odd: no bank conflict).
template <CacheGrad OUT>
__device__ __forceinline__ void store_coef(float *__restrict__ coef, const float *s, const float *ri,
                                           const float *ds, const float *alpha, int s_pad, int P,
                                           int n0, int ib, int ie, int N, float inv_r, int thread,
                                           int nthreads)
{
    const int count = min(P, N - n0);
    for (int k = thread; k < P * (ie - ib); k += nthreads) {
        const int t = k % P, i = ib + k / P;
        if (t >= count)
            continue;
        const int at = t * s_pad + i;
        if constexpr (OUT != kGradCoef) {
            coef[(size_t)i * N + n0 + t] = alpha[at];
            continue;
        }
        const float cq = ds[at] * ri[at];
        float *c = coef + (size_t)i * 3 * N + n0 + t;
        c[0] = alpha[at];
        c[N] = cq;
        c[2 * (size_t)N] = cq * s[at] * inv_r;
    }
}

// Projected / sliced keys.  A wave owns the P = G TW adjacent tokens of its G
// groups of lanes; each trip forms the dots of four (source, token) pairs of
// every group.  It writes the key gradients and the dq partials, and into coef the
// coefficients or (gradient rows) the weights [S][N], from which
// cache_value_grads writes the rest of dV: reads and writes of HBM in turn, not
// mixed (in one kernel the size above took 1380 us).
template <int FMT, typename T, int LG, int NCH, bool SLICED, CacheGrad OUT, int TW>
__global__ void __launch_bounds__(kBlock)
cache_bwd_lr(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales,
             const void *__restrict__ K, const float *__restrict__ q, const T *__restrict__ dH,
             T *__restrict__ dV, T *__restrict__ dK, float *__restrict__ coef,
             float *__restrict__ partial, int S, int N, int d, int r, float eps, int s_pad,
             int r_pad)
{
    constexpr int G = kWaveSize / LG, CW = unit_cols<FMT>(), P = G * TW, SB = 4 / TW;
    constexpr int per = kCacheBlock / CW;  // units a block
    extern __shared__ float lds[];
    const int lane = threadIdx.x & (kWaveSize - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWaveSize);
    const int array = kWaves * P * s_pad;  // one of the four: [tokens of the workgroup][s_pad]
    float *s = lds + wave * P * s_pad, *ri = s + array, *g = ri + array, *alpha = g + array;
    float *stage = lds + 4 * array;        // [kWaves][r_pad]
    const int bx = xcd_block().x;
    const int n0 = (bx * kWaves + wave) * P;
    const Keys<FMT, T, SLICED> keys(K, codes, scales, N, d, r);
    const Lanes<FMT, LG, NCH> ln(lane, d);
    float qk[8], dq_acc[8];
    keys.query(q, lane % keys.lps, qk);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        dq_acc[e] = 0.0f;

    if (n0 < N) {  // wave-uniform; the barriers are after it
        float dh[TW][NCH][CW];
        unsigned at[TW][NCH];
#pragma unroll
        for (int t = 0; t < TW; ++t) {
            const int n = min(n0 + t * G + ln.g, N - 1);
            load_dh<FMT, T, LG, NCH>(dH + (size_t)n * d, ln, d, dh[t]);
#pragma unroll
            for (int c = 0; c < NCH; ++c)
                at[t][c] = (unsigned)((n - n0) * ln.nu) + ln.at[c];
        }
        cache_scores<FMT, T, SLICED, P, P <= 2 ? 4 : P <= 4 ? 2 : 1>(keys, q, 0, S, n0, eps, lane, s,
                                                                    ri, s_pad);
        wave_lds_sync();
#pragma unroll
        for (int t = 0; t < TW; ++t)
            group_softmax<LG>(s + t * G * s_pad, alpha + t * G * s_pad, s_pad, S, ln.g, ln.lu);

        // The dots of dH with the stored rows.
        const size_t first = (size_t)n0 * ln.nu, plane = (size_t)N * ln.nu;
        for (int i0 = 0; i0 < S; i0 += SB) {
            UnitRaw<FMT> w[SB][TW][NCH];
#pragma unroll
            for (int u = 0; u < SB; ++u) {
                const size_t b = min(i0 + u, S - 1) * plane + first;
#pragma unroll
                for (int t = 0; t < TW; ++t)
#pragma unroll
                    for (int c = 0; c < NCH; ++c)
                        load_unit<FMT>(codes + b * 16, scales + b / per, at[t][c], w[u][t][c]);
            }
            __builtin_amdgcn_sched_barrier(0);
            float p[4];
#pragma unroll
            for (int u = 0; u < SB; ++u)
#pragma unroll
                for (int t = 0; t < TW; ++t) {
                    p[u * TW + t] = 0.0f;
#pragma unroll
                    for (int c = 0; c < NCH; ++c)
                        p[u * TW + t] = dot_unit<FMT>(w[u][t][c], dh[t][c], p[u * TW + t]);
                }
            const float sum = four_sums<LG>(p, lane);
            const int k = four_index<LG>(lane), i = i0 + k / TW;
            if (lane % (LG / 4) == 0 && i < S)
                g[(k % TW * G + ln.g) * s_pad + i] = sum;
            __builtin_amdgcn_sched_barrier(0);
        }
        wave_lds_sync();
#pragma unroll
        for (int t = 0; t < TW; ++t) {
            float *gr = g + (t * G + ln.g) * s_pad;
            const float *ar = alpha + (t * G + ln.g) * s_pad;
            float gb = 0.0f;
            for (int i = ln.lu; i < S; i += LG)
                gb = fmaf(ar[i], gr[i], gb);
            gb = group_sum(gb, LG);
            for (int i = ln.lu; i < S; i += LG)
                gr[i] = ar[i] * (gr[i] - gb);  // g now holds ds
        }
        wave_lds_sync();
        for (int t = 0; t < P && n0 + t < N; ++t) {
            const int o = t * s_pad;
            key_grads<FMT, T, SLICED, OUT>(keys, dH + (size_t)(n0 + t) * d, dV, dK, qk, 0, S, n0 + t,
                                           lane, s + o, ri + o, g + o, alpha + o, dq_acc);
        }
    }
    store_dq<kWaves>(keys, dq_acc, stage, r_pad, partial, bx, wave, lane);  // (a barrier: LDS is written)
    store_coef<OUT>(coef, lds, lds + array, lds + 2 * array, lds + 3 * array, s_pad, kWaves * P,
                    bx * kWaves * P, 0, S, N, 1.0f / (float)r, threadIdx.x, kBlock);
}

// The value rows dV_i = alpha_i dH before column wend: a wave holds TT tokens' dH
// and walks the planes, TT adjacent rows a plane (4.29 GB of d = 2048: one token 790
// us, 4 760, 8 664).
template <typename T, int NO, CacheGrad OUT, int TT>
__global__ void __launch_bounds__(kBlock)
cache_value_grads(const T *__restrict__ dH, const float *__restrict__ alpha, T *__restrict__ dV, int S,
                  int N, int d, int wend, int per)
{
    const int lane = threadIdx.x & (kWaveSize - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWaveSize);
    const BlockXY bk = xcd_block();
    const int n0 = (bk.x * kWaves + wave) * TT;
    if (n0 >= N)
        return;
    value_grads<T, NO, OUT, TT>(dH, dV, bk.y * per, min(S, (bk.y + 1) * per), n0, N, d, wend, lane,
                                alpha + n0, (size_t)N, 1);
}

// The same for few tokens: one token a workgroup, its sources cut into a range a
// wave, whose groups take every G-th one, U of them in flight a lane; scores and
// dots of all of them meet in LDS.
template <int FMT, typename T, int LG, int NCH, bool SLICED, CacheGrad OUT, int W>
__global__ void __launch_bounds__(W * kWaveSize)
cache_bwd_lr_wg(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales,
                const void *__restrict__ K, const float *__restrict__ q, const T *__restrict__ dH,
                T *__restrict__ dV, T *__restrict__ dK, float *__restrict__ coef,
                float *__restrict__ partial, int S, int N, int d, int r, float eps, int s_pad,
                int r_pad)
{
    constexpr int G = kWaveSize / LG, CW = unit_cols<FMT>();
    constexpr int per_block = kCacheBlock / CW, U = NCH >= 4 ? 4 : 8;
    extern __shared__ float lds[];
    const int lane = threadIdx.x & (kWaveSize - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWaveSize);
    float *s = lds, *ri = s + s_pad, *g = ri + s_pad, *ds = g + s_pad;
    float *alpha = ds + s_pad + wave * s_pad;  // a wave's own
    float *stage = lds + (4 + W) * s_pad;
    const int n = xcd_block().x;
    const int per = (S + W - 1) / W;
    const int ib = min(S, wave * per), ie = min(S, ib + per);
    const Keys<FMT, T, SLICED> keys(K, codes, scales, N, d, r);
    const Lanes<FMT, LG, NCH> ln(lane, d);
    const T *dhrow = dH + (size_t)n * d;
    float qk[8], dq_acc[8];
    keys.query(q, lane % keys.lps, qk);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        dq_acc[e] = 0.0f;
    if (ib < ie) {  // wave-uniform
        const size_t first = (size_t)n * ln.nu, plane = (size_t)N * ln.nu;
        UnitRaw<FMT> w[U][NCH];
        auto load = [&](int i0) {
#pragma unroll
            for (int h = 0; h < U; h += 4)
                if (h == 0 || i0 + h * G < ie)  // wave-uniform
#pragma unroll
                    for (int u = h; u < h + 4; ++u) {
                        const size_t b = min(i0 + u * G + ln.g, ie - 1) * plane + first;
#pragma unroll
                        for (int c = 0; c < NCH; ++c)
                            load_unit<FMT>(codes + b * 16, scales + b / per_block, ln.at[c], w[u][c]);
                    }
        };
        float dh[NCH][CW];
        load_dh<FMT, T, LG, NCH>(dhrow, ln, d, dh);
        load(ib);
        cache_scores<FMT, T, SLICED, 1, 4>(keys, q, ib, ie, n, eps, lane, s, ri, s_pad);
        for (int i0 = ib; i0 < ie; i0 += U * G) {
            if (i0 > ib)
                load(i0);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int h = 0; h < U; h += 4) {
                if (h > 0 && i0 + h * G >= ie)
                    break;
                float p[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    p[u] = 0.0f;
#pragma unroll
                    for (int c = 0; c < NCH; ++c)
                        p[u] = dot_unit<FMT>(w[h + u][c], dh[c], p[u]);
                }
                const float sum = four_sums<LG>(p, lane);
                const int i = i0 + (h + four_index<LG>(lane)) * G + ln.g;
                if (lane % (LG / 4) == 0 && i < ie)
                    g[i] = sum;
            }
        }
    }
    lds_barrier();
    float m = -INFINITY, z = 0.0f, gb = 0.0f;
    for (int i = lane; i < S; i += kWaveSize)
        m = fmaxf(m, s[i]);
    m = group_max(m, kWaveSize);
    for (int i = lane; i < S; i += kWaveSize) {
        const float e = expf(s[i] - m);
        alpha[i] = e;
        z += e;
    }
    const float inv = 1.0f / group_sum(z, kWaveSize);
    for (int i = lane; i < S; i += kWaveSize) {
        const float a = alpha[i] * inv;
        alpha[i] = a;
        gb = fmaf(a, g[i], gb);
    }
    gb = group_sum(gb, kWaveSize);
    wave_lds_sync();
    for (int i = ib + lane; i < ie; i += kWaveSize)
        ds[i] = alpha[i] * (g[i] - gb);
    wave_lds_sync();
    if constexpr (OUT == kGradCoef)
        store_coef<OUT>(coef, s, ri, ds, alpha, 0, 1, n, ib, ie, N, 1.0f / (float)r, lane, kWaveSize);
    else
        value_grads<T, value_chunks<T>(NCH * LG * CW), OUT, 1>(
            dH, dV, ib, ie, n, N, d, SLICED ? keys.base : d, lane, alpha, 1, 0);
    key_grads<FMT, T, SLICED, OUT>(keys, dhrow, dV, dK, qk, ib, ie, n, lane, s, ri, ds, alpha, dq_acc);
    store_dq<W>(keys, dq_acc, stage, r_pad, partial, n, wave, lane);
}

// VO = 16 / sizeof(T) consecutive columns of a cache row, as a lane that writes 16
// bytes of a gradient row reads them.
template <int FMT, int VO> struct OutCodes {
    typedef std::conditional_t<VO * 2 / Codes<FMT>::per_byte == 16, u32x2_t,
                               std::conditional_t<VO * 2 / Codes<FMT>::per_byte == 8, unsigned, uint16_t>>
        code_t;
    code_t c;
    unsigned e;
    // Columns col .. of the row `row` (columns past its last block: that block's).
    __device__ __forceinline__ void load(const uint8_t *__restrict__ codes,
                                         const uint8_t *__restrict__ scales, size_t row, int nb, int col)
    {
        col = min(col, nb * kCacheBlock - VO);
        c = *reinterpret_cast<const code_t *>(codes + (row * nb * kCacheBlock) / Codes<FMT>::per_byte +
                                              (unsigned)(col / Codes<FMT>::per_byte));
        e = scales[row * nb + (unsigned)col / kCacheBlock];
    }
    __device__ __forceinline__ void values(float (&x)[VO]) const
    {
        const float sc = block_scale(e);
        float y[8];
        if constexpr (VO == 8) {
            decode<FMT>(c, sc, y);
        } else if constexpr (FMT == LRAR_CACHE_FP8) {
            decode_fp8(c, sc, y);
        } else {
            decode_fp4(c, sc, y);
        }
#pragma unroll
        for (int k = 0; k < VO; ++k)
            x[k] = y[k];
    }
};

// Full-rank dots on the matrix cores (cache_full.h has both sides measured).
template <int FMT, int LG, int NCH> constexpr bool full_tiles()
{
    return FMT == LRAR_CACHE_FP4 && NCH * LG * unit_cols<FMT>() <= kTileUnits * kCacheBlock;
}

// Full-rank keys: one token a workgroup at a time (tpw in turn).  Pass 1 forms
// |x|^2, q.x and dH.x of its sources, which meet in LDS: e2m1 rows of up to 1024
// columns on the matrix cores (tile_dots), others dealt to the waves' groups of lanes.  Pass 2 deals
// the sources to the waves, reads the rows again (from the L2) in the layout of the
// gradient rows, whole lines a store, and writes
//     dV_i = alpha_i dH + (ds_i / rho_i)(q - x_i s_i / (rho_i d)),
// adding (ds_i / rho_i) x_i to dq.
template <int FMT, typename T, int LG, int NCH, bool ADD>
__global__ void __launch_bounds__(kBlock)
cache_bwd_full(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales,
               const float *__restrict__ q, const T *__restrict__ dH, T *__restrict__ dV,
               float *__restrict__ partial, int S, int N, int d, float eps, int s_pad, int tpw)
{
    constexpr int G = kWaveSize / LG, CW = unit_cols<FMT>(), GG = kWaves * G;
    constexpr int per = kCacheBlock / CW;  // units a block
    constexpr int VO = 16 / sizeof(T), NO = value_chunks<T>(NCH * LG * CW), B = NO >= 8 ? 2 : 4;
    constexpr bool TILES = full_tiles<FMT, LG, NCH>();
    extern __shared__ float lds[];
    const int lane = threadIdx.x & (kWaveSize - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWaveSize);
    const Lanes<FMT, LG, NCH> ln(lane, d);
    // The scores, 1 / rho and dH.x of the sources (before that q.x, |x|^2 and dH.x).
    float *sc = lds, *ri = sc + s_pad, *g = ri + s_pad;
    float *alpha = g + (1 + wave) * s_pad;    // a wave's own
    float *stage = g + (1 + kWaves) * s_pad;  // [NO * 64 * VO]: q, at the end dq
    uint8_t *qop = reinterpret_cast<uint8_t *>(stage + NO * kWaveSize * VO);  // TILES: operands, tiles
    uint8_t *dop = qop + row_terms<float>() * term_bytes(d);
    uint8_t *tile = dop + row_terms<T>() * term_bytes(d) + wave * kTileBytes;
    const float inv_d = 1.0f / (float)d;
    const int nb = (d + kCacheBlock - 1) / kCacheBlock;
    // The query in LDS: both passes read it in their own layout, and hold it only
    // while they run.
    float *ql = stage;
    for (int j = threadIdx.x; j < NO * kWaveSize * VO; j += kBlock)
        ql[j] = j < d ? q[j] : 0.0f;
    if constexpr (TILES)
        make_operand(q, d, qop, threadIdx.x, kBlock);
    lds_barrier();
    float dqa[NO][VO];
#pragma unroll
    for (int c = 0; c < NO; ++c)
#pragma unroll
        for (int e = 0; e < VO; ++e)
            dqa[c][e] = 0.0f;
    const int bx = xcd_block().x;
    for (int t = 0; t < tpw; ++t) {
        const int n = bx * tpw + t;
        if (n >= N)
            break;  // workgroup-uniform
        if constexpr (TILES) {
            make_operand(dH + (size_t)n * d, d, dop, threadIdx.x, kBlock);
            lds_barrier();
            tile_dots<T>(codes, scales, n, N, 0, S, d, qop, tile, wave, kWaves, lane, sc, s_pad);
            lds_barrier();
            for (int i = threadIdx.x; i < S; i += kBlock) {
                const float rv = rsqrtf(ri[i] * inv_d + eps);
                sc[i] *= rv;
                ri[i] = rv;
            }
        } else {
            constexpr int U = NCH >= 4 ? 4 : 8;  // sources a group in flight
            const int i1 = wave * G + ln.g;      // its first; every GG-th follows
            const size_t first = (size_t)n * ln.nu, plane = (size_t)N * ln.nu;
            float dh[NCH][CW], qv[NCH][CW];
            load_dh<FMT, T, LG, NCH>(dH + (size_t)n * d, ln, d, dh);
#pragma unroll
            for (int c = 0; c < NCH; ++c)
#pragma unroll
                for (int e = 0; e < CW; e += 4) {
                    const f32x4_t x = *reinterpret_cast<const f32x4_t *>(ql + ln.col(c) + e);
                    qv[c][e] = x.x; qv[c][e + 1] = x.y; qv[c][e + 2] = x.z; qv[c][e + 3] = x.w;
                }
            for (int i0 = 0; i0 < S; i0 += U * GG) {
                UnitRaw<FMT> w[U][NCH];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const size_t b = min(i0 + u * GG + i1, S - 1) * plane + first;
#pragma unroll
                    for (int c = 0; c < NCH; ++c)
                        load_unit<FMT>(codes + b * 16, scales + b / per, ln.at[c], w[u][c]);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int v = 0; v < U; v += 4) {
                    if (i0 + v * GG >= S)
                        break;  // uniform
                    float ss[4], dot[4], p[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        ss[u] = dot[u] = p[u] = 0.0f;
#pragma unroll
                        for (int c = 0; c < NCH; ++c) {
                            float a = 0.0f;
#pragma unroll
                            for (int h = 0; h < CW / 16; ++h) {
                                float x[16];
                                unit_values<FMT>(w[v + u][c], h, x);
#pragma unroll
                                for (int e = 0; e < 16; ++e) {
                                    a = fmaf(x[e], x[e], a);
                                    dot[u] = fmaf(qv[c][16 * h + e], x[e], dot[u]);
                                    p[u] = fmaf(dh[c][16 * h + e], x[e], p[u]);
                                }
                            }
                            ss[u] += ln.in[c] ? a : 0.0f;
                        }
                    }
                    const float tss = four_sums<LG>(ss, lane), tdot = four_sums<LG>(dot, lane),
                                tg = four_sums<LG>(p, lane);
                    const int i = i0 + (v + four_index<LG>(lane)) * GG + i1;
                    if (lane % (LG / 4) == 0 && i < S) {
                        const float rv = rsqrtf(tss * inv_d + eps);
                        ri[i] = rv;
                        sc[i] = tdot * rv;
                        g[i] = tg;
                    }
                }
            }
        }
        lds_barrier();
        float m = -INFINITY, z = 0.0f, gb = 0.0f;
        for (int i = lane; i < S; i += kWaveSize)
            m = fmaxf(m, sc[i]);
        m = group_max(m, kWaveSize);
        for (int i = lane; i < S; i += kWaveSize) {
            const float e = expf(sc[i] - m);
            alpha[i] = e;
            z += e;
        }
        const float inv = 1.0f / group_sum(z, kWaveSize);
        for (int i = lane; i < S; i += kWaveSize) {
            const float a = alpha[i] * inv;
            alpha[i] = a;
            gb = fmaf(a, g[i], gb);
        }
        gb = group_sum(gb, kWaveSize);
        wave_lds_sync();

        float dho[NO][VO], qo[NO][VO];
#pragma unroll
        for (int c = 0; c < NO; ++c) {
            const int col = (c * kWaveSize + lane) * VO;
            const u32x4_t r = load16_elems(dH + (size_t)n * d, col, d);
            if constexpr (VO == 8)
                widen(r, dho[c]);
            else
                widen(__builtin_bit_cast(f32x4_t, r), dho[c]);
#pragma unroll
            for (int e = 0; e < VO; ++e)
                qo[c][e] = ql[col + e];
        }
        for (int i0 = wave; i0 < S; i0 += B * kWaves) {
            OutCodes<FMT, VO> z[B][NO];
#pragma unroll
            for (int u = 0; u < B; ++u)
#pragma unroll
                for (int c = 0; c < NO; ++c)
                    z[u][c].load(codes, scales, (size_t)min(i0 + u * kWaves, S - 1) * N + n, nb,
                                 (c * kWaveSize + lane) * VO);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < B; ++u) {
                const int i = i0 + u * kWaves;
                if (i >= S)
                    break;  // wave-uniform
                const float a = alpha[i];
                const float c1 = a * (g[i] - gb) * ri[i];      // ds_i / rho_i
                const float c2 = c1 * sc[i] * ri[i] * inv_d;   // ds_i s_i / (rho_i^2 d)
                T *orow = dV + ((size_t)i * N + n) * d;
#pragma unroll
                for (int c = 0; c < NO; ++c) {
                    const int col = (c * kWaveSize + lane) * VO;
                    float x[VO], y[VO];
                    z[u][c].values(x);
#pragma unroll
                    for (int e = 0; e < VO; ++e) {
                        y[e] = fmaf(a, dho[c][e], fmaf(c1, qo[c][e], -c2 * x[e]));
                        dqa[c][e] = fmaf(c1, x[e], dqa[c][e]);
                    }
                    if constexpr (ADD) {
                        const u32x4_t o = load16_elems(orow, col, d);
                        if constexpr (VO == 8)
                            add_stored(y, o);
                        else
                            add_stored(y, __builtin_bit_cast(f32x4_t, o));
                    }
                    store16_elems<T, kBwdNtStore>(orow, col, d,
                                                  __builtin_bit_cast(u32x4_t, Narrow<T, VO>::run(y)));
                }
            }
        }
        lds_barrier();  // LDS of this token is reused by the next one
    }
    // dq: the waves add their columns in turn.
    for (int w = 0; w < kWaves; ++w) {
        if (wave == w) {
#pragma unroll
            for (int c = 0; c < NO; ++c)
#pragma unroll
                for (int e = 0; e < VO; ++e) {
                    float *p = stage + (c * VO + e) * kWaveSize + lane;
                    *p = (w == 0 ? 0.0f : *p) + dqa[c][e];
                }
        }
        lds_barrier();
    }
    for (int j = threadIdx.x; j < d; j += kBlock) {
        const int at = j / VO, e = j % VO;  // at = c * 64 + lane
        partial[(size_t)bx * d + j] = stage[(at / kWaveSize * VO + e) * kWaveSize + at % kWaveSize];
    }
}

// How a backward is laid out over workgroups.
struct CacheBwdPlan {
    bool split;   // low rank: one token a workgroup
    bool many;    // low rank: several tokens a group
    int tpw, nblocks;
};
CacheBwdPlan cache_bwd_plan(const CacheProblem &p);

// Workgroups that keep the write stream of the value rows busy: from that many on
// its waves take 8 tokens (e4m3, 49 sources, 8192 tokens, d = 1024, whole backward:
// 224 us; with 2 tokens 244); with fewer tokens the sources are cut too.
constexpr int kValueBlocks = 256;
// Tokens a group of the low-rank backward where there are many, by the columns
// that its lanes hold (their dH stays in registers).
constexpr int bwd_many(int64_t cols) { return cols <= 2048 ? 4 : 2; }

template <int FMT, typename T>
hipError_t launch_cache_bwd_as(const CacheProblem &p, const void *dH, void *dV, void *dK,
                               float *coef, bool deferred, float *partial, bool accumulate,
                               hipStream_t st)
{
    const CacheBwdPlan pl = cache_bwd_plan(p);
    const T *dh = static_cast<const T *>(dH);
    T *dv = static_cast<T *>(dV), *dk = static_cast<T *>(dK);
    const int S = (int)p.S, N = (int)p.N, d = (int)p.d, r = (int)p.r;
    const int s_pad = S | 1, r_pad = (r + 3) / 4 * 4;
    return dispatch_lanes<FMT>(p.d, [&](auto lg, auto nc) -> hipError_t {
        constexpr int LG = decltype(lg)::value, NCH = decltype(nc)::value, G = kWaveSize / LG;
        if (p.mode == LRAR_MODE_FULL) {
            constexpr int NO = value_chunks<T>(NCH * LG * unit_cols<FMT>());
            const int s4 = (S + 3) / 4 * 4;  // 16-byte aligned rows behind the scores
            size_t lds = ((size_t)(3 + kWaves) * s4 + NO * (1024 / sizeof(T))) * sizeof(float);
            if constexpr (full_tiles<FMT, LG, NCH>())
                lds += (row_terms<float>() + row_terms<T>()) * term_bytes(d) + kWaves * kTileBytes;
            auto launch = [&](auto add) {
                hipLaunchKernelGGL((cache_bwd_full<FMT, T, LG, NCH, decltype(add)::value>), dim3(pl.nblocks),
                                   dim3(kBlock), lds, st, p.codes, p.scales, p.q, dh, dv, partial, S, N,
                                   d, p.eps, s4, pl.tpw);
            };
            if (accumulate)
                launch(std::true_type{});
            else
                launch(std::false_type{});
            return hipGetLastError();
        }
        auto by_form = [&](auto sliced, auto out) {
            constexpr bool SL = decltype(sliced)::value;
            constexpr CacheGrad OUT = decltype(out)::value;
            auto launch = [&](auto tw) {
                constexpr int TW = decltype(tw)::value;
                const size_t lds = ((size_t)4 * kWaves * G * TW * s_pad + kWaves * r_pad) * sizeof(float);
                hipLaunchKernelGGL((cache_bwd_lr<FMT, T, LG, NCH, SL, OUT, TW>), dim3(pl.nblocks),
                                   dim3(kBlock), lds, st, p.codes, p.scales, p.K, p.q, dh, dv, dk,
                                   coef, partial, S, N, d, r, p.eps, s_pad, r_pad);
                if constexpr (OUT != kGradCoef) {
                    constexpr int NO = value_chunks<T>(NCH * LG * unit_cols<FMT>());
                    auto rows = [&](auto tt) {
                        constexpr int TT = decltype(tt)::value;
                        const int tokens = kWaves * TT, gx = (N + tokens - 1) / tokens;
                        // Source ranges, for at least kValueBlocks workgroups.
                        const int parts = min(S, (kValueBlocks + gx - 1) / gx);
                        const int per = (S + parts - 1) / parts;
                        hipLaunchKernelGGL((cache_value_grads<T, NO, OUT, TT>),
                                           dim3((unsigned)gx, (unsigned)((S + per - 1) / per)),
                                           dim3(kBlock), 0, st, dh, coef, dv, S, N, d,
                                           SL ? (d - r) / 8 * 8 : d, per);
                    };
                    // Adding, a wave's loads of one token's rows are enough on the way, and
                    // more of them split the store stream: one token / two / the most,
                    // e4m3, whole backward: 64 x 16384 x 2048 2213 / 2219 / 3375 us, 49 x
                    // 8192 x 1024 428 / 410 / 656, 33 x 4096 x 1024 130 / 163 / -, 20 x
                    // 3000 x 4000 255 / 341 / -; fp32, 30 x 8192 x 1024 492 / 447 / 728.
                    constexpr int TM = NO <= 4 ? 8 : 4;
                    if constexpr (OUT == kGradAdd)
                        rows(std::integral_constant<int, 1>{});
                    else if (N >= kValueBlocks * kWaves * TM)
                        rows(std::integral_constant<int, TM>{});
                    else
                        rows(std::integral_constant<int, 2>{});
                }
            };
            if (pl.split)
                hipLaunchKernelGGL((cache_bwd_lr_wg<FMT, T, LG, NCH, SL, OUT, kWaves>), dim3(pl.nblocks),
                                   dim3(kBlock), ((4 + kWaves) * s_pad + kWaves * r_pad) * sizeof(float),
                                   st, p.codes, p.scales, p.K, p.q, dh, dv, dk, coef, partial, S, N,
                                   d, r, p.eps, s_pad, r_pad);
            else if (pl.many)
                launch(std::integral_constant<int, bwd_many(NCH * LG * unit_cols<FMT>())>{});
            else
                launch(std::integral_constant<int, 1>{});
        };
        auto by_out = [&](auto sliced) {
            if (deferred)
                by_form(sliced, std::integral_constant<CacheGrad, kGradCoef>{});
            else if (accumulate)
                by_form(sliced, std::integral_constant<CacheGrad, kGradAdd>{});
            else
                by_form(sliced, std::integral_constant<CacheGrad, kGradWrite>{});
        };
        if (p.mode == LRAR_MODE_SLICED)
            by_out(std::true_type{});
        else
            by_out(std::false_type{});
        return hipGetLastError();
    });
}

// Per format, each in a translation unit of its own.
hipError_t launch_cache_bwd_fp8(const CacheProblem &p, const void *dH, void *dV, void *dK,
                                float *coef, bool deferred, float *partial, bool accumulate,
                                hipStream_t st);
hipError_t launch_cache_bwd_fp4(const CacheProblem &p, const void *dH, void *dV, void *dK,
                                float *coef, bool deferred, float *partial, bool accumulate,
                                hipStream_t st);

}  // namespace lrar

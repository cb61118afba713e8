// Backward of the depth routing over a source stack in 8 or 4 bits: kernels and
// launch template, instantiated per format.  Internal to the library.
//
// With x_i the stored values and dH the upstream gradient of a token,
//     g_i = dH . x_i,  ds_i = alpha_i (g_i - sum_l alpha_l g_l),
//     dV_i = alpha_i dH (+ the key gradient in sliced and full-rank keys'
//     columns),  dk_i = (ds_i / rho_i)(q - k_i s_i / (rho_i^2 r)),
//     dq = sum ds_i k_i / rho_i,
// the weights recomputed from the keys.  The stack is read once (full rank:
// twice), in lanes of 16 columns; dV, which does not depend on it beyond the
// key columns, is written from dH alone in lanes of 8 columns, whole lines a
// wave.
#pragma once

#include "cache_device.h"

namespace lrar {

// What the backward of one site writes per source.
enum CacheGrad { kGradWrite, kGradAdd, kGradCoef };

// dq partials of the workgroup: the waves' shares in wave order.
__device__ __forceinline__ void store_dq_partial(const float *stage, int stride,
                                                 float *__restrict__ partial, int bx, int r)
{
    __syncthreads();
    for (int j = threadIdx.x; j < r; j += kBlock) {
        float sum = 0.0f;
        for (int w = 0; w < kWaves; ++w)
            sum += stage[w * stride + j];
        partial[(size_t)bx * r + j] = sum;
    }
}

// Projected / sliced keys.  A wave owns tpw tokens in turn; or (SPLIT, few
// tokens) a workgroup owns one token, its sources cut into kWaves ranges, and
// the scores and dots meet in LDS.
template <int FMT, typename T, int NCH, bool SLICED, CacheGrad OUT, bool SPLIT>
__global__ void __launch_bounds__(kBlock)
cache_bwd_lr(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales,
             const void *__restrict__ K, const float *__restrict__ q, const T *__restrict__ dH,
             T *__restrict__ dV, T *__restrict__ dK, float *__restrict__ coef,
             float *__restrict__ partial, int S, int N, int d, int r, float eps, int s_pad,
             int r_pad, int tpw)
{
    extern __shared__ float lds[];
    const int lane = threadIdx.x & (kWaveSize - 1);
    const int wave = threadIdx.x / kWaveSize;
    const int slice = SPLIT ? 0 : 4 * wave;  // s, rho, g of the workgroup when split
    float *s = lds + (slice + 0) * s_pad;
    float *rho = lds + (slice + 1) * s_pad;
    float *g = lds + (slice + 2) * s_pad;
    float *alpha = lds + (slice + 3 + (SPLIT ? wave : 0)) * s_pad;
    float *stage = lds + 4 * kWaves * s_pad;  // [kWaves][r_pad]
    const int per = SPLIT ? (S + kWaves - 1) / kWaves : S;
    const int ib = SPLIT ? min(S, wave * per) : 0, ie = SPLIT ? min(S, ib + per) : S;
    auto meet = [&]() {
        if constexpr (SPLIT)
            __syncthreads();
        else
            wave_lds_sync();
    };

    const Keys<FMT, T, SLICED> keys(K, codes, scales, N, d, r);
    const int lps = keys.lps, spi = kWaveSize / lps;
    const int isub = lane / lps, v = lane % lps;
    const int nb = (d + kCacheBlock - 1) / kCacheBlock;
    const int wend = SLICED ? keys.base : d;  // columns [0, wend) of dV are alpha dH alone
    const bool vec = d % 8 == 0;
    const float inv_r = 1.0f / (float)r;
    float qk[8], dq_acc[8];
    keys.query(q, v, qk);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        dq_acc[e] = 0.0f;

    const int bx = blockIdx.x;
    for (int t = 0; t < tpw; ++t) {
        const int n = SPLIT ? bx : (bx * tpw + t) * kWaves + wave;
        if (n >= N)
            break;  // wave-uniform; the barrier below is outside the loop (SPLIT: n < N)
        const T *dhrow = dH + (size_t)n * d;
        if (ie > ib)
            cache_scores<FMT, T, SLICED, 1>(keys, q, ib, ie, n, eps, lane, s, rho, s_pad);
        meet();
        depth_softmax<true>(s, alpha, S, lane);

        // The dots of dH with the stored rows.
        {
            float dh[NCH][16];
#pragma unroll
            for (int c = 0; c < NCH; ++c)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float y[8];
                    load8(dhrow, lane * kCacheVec + c * 1024 + 8 * h, d, vec, y);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        dh[c][8 * h + e] = y[e];
                }
            constexpr int U = NCH >= 4 ? 2 : 4;
            for (int i0 = ib; i0 < ie; i0 += 8) {
                float part[8];
#pragma unroll
                for (int h = 0; h < 8; h += U) {
                    RowRaw<FMT> w[U][NCH];
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int c = 0; c < NCH; ++c)
                            load_row<FMT>(codes, scales, (size_t)min(i0 + h + u, ie - 1) * N + n,
                                          nb, RowAt<FMT>(lane * kCacheVec + c * 1024, nb),
                                          w[u][c]);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        float p = 0.0f;
#pragma unroll
                        for (int c = 0; c < NCH; ++c) {
                            float x[16];
                            row_values<FMT>(w[u][c], x);
#pragma unroll
                            for (int e = 0; e < 16; ++e)
                                p = fmaf(dh[c][e], x[e], p);
                        }
                        part[h + u] = p;
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                const float tot = multi_sum<8>(part, lane);
                const int idx = multi_sum_index<8>(lane);
                if (multi_sum_writer<8>(lane) && i0 + idx < ie)
                    g[i0 + idx] = tot;
            }
        }
        meet();
        float gb = 0.0f;
        for (int i = lane; i < S; i += kWaveSize)
            gb = fmaf(alpha[i], g[i], gb);
        gb = wave_sum_t<true>(gb);
        if constexpr (SPLIT)
            meet();  // every wave has read the dots
        for (int i = ib + lane; i < ie; i += kWaveSize)
            g[i] = alpha[i] * (g[i] - gb);  // g now holds ds
        wave_lds_sync();

        // Key gradients: lanes over (source, key slot).
        float dhk[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            dhk[e] = 0.0f;
        if (SLICED && OUT != kGradCoef && v < keys.nkv)
            load8(dhrow, keys.base + v * 8, d, vec, dhk);
        for (int i0 = ib; i0 < ie; i0 += spi) {
            const int i = i0 + isub;
            if (v >= keys.nkv || i >= ie)
                continue;
            typename Keys<FMT, T, SLICED>::Raw w;
            float x[8];
            keys.load(i, n, v, w);
            keys.values(w, v, x);
            const size_t row = (size_t)i * N + n;
            const float ri = 1.0f / rho[i];
            const float dsi = g[i];
            const float cq = dsi * ri;           // ds_i / rho_i
            const float ck = cq * s[i] * inv_r;  // ds_i s_i / (rho_i r)
            if (OUT == kGradCoef && v == 0) {
                coef[((size_t)i * 3 + 0) * N + n] = alpha[i];
                coef[((size_t)i * 3 + 1) * N + n] = cq;
                coef[((size_t)i * 3 + 2) * N + n] = ck;
            }
            float y[8];
            const float a = SLICED ? alpha[i] : 0.0f;
            const int j = keys.first(v);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float kb = x[e] * ri;
                dq_acc[e] = fmaf(dsi, kb, dq_acc[e]);
                y[e] = a * dhk[e];
                if (j + e >= 0)
                    y[e] += fmaf(cq, qk[e], -ck * kb);
            }
            if constexpr (OUT != kGradCoef) {
                T *orow = SLICED ? dV + row * d : dK + row * r;
                const int ocol = SLICED ? keys.base + v * 8 : v * 8;
                const int width = SLICED ? d : r;
                const bool ovec = SLICED ? vec : keys.vec;
                if constexpr (OUT == kGradAdd) {
                    float o[8];
                    load8(orow, ocol, width, ovec, o);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        y[e] += o[e];
                }
                store8<T, false>(orow, ocol, width, ovec, y);
            }
        }

        // dV_i = alpha_i dH before the key columns.
        if constexpr (OUT != kGradCoef) {
            constexpr int NO = 2 * NCH;  // chunks of 512 columns
            float dh[NO][8];
#pragma unroll
            for (int c = 0; c < NO; ++c)
                load8(dhrow, lane * 8 + c * 512, d, vec, dh[c]);
            for (int i = ib; i < ie; ++i) {
                const float a = alpha[i];
                T *orow = dV + ((size_t)i * N + n) * d;
#pragma unroll
                for (int c = 0; c < NO; ++c) {
                    const int col = lane * 8 + c * 512;
                    float y[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        y[e] = a * dh[c][e];
                    if constexpr (OUT == kGradAdd) {
                        float o[8];
                        load8(orow, col, wend, vec, o);
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            y[e] += o[e];
                    }
                    store8<T, true>(orow, col, wend, vec, y);
                }
            }
        }
        wave_lds_sync();  // LDS of this token is reused by the next one
    }

    // dq: over the source groups of the wave, then over the waves.
#pragma unroll
    for (int e = 0; e < 8; ++e)
        for (int m = lps; m < kWaveSize; m <<= 1)
            dq_acc[e] += __shfl_xor(dq_acc[e], m, kWaveSize);
    float *my = stage + wave * r_pad;
    if (isub == 0 && v < keys.nkv) {
        const int j = keys.first(v);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (j + e >= 0 && j + e < r)
                my[j + e] = dq_acc[e];
    }
    store_dq_partial(stage, r_pad, partial, bx, r);
}

// Full-rank keys: pass 1 reads the rows for sum(x^2), q.x and dH.x; pass 2 reads
// them again for dV_i = alpha_i dH + (ds_i / rho_i)(q - x_i s_i / (rho_i d)) and
// dq.  One token a wave at a time, tpw in turn.
template <int FMT, typename T, int NCH, bool ADD>
__global__ void __launch_bounds__(kBlock)
cache_bwd_full(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales,
               const float *__restrict__ q, const T *__restrict__ dH, T *__restrict__ dV,
               float *__restrict__ partial, int S, int N, int d, float eps, int s_pad, int tpw)
{
    extern __shared__ float lds[];
    const int lane = threadIdx.x & (kWaveSize - 1);
    const int wave = threadIdx.x / kWaveSize;
    float *ss = lds + (4 * wave + 0) * s_pad;     // sum x^2, then rho
    float *sc = lds + (4 * wave + 1) * s_pad;     // q.x, then the score
    float *g = lds + (4 * wave + 2) * s_pad;      // dH.x, then ds
    float *alpha = lds + (4 * wave + 3) * s_pad;
    float *stage = lds + 4 * kWaves * s_pad;      // [NCH * 1024]
    const int nb = (d + kCacheBlock - 1) / kCacheBlock;
    const int col = lane * kCacheVec;
    const bool vec = d % 8 == 0;
    const float inv_d = 1.0f / (float)d;
    float qv[NCH][16], dqa[NCH][16];
    bool in[NCH];
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        in[c] = col + c * 1024 < nb * kCacheBlock;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int j = col + c * 1024 + e;
            qv[c][e] = j < d ? q[j] : 0.0f;
            dqa[c][e] = 0.0f;
        }
    }
    const int bx = blockIdx.x;
    for (int t = 0; t < tpw; ++t) {
        const int n = (bx * tpw + t) * kWaves + wave;
        if (n >= N)
            break;  // wave-uniform; the workgroup barriers are after the loop
        float dh[NCH][16];
#pragma unroll
        for (int c = 0; c < NCH; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float y[8];
                load8(dH + (size_t)n * d, col + c * 1024 + 8 * h, d, vec, y);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    dh[c][8 * h + e] = y[e];
            }
        for (int i0 = 0; i0 < S; i0 += 4) {
            RowRaw<FMT> w[4][NCH];
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int c = 0; c < NCH; ++c)
                    load_row<FMT>(codes, scales, (size_t)min(i0 + u, S - 1) * N + n, nb,
                                  RowAt<FMT>(col + c * 1024, nb), w[u][c]);
            __builtin_amdgcn_sched_barrier(0);
            float part[16];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                float a = 0.0f, b = 0.0f, p = 0.0f;
#pragma unroll
                for (int c = 0; c < NCH; ++c) {
                    float x[16], ac = 0.0f;
                    row_values<FMT>(w[u][c], x);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        ac = fmaf(x[e], x[e], ac);
                        b = fmaf(qv[c][e], x[e], b);
                        p = fmaf(dh[c][e], x[e], p);
                    }
                    a += in[c] ? ac : 0.0f;
                }
                part[u] = a;
                part[4 + u] = b;
                part[8 + u] = p;
                part[12 + u] = 0.0f;
            }
            const float tot = multi_sum<16>(part, lane);
            const int idx = multi_sum_index<16>(lane);
            const int i = i0 + (idx & 3);
            if (multi_sum_writer<16>(lane) && idx < 12 && i < S)
                (idx < 4 ? ss : idx < 8 ? sc : g)[i] = tot;
        }
        wave_lds_sync();
        for (int i = lane; i < S; i += kWaveSize) {
            const float rho = sqrtf(ss[i] / (float)d + eps);
            ss[i] = rho;
            sc[i] = sc[i] / rho;
        }
        wave_lds_sync();
        depth_softmax<true>(sc, alpha, S, lane);
        float gb = 0.0f;
        for (int i = lane; i < S; i += kWaveSize)
            gb = fmaf(alpha[i], g[i], gb);
        gb = wave_sum_t<true>(gb);
        for (int i = lane; i < S; i += kWaveSize)
            g[i] = alpha[i] * (g[i] - gb);
        wave_lds_sync();

        for (int i = 0; i < S; ++i) {
            const float a = alpha[i];
            const float c1 = g[i] / ss[i];                  // ds_i / rho_i
            const float c2 = c1 * sc[i] / ss[i] * inv_d;    // ds_i s_i / (rho_i^2 d)
            T *orow = dV + ((size_t)i * N + n) * d;
            RowRaw<FMT> w[NCH];
#pragma unroll
            for (int c = 0; c < NCH; ++c)
                load_row<FMT>(codes, scales, (size_t)i * N + n, nb,
                              RowAt<FMT>(col + c * 1024, nb), w[c]);
#pragma unroll
            for (int c = 0; c < NCH; ++c) {
                float x[16];
                row_values<FMT>(w[c], x);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int oc = col + c * 1024 + 8 * h;
                    float y[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int k = 8 * h + e;
                        y[e] = fmaf(a, dh[c][k], fmaf(c1, qv[c][k], -c2 * x[k]));
                        dqa[c][k] = fmaf(c1, x[k], dqa[c][k]);
                    }
                    if constexpr (ADD) {
                        float o[8];
                        load8(orow, oc, d, vec, o);
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            y[e] += o[e];
                    }
                    store8<T, false>(orow, oc, d, vec, y);
                }
            }
        }
        wave_lds_sync();
    }
    // dq: the waves add their columns in turn.
    for (int w = 0; w < kWaves; ++w) {
        if (wave == w) {
#pragma unroll
            for (int c = 0; c < NCH; ++c)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    float *p = stage + c * 1024 + e * 64 + lane;
                    *p = (w == 0 ? 0.0f : *p) + dqa[c][e];
                }
        }
        __syncthreads();
    }
    for (int j = threadIdx.x; j < d; j += kBlock) {
        const int k = j % 1024;
        partial[(size_t)bx * d + j] = stage[j - k + k % 16 * 64 + k / 16];
    }
}

// How a backward is laid out over workgroups.
struct CacheBwdPlan {
    bool split;
    int tpw, nblocks;
};
CacheBwdPlan cache_bwd_plan(const CacheProblem &p);

template <int FMT, typename T>
hipError_t launch_cache_bwd_as(const CacheProblem &p, const void *dH, void *dV, void *dK,
                               float *coef, float *partial, bool accumulate, hipStream_t st)
{
    const CacheBwdPlan pl = cache_bwd_plan(p);
    const T *dh = static_cast<const T *>(dH);
    T *dv = static_cast<T *>(dV), *dk = static_cast<T *>(dK);
    const int S = (int)p.S, N = (int)p.N, d = (int)p.d, r = (int)p.r;
    const int s_pad = (S + 3) / 4 * 4, r_pad = (r + 3) / 4 * 4;
    const size_t slices = (size_t)4 * kWaves * s_pad;
    return dispatch_row_chunks(p.d, [&](auto nch) -> hipError_t {
        constexpr int NCH = decltype(nch)::value;
        if (p.mode == LRAR_MODE_FULL) {
            const size_t lds = (slices + NCH * 1024) * sizeof(float);
            if (accumulate)
                hipLaunchKernelGGL((cache_bwd_full<FMT, T, NCH, true>), dim3(pl.nblocks),
                                   dim3(kBlock), lds, st, p.codes, p.scales, p.q, dh, dv, partial,
                                   S, N, d, p.eps, s_pad, pl.tpw);
            else
                hipLaunchKernelGGL((cache_bwd_full<FMT, T, NCH, false>), dim3(pl.nblocks),
                                   dim3(kBlock), lds, st, p.codes, p.scales, p.q, dh, dv, partial,
                                   S, N, d, p.eps, s_pad, pl.tpw);
            return hipGetLastError();
        }
        const size_t lds = (slices + kWaves * r_pad) * sizeof(float);
        auto launch = [&](auto sliced, auto out, auto split) {
            hipLaunchKernelGGL((cache_bwd_lr<FMT, T, NCH, decltype(sliced)::value,
                                             decltype(out)::value, decltype(split)::value>),
                               dim3(pl.nblocks), dim3(kBlock), lds, st, p.codes, p.scales, p.K,
                               p.q, dh, dv, dk, coef, partial, S, N, d, r, p.eps, s_pad, r_pad,
                               pl.tpw);
        };
        auto by_split = [&](auto sliced, auto out) {
            if (pl.split)
                launch(sliced, out, std::true_type{});
            else
                launch(sliced, out, std::false_type{});
        };
        auto by_out = [&](auto sliced) {
            if (coef)
                by_split(sliced, std::integral_constant<CacheGrad, kGradCoef>{});
            else if (accumulate)
                by_split(sliced, std::integral_constant<CacheGrad, kGradAdd>{});
            else
                by_split(sliced, std::integral_constant<CacheGrad, kGradWrite>{});
        };
        if (p.mode == LRAR_MODE_SLICED)
            by_out(std::true_type{});
        else
            by_out(std::false_type{});
        return hipGetLastError();
    });
}

// Per format and storage, each in a translation unit of its own.
hipError_t launch_cache_bwd_fp8(const CacheProblem &p, const void *dH, void *dV, void *dK,
                                float *coef, float *partial, bool accumulate, hipStream_t st);
hipError_t launch_cache_bwd_fp4(const CacheProblem &p, const void *dH, void *dV, void *dK,
                                float *coef, float *partial, bool accumulate, hipStream_t st);

}  // namespace lrar

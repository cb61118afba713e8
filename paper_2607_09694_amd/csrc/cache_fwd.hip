// Forward of the depth routing over a source stack in 8 or 4 bits (Sec. 3.2,
// Eqs. lr_key_norm, lr_attnres_weight, lr_attnres_output, with the values that
// the stack holds).
//
// A wave owns a token; a lane owns 16 columns of each chunk of 1024, one load of
// 16 (e4m3) or 8 (e2m1) bytes and one scale byte a source.  Decoding costs half
// an instruction a column and the sum one, so the reads of the stack stay the
// bound as they are in bf16.
#include "cache_device.h"

namespace lrar {

namespace {

// H's row of a wave: lane columns col .. col + 15 of each chunk.
template <typename T, int NCH>
__device__ __forceinline__ void store_h(T *__restrict__ hrow, int col, int d, bool vec,
                                        const float (&acc)[NCH][16])
{
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                y[e] = acc[c][8 * h + e];
            store8<T, false>(hrow, col + c * 1024 + 8 * h, d, vec, y);
        }
}

// Merges the online-softmax states (m, l, acc) that the W waves of a workgroup
// hold of one token's sources, and stores h:
//     m* = max_w m_w,  h = sum_w e^(m_w - m*) acc_w / sum_w e^(m_w - m*) l_w.
// stat: 2 W floats; part: the accumulators of waves 1 .. W-1.  Every wave calls it.
template <typename T, int NCH, int W>
__device__ __forceinline__ void merge_store(float (&acc)[NCH][16], float m, float l, float *stat,
                                            float *part, T *__restrict__ hrow, int col, int d,
                                            bool vec, int wave, int lane)
{
    constexpr int kRow = NCH * 1024;
    if (lane == 0) {
        stat[wave] = m;
        stat[W + wave] = l;
    }
    if (wave > 0) {
#pragma unroll
        for (int c = 0; c < NCH; ++c)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<f32x4_t *>(part + (wave - 1) * kRow + c * 1024 + e * 64 + lane * 4) =
                    f32x4_t{acc[c][e], acc[c][e + 1], acc[c][e + 2], acc[c][e + 3]};
    }
    __syncthreads();
    if (wave != 0)
        return;
    float mg = stat[0];
    for (int u = 1; u < W; ++u)
        mg = fmaxf(mg, stat[u]);
    float ls = 0.0f;
    for (int u = 0; u < W; ++u)
        ls = fmaf(expf(stat[u] - mg), stat[W + u], ls);  // 0 for a wave without sources
    const float inv = 1.0f / ls;
    const float s0 = expf(stat[0] - mg);
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            acc[c][e] *= s0;
    for (int u = 1; u < W; ++u) {
        const float su = expf(stat[u] - mg);
#pragma unroll
        for (int c = 0; c < NCH; ++c)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const f32x4_t y = *reinterpret_cast<const f32x4_t *>(part + (u - 1) * kRow +
                                                                     c * 1024 + e * 64 + lane * 4);
                acc[c][e] = fmaf(su, y.x, acc[c][e]);
                acc[c][e + 1] = fmaf(su, y.y, acc[c][e + 1]);
                acc[c][e + 2] = fmaf(su, y.z, acc[c][e + 2]);
                acc[c][e + 3] = fmaf(su, y.w, acc[c][e + 3]);
            }
    }
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            acc[c][e] *= inv;
    store_h<T, NCH>(hrow, col, d, vec, acc);
}

}  // namespace

// Projected / sliced keys, one token a wave.  Grid x = tokens in groups of
// kWaves, y = column blocks of NCH * 1024 (each recomputes the cheap scores).
template <int FMT, typename T, int NCH, bool SLICED>
__global__ void __launch_bounds__(kBlock)
cache_fwd_lr(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales,
             const void *__restrict__ K, const float *__restrict__ q, T *__restrict__ H, int S,
             int N, int d, int r, float eps, int s_pad)
{
    constexpr int U = NCH >= 4 ? 2 : 4;
    extern __shared__ float lds[];
    const int lane = threadIdx.x & (kWaveSize - 1);
    const int wave = threadIdx.x / kWaveSize;
    const int n = (int)blockIdx.x * kWaves + wave;
    if (n >= N)
        return;  // wave-uniform; this kernel has no workgroup barrier
    float *s = lds + wave * s_pad;
    const int nb = (d + kCacheBlock - 1) / kCacheBlock;
    const int col = (int)blockIdx.y * NCH * 1024 + lane * kCacheVec;
    cache_scores<FMT, T, SLICED, 1>(Keys<FMT, T, SLICED>(K, codes, scales, N, d, r), q, 0, S, n,
                                    eps, lane, s, nullptr, s_pad);
    wave_lds_sync();
    depth_softmax<true>(s, s, S, lane);
    float acc[NCH][16];
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            acc[c][e] = 0.0f;
    for (int i0 = 0; i0 < S; i0 += U) {
        RowRaw<FMT> w[U][NCH];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int c = 0; c < NCH; ++c)
                load_row<FMT>(codes, scales, (size_t)min(i0 + u, S - 1) * N + n, nb,
                              RowAt<FMT>(col + c * 1024, nb), w[u][c]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float a = i0 + u < S ? s[min(i0 + u, S - 1)] : 0.0f;
#pragma unroll
            for (int c = 0; c < NCH; ++c) {
                float x[16];
                row_values<FMT>(w[u][c], x);
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    acc[c][e] = fmaf(a, x[e], acc[c][e]);
            }
        }
    }
    store_h<T, NCH>(H + (size_t)n * d, col, d, d % 8 == 0, acc);
}

// The same for few tokens: one token a workgroup of W waves, its sources cut
// into W ranges, whose online-softmax states meet in LDS.
template <int FMT, typename T, int NCH, bool SLICED, int W>
__global__ void __launch_bounds__(W * kWaveSize)
cache_fwd_lr_wg(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales,
                const void *__restrict__ K, const float *__restrict__ q, T *__restrict__ H, int S,
                int N, int d, int r, float eps, int s_pad)
{
    constexpr int U = NCH >= 4 ? 2 : 4;
    extern __shared__ float lds[];
    const int lane = threadIdx.x & (kWaveSize - 1);
    const int wave = threadIdx.x / kWaveSize;
    const int n = blockIdx.x;
    const int per = (S + W - 1) / W;
    const int ib = min(S, wave * per), ie = min(S, ib + per);
    float *stat = lds;
    float *part = lds + 2 * W;
    float *s = part + (W - 1) * NCH * 1024 + wave * s_pad - ib;  // s[ib .. ie - 1]
    const int nb = (d + kCacheBlock - 1) / kCacheBlock;
    const int col = (int)blockIdx.y * NCH * 1024 + lane * kCacheVec;
    float acc[NCH][16];
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            acc[c][e] = 0.0f;
    float m = -INFINITY, l = 0.0f;
    if (ib < ie) {  // wave-uniform
        RowRaw<FMT> w[U][NCH];
        auto load = [&](int i0) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int c = 0; c < NCH; ++c)
                    load_row<FMT>(codes, scales, (size_t)min(i0 + u, ie - 1) * N + n, nb,
                                  RowAt<FMT>(col + c * 1024, nb), w[u][c]);
        };
        load(ib);  // does not depend on the scores: waits with the key loads
        cache_scores<FMT, T, SLICED, 1>(Keys<FMT, T, SLICED>(K, codes, scales, N, d, r), q, ib,
                                        ie, n, eps, lane, s, nullptr, s_pad);
        wave_lds_sync();
        for (int i = ib + lane; i < ie; i += kWaveSize)
            m = fmaxf(m, s[i]);
        m = wave_max_t<true>(m);
        for (int i = ib + lane; i < ie; i += kWaveSize) {
            const float e = expf(s[i] - m);
            s[i] = e;
            l += e;
        }
        l = wave_sum_t<true>(l);
        wave_lds_sync();
        for (int i0 = ib; i0 < ie; i0 += U) {
            if (i0 > ib)
                load(i0);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float a = i0 + u < ie ? s[min(i0 + u, ie - 1)] : 0.0f;
#pragma unroll
                for (int c = 0; c < NCH; ++c) {
                    float x[16];
                    row_values<FMT>(w[u][c], x);
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        acc[c][e] = fmaf(a, x[e], acc[c][e]);
                }
            }
        }
    }
    merge_store<T, NCH, W>(acc, m, l, stat, part, H + (size_t)n * d, col, d, d % 8 == 0, wave,
                           lane);
}

// Full-rank keys: each batch of four sources is scored from the rows in
// registers and joins the online softmax.  W = 0: a token a wave, kWaves waves;
// else a token a workgroup of W waves as above.
template <int FMT, typename T, int NCH, int W>
__global__ void __launch_bounds__(W == 0 ? kBlock : W * kWaveSize)
cache_fwd_full(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales,
               const float *__restrict__ q, T *__restrict__ H, int S, int N, int d, float eps)
{
    extern __shared__ float lds[];
    const int lane = threadIdx.x & (kWaveSize - 1);
    const int wave = threadIdx.x / kWaveSize;
    const int n = W == 0 ? (int)blockIdx.x * kWaves + wave : (int)blockIdx.x;
    if (W == 0 && n >= N)
        return;  // wave-uniform; no workgroup barrier on this path
    const int per = W == 0 ? S : (S + W - 1) / W;
    const int ib = W == 0 ? 0 : min(S, wave * per), ie = min(S, ib + per);
    const int nb = (d + kCacheBlock - 1) / kCacheBlock;
    const int col = lane * kCacheVec;
    float qv[NCH][16], acc[NCH][16];
    bool in[NCH];  // a lane past the row re-reads other lanes' columns: not counted
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        in[c] = col + c * 1024 < nb * kCacheBlock;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int j = col + c * 1024 + e;
            qv[c][e] = j < d ? q[j] : 0.0f;
            acc[c][e] = 0.0f;
        }
    }
    float m = -INFINITY, l = 0.0f;
    for (int i0 = ib; i0 < ie; i0 += 4) {
        RowRaw<FMT> w[4][NCH];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int c = 0; c < NCH; ++c)
                load_row<FMT>(codes, scales, (size_t)min(i0 + u, ie - 1) * N + n, nb,
                              RowAt<FMT>(col + c * 1024, nb), w[u][c]);
        __builtin_amdgcn_sched_barrier(0);
        float part[8];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            float a = 0.0f, b = 0.0f;
#pragma unroll
            for (int c = 0; c < NCH; ++c) {
                float x[16], ac = 0.0f;
                row_values<FMT>(w[u][c], x);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    ac = fmaf(x[e], x[e], ac);
                    b = fmaf(qv[c][e], x[e], b);
                }
                a += in[c] ? ac : 0.0f;
            }
            part[u] = a;
            part[4 + u] = b;
        }
        const float tot = multi_sum<8>(part, lane);
        float sc[4], mb = -INFINITY;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float ss = lane_value<8>(tot, u), dot = lane_value<8>(tot, 4 + u);
            sc[u] = i0 + u < ie ? dot / sqrtf(ss / (float)d + eps) : -INFINITY;
            mb = fmaxf(mb, sc[u]);
        }
        if (mb > m) {  // wave-uniform
            const float scale = expf(m - mb);
            l *= scale;
#pragma unroll
            for (int c = 0; c < NCH; ++c)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    acc[c][e] *= scale;
            m = mb;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float a = i0 + u < ie ? expf(sc[u] - m) : 0.0f;
            l += a;
#pragma unroll
            for (int c = 0; c < NCH; ++c) {
                float x[16];
                row_values<FMT>(w[u][c], x);
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    acc[c][e] = fmaf(a, x[e], acc[c][e]);
            }
        }
    }
    T *hrow = H + (size_t)n * d;
    if constexpr (W != 0) {
        merge_store<T, NCH, W>(acc, m, l, lds, lds + 2 * W, hrow, col, d, d % 8 == 0, wave, lane);
    } else {
        const float inv = 1.0f / l;
#pragma unroll
        for (int c = 0; c < NCH; ++c)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                acc[c][e] *= inv;
        store_h<T, NCH>(hrow, col, d, d % 8 == 0, acc);
    }
}

namespace {

constexpr int64_t kMaxSourcesFwd = 1024, kMaxSourcesBwd = 512, kMaxRankBwd = 256;
constexpr int64_t kMaxRow = 4096;            // columns that a wave holds
constexpr int64_t kMaxColumns = 1 << 20;     // of a row in column blocks

// Tokens up to which a token's sources are split over a workgroup.
constexpr int64_t kSplitTokens = 2048;

template <int FMT, typename T>
hipError_t launch_fwd_as(const CacheProblem &p, void *H, hipStream_t st)
{
    T *h = static_cast<T *>(H);
    const int S = (int)p.S, N = (int)p.N, d = (int)p.d, r = (int)p.r;
    constexpr int W = kWaves;
    const bool split = p.N <= kSplitTokens && p.S > 1;
    const unsigned gx = (unsigned)(split ? N : (N + kWaves - 1) / kWaves);
    return dispatch_row_chunks(p.d, [&](auto nch) -> hipError_t {
        constexpr int NCH = decltype(nch)::value;
        const unsigned gy = (unsigned)((d + NCH * 1024 - 1) / (NCH * 1024));
        const size_t meet = (2 * W + (W - 1) * NCH * 1024) * sizeof(float);
        if (p.mode == LRAR_MODE_FULL) {
            if (split)
                hipLaunchKernelGGL((cache_fwd_full<FMT, T, NCH, W>), dim3(gx), dim3(kBlock), meet,
                                   st, p.codes, p.scales, p.q, h, S, N, d, p.eps);
            else
                hipLaunchKernelGGL((cache_fwd_full<FMT, T, NCH, 0>), dim3(gx), dim3(kBlock), 0, st,
                                   p.codes, p.scales, p.q, h, S, N, d, p.eps);
            return hipGetLastError();
        }
        auto launch = [&](auto sliced) {
            constexpr bool SL = decltype(sliced)::value;
            if (split) {
                const int s_pad = (S + W - 1) / W;
                hipLaunchKernelGGL((cache_fwd_lr_wg<FMT, T, NCH, SL, W>), dim3(gx, gy),
                                   dim3(kBlock), meet + W * s_pad * sizeof(float), st, p.codes,
                                   p.scales, p.K, p.q, h, S, N, d, r, p.eps, s_pad);
            } else {
                hipLaunchKernelGGL((cache_fwd_lr<FMT, T, NCH, SL>), dim3(gx, gy), dim3(kBlock),
                                   kWaves * S * sizeof(float), st, p.codes, p.scales, p.K, p.q, h,
                                   S, N, d, r, p.eps, S);
            }
        };
        if (p.mode == LRAR_MODE_SLICED)
            launch(std::true_type{});
        else
            launch(std::false_type{});
        return hipGetLastError();
    });
}

}  // namespace

int check_cache_supported(const CacheProblem &p, bool bwd, std::string *why)
{
    if (p.N > (1 << 30)) {
        *why = "N exceeds 2^30 tokens";
    } else if (p.S > (bwd ? kMaxSourcesBwd : kMaxSourcesFwd)) {
        *why = bwd ? "backward supports at most 512 sources" : "forward supports at most 1024 sources";
    } else if (bwd && p.mode != LRAR_MODE_FULL && p.r > kMaxRankBwd) {
        *why = "backward with projected or sliced keys supports r <= 256";
    } else if (p.d > (bwd || p.mode == LRAR_MODE_FULL ? kMaxRow : kMaxColumns)) {
        *why = "row width d too large";
    } else if (p.mode == LRAR_MODE_PROJECTED && p.r > kMaxColumns) {
        *why = "key width r too large";
    } else {
        return LRAR_OK;
    }
    return LRAR_EUNSUPPORTED;
}

int launch_cache_fwd(const CacheProblem &p, const void *o_new, void *H, hipStream_t st,
                     std::string *err)
{
    if (p.N == 0)
        return LRAR_OK;
    if (o_new) {
        const int64_t first = (p.S - 1) * p.N;
        const int rc = launch_cache_write(
            o_new, const_cast<uint8_t *>(p.codes) + first * cache_row_bytes(p.d, p.format),
            const_cast<uint8_t *>(p.scales) + first * cache_blocks(p.d), p.N, p.d, p.format,
            p.dtype, st, err);
        if (rc)
            return rc;
    }
    hipError_t e;
    if (p.dtype == LRAR_DTYPE_BF16)
        e = p.format == LRAR_CACHE_FP8 ? launch_fwd_as<LRAR_CACHE_FP8, uint16_t>(p, H, st)
                                       : launch_fwd_as<LRAR_CACHE_FP4, uint16_t>(p, H, st);
    else
        e = p.format == LRAR_CACHE_FP8 ? launch_fwd_as<LRAR_CACHE_FP8, float>(p, H, st)
                                       : launch_fwd_as<LRAR_CACHE_FP4, float>(p, H, st);
    return hip_status(e, "cache_route_fwd launch", err);
}

}  // namespace lrar

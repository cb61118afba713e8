// Forward of the depth routing over a source stack in 8 or 4 bits (Sec. 3.2,
// Eqs. lr_key_norm, lr_attnres_weight, lr_attnres_output, with the values that
// the stack holds).
//
// A lane takes 16 bytes of codes and one scale byte a source.  Decoding costs half
// an instruction a column and the sum one, so the reads of the stack stay the
// bound, as they are in bf16: 64 sources, 16384 tokens, d = 2048, e4m3, projected
// r = 32 takes 350 us, 6.7 TB/s (a bf16 stack: 656 us).  Full-rank keys add two
// products a column (|x|^2 and q . x) and the second decoding, and are bound by
// them where the codes are small: 49 sources, 4096 tokens, d = 1024, e2m1 36 us,
// of which the vector instructions are about two thirds.
#include "cache_device.h"

namespace lrar {

namespace {

// Row of h from a lane's units.
template <int FMT, typename T, int LG, int NCH>
__device__ __forceinline__ void store_h(T *__restrict__ hrow, const Lanes<FMT, LG, NCH> &ln, int col0,
                                        int d, const float (&acc)[NCH][UnitRaw<FMT>::cols])
{
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int h = 0; h < unit_cols<FMT>() / 8; ++h) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                y[e] = acc[c][8 * h + e];
            store8<T, false>(hrow, col0 + ln.col(c) + 8 * h, d, y);
        }
}

// Merges the online-softmax states (m, l, acc) of one token's sources that the W
// waves of a workgroup hold, each group of LG lanes its share of acc, and stores
// h:  m* = max_w m_w,  h = sum_w e^(m_w - m*) acc_w / sum_w e^(m_w - m*) l_w.
// The groups' shares are added by halving exchanges, which leave every lane
// CW / G of its unit's columns; the waves' rows then meet in LDS and every thread
// finishes four columns at a time.  stat: 2 W floats; part: W rows.
template <int FMT, typename T, int LG, int NCH, int W>
__device__ __forceinline__ void merge_store(float (&acc)[NCH][UnitRaw<FMT>::cols],
                                            const Lanes<FMT, LG, NCH> &ln, float m, float l,
                                            float *stat, float *part, T *__restrict__ hrow,
                                            int col0, int d, int wave, int lane)
{
    constexpr int CW = unit_cols<FMT>(), G = kWaveSize / LG, kRow = NCH * LG * CW;
    if (lane == 0) {
        stat[wave] = m;
        stat[W + wave] = l;
    }
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        float *v = acc[c];
        if constexpr (G >= 2) {
#pragma unroll
            for (int e = 0; e < CW / 2; ++e)
                v[e] = halve32(v[e], v[e + CW / 2]);
        }
        if constexpr (G >= 4) {
#pragma unroll
            for (int e = 0; e < CW / 4; ++e)
                v[e] = halve16(v[e], v[e + CW / 4]);
        }
        const int share = (G >= 2 && (lane & 32) ? CW / 2 : 0) + (G >= 4 && (lane & 16) ? CW / 4 : 0);
        float *dst = part + wave * kRow + (ln.lu + c * LG) * CW + share;
#pragma unroll
        for (int e = 0; e < CW / G; e += 4)
            *reinterpret_cast<f32x4_t *>(dst + e) = f32x4_t{v[e], v[e + 1], v[e + 2], v[e + 3]};
    }
    lds_barrier();
    float mg = stat[0];
#pragma unroll
    for (int u = 1; u < W; ++u)
        mg = fmaxf(mg, stat[u]);
    float sc[W], ls = 0.0f;
#pragma unroll
    for (int u = 0; u < W; ++u) {
        sc[u] = expf(stat[u] - mg);  // 0 for a wave without sources
        ls = fmaf(sc[u], stat[W + u], ls);
    }
    const float inv = 1.0f / ls;
    for (int j = (wave * kWaveSize + lane) * 4; j < kRow && col0 + j < d; j += W * kWaveSize * 4) {
        f32x4_t y = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int u = 0; u < W; ++u) {
            const f32x4_t x = *reinterpret_cast<const f32x4_t *>(part + u * kRow + j);
            y.x = fmaf(sc[u], x.x, y.x);
            y.y = fmaf(sc[u], x.y, y.y);
            y.z = fmaf(sc[u], x.z, y.z);
            y.w = fmaf(sc[u], x.w, y.w);
        }
        const float h[4] = {y.x * inv, y.y * inv, y.z * inv, y.w * inv};
        if (d % 4 == 0) {
            store_raw<T, 4>(hrow + col0 + j, Narrow<T, 4>::run(h));
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (col0 + j + e < d)
                    store_elem(hrow + col0 + j + e, h[e]);
        }
    }
}

// acc += a * the unit's values.
template <int FMT>
__device__ __forceinline__ void add_unit(const UnitRaw<FMT> &w, float a, float (&acc)[UnitRaw<FMT>::cols])
{
#pragma unroll
    for (int h = 0; h < unit_cols<FMT>() / 16; ++h) {
        float x[16];
        unit_values<FMT>(w, h, x);
#pragma unroll
        for (int e = 0; e < 16; ++e)
            acc[16 * h + e] = fmaf(a, x[e], acc[16 * h + e]);
    }
}

}  // namespace

// Projected / sliced keys.  A wave owns the adjacent tokens of 64 / LG groups of
// lanes, TW of them a group, whose rows are adjacent in every plane, and loads SB
// sources of them a trip.  Long runs of adjacent rows read best: tokens x sources a
// trip at the size above, H's allocation included: 1 x 4 418 us, 2 x 1 391, 4 x 2
// 387, 4 x 1 370.  Grid x = tokens, y = column blocks of NCH * LG units (each
// recomputes the cheap scores).
template <int FMT, typename T, int LG, int NCH, bool SLICED, int TW, int SB>
__global__ void __launch_bounds__(kBlock)
cache_fwd_lr(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales,
             const void *__restrict__ K, const float *__restrict__ q, T *__restrict__ H, int S,
             int N, int d, int r, float eps, int s_pad)
{
    constexpr int G = kWaveSize / LG, CW = unit_cols<FMT>();
    constexpr int per = kCacheBlock / CW;  // units a block
    extern __shared__ float lds[];
    const int lane = threadIdx.x & (kWaveSize - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWaveSize);
    const BlockXY bk = xcd_block();
    const int n0 = (bk.x * kWaves + wave) * G * TW;
    if (n0 >= N)
        return;  // wave-uniform; this kernel has no workgroup barrier
    float *s = lds + wave * G * TW * s_pad;
    const Lanes<FMT, LG, NCH> ln(lane, d);
    const int c0 = bk.y * NCH * LG;  // first unit of the column block
    unsigned at[TW][NCH];
#pragma unroll
    for (int t = 0; t < TW; ++t)
#pragma unroll
        for (int c = 0; c < NCH; ++c)
            at[t][c] = (unsigned)((min(n0 + t * G + ln.g, N - 1) - n0) * ln.nu +
                                  min(c0 + ln.lu + c * LG, ln.nu - 1));
    const size_t first = (size_t)n0 * ln.nu, plane = (size_t)N * ln.nu;
    typedef UnitRaw<FMT> Trip[SB][TW][NCH];
    Trip w;
    auto load = [&](Trip &w, int i0) {
#pragma unroll
        for (int u = 0; u < SB; ++u) {
            const size_t b = min(i0 + u, S - 1) * plane + first;
#pragma unroll
            for (int t = 0; t < TW; ++t)
#pragma unroll
                for (int c = 0; c < NCH; ++c)
                    load_unit<FMT>(codes + b * 16, scales + b / per, at[t][c], w[u][t][c]);
        }
    };
    load(w, 0);  // does not depend on the scores: goes out before the keys' loads
    cache_scores<FMT, T, SLICED, G * TW, G * TW <= 2 ? 4 : G * TW <= 4 ? 2 : 1>(
        Keys<FMT, T, SLICED>(K, codes, scales, N, d, r), q, 0, S, n0, eps, lane, s, nullptr, s_pad);
    wave_lds_sync();
#pragma unroll
    for (int t = 0; t < TW; ++t)
        group_softmax<LG>(s + t * G * s_pad, s + t * G * s_pad, s_pad, S, ln.g, ln.lu);
    wave_lds_sync();
    float acc[TW][NCH][CW];
#pragma unroll
    for (int t = 0; t < TW; ++t)
#pragma unroll
        for (int c = 0; c < NCH; ++c)
#pragma unroll
            for (int e = 0; e < CW; ++e)
                acc[t][c][e] = 0.0f;
    auto add = [&](const Trip &w, int i0) {
#pragma unroll
        for (int u = 0; u < SB; ++u)
#pragma unroll
            for (int t = 0; t < TW; ++t) {
                const float a = i0 + u < S ? s[(t * G + ln.g) * s_pad + min(i0 + u, S - 1)] : 0.0f;
#pragma unroll
                for (int c = 0; c < NCH; ++c)
                    add_unit<FMT>(w[u][t][c], a, acc[t][c]);
            }
    };
    // A wave of several tokens a group has loads enough in flight, and rows of more
    // units no registers for a second buffer (e4m3, 20 x 3000 x 4000: 46 us, with it 55).
    if constexpr (TW == 1 && NCH == 1) {
        pipelined(0, S, SB, w, load, add);
    } else {
        for (int i0 = 0; i0 < S; i0 += SB) {
            if (i0 > 0)
                load(w, i0);
            __builtin_amdgcn_sched_barrier(0);
            add(w, i0);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
#pragma unroll
    for (int t = 0; t < TW; ++t) {
        const int n = n0 + t * G + ln.g;
        if (n < N)
            store_h<FMT, T, LG, NCH>(H + (size_t)n * d, ln, c0 * CW, d, acc[t]);
    }
}

// The same for few tokens: one token a workgroup of W waves, its sources cut into
// W ranges, whose online-softmax states meet in LDS.  The groups of a wave take
// every G-th source of its range, U of them in flight a lane: what bounds a
// launch of few tokens is the chain of dependent loads.
// o_new: the newest source of every token (or NULL): the wave whose range ends with
// source S-1 quantises it from there, stores it into plane S-1 and reads it back with
// the others.  (That plane is written here and read again: no restrict.)
template <int FMT, typename T, int LG, int NCH, bool SLICED, int W>
__global__ void __launch_bounds__(W * kWaveSize)
cache_fwd_lr_wg(uint8_t *codes, uint8_t *scales, const void *__restrict__ K,
                const float *__restrict__ q, const T *__restrict__ o_new, T *__restrict__ H, int S,
                int N, int d, int r, float eps, int s_pad)
{
    constexpr int G = kWaveSize / LG, CW = unit_cols<FMT>();
    constexpr int per_block = kCacheBlock / CW;
    constexpr int U = NCH >= 4 ? 2 : NCH == 2 ? 4 : 8;
    extern __shared__ float lds[];
    const int lane = threadIdx.x & (kWaveSize - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWaveSize);
    const BlockXY bk = xcd_block();
    const int n = bk.x;
    const int per = (S + W - 1) / W;
    const int ib = min(S, wave * per), ie = min(S, ib + per);
    float *stat = lds;
    float *part = lds + 2 * W;
    float *s = part + W * NCH * LG * CW + wave * s_pad - ib;  // s[ib .. ie - 1]
    const Lanes<FMT, LG, NCH> ln(lane, d);
    const int c0 = bk.y * NCH * LG;  // first unit of the column block
    const size_t first = (size_t)n * ln.nu, plane = (size_t)N * ln.nu;
    float acc[NCH][CW];
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < CW; ++e)
            acc[c][e] = 0.0f;
    float m = -INFINITY, l = 0.0f;
    if (ib < ie) {  // wave-uniform
        UnitRaw<FMT> w[U][NCH];
        constexpr int B = U < 4 ? U : 4;  // sources a group that are skipped together
        auto load = [&](int i0) {
#pragma unroll
            for (int h = 0; h < U; h += B)
                if (h == 0 || i0 + h * G < ie)  // wave-uniform
#pragma unroll
                    for (int u = h; u < h + B; ++u) {
                        const size_t b = min(i0 + u * G + ln.g, ie - 1) * plane + first;
#pragma unroll
                        for (int c = 0; c < NCH; ++c)
                            load_unit<FMT>(codes + b * 16, scales + b / per_block,
                                           (unsigned)min(c0 + ln.lu + c * LG, ln.nu - 1), w[u][c]);
                    }
        };
        if (o_new && ie == S) {
            // Group 0 stores the row; the loads below read it back.
            if (ln.g == 0) {
                const size_t b = (size_t)(S - 1) * plane + first;
#pragma unroll
                for (int c = 0; c < NCH; ++c) {
                    const int unit = c0 + ln.lu + c * LG;
                    float x[CW];
#pragma unroll
                    for (int h = 0; h < CW / 8; ++h) {
                        float y[8];
                        load8(o_new + (size_t)n * d, unit * CW + 8 * h, d, y);
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            x[8 * h + e] = y[e];
                    }
                    UnitRaw<FMT> z;
                    encode_unit<FMT>(x, z);
                    if (unit < ln.nu)
                        store_unit<FMT>(codes + b * 16, scales + b / per_block, (unsigned)unit, z);
                }
            }
            __threadfence_block();
        }
        load(ib);  // does not depend on the scores: goes out before the keys' loads
        cache_scores<FMT, T, SLICED, 1, 4>(Keys<FMT, T, SLICED>(K, codes, scales, N, d, r), q, ib,
                                           ie, n, eps, lane, s, nullptr, s_pad);
        wave_lds_sync();
        for (int i = ib + lane; i < ie; i += kWaveSize)
            m = fmaxf(m, s[i]);
        m = group_max(m, kWaveSize);
        for (int i = ib + lane; i < ie; i += kWaveSize) {
            // (A range may hold no score above -inf, and then weighs nothing beside the
            // others; NaN stays NaN.)
            const float e = s[i] == -INFINITY ? 0.0f : expf(s[i] - m);
            s[i] = e;
            l += e;
        }
        l = group_sum(l, kWaveSize);
        wave_lds_sync();
        for (int i0 = ib; i0 < ie; i0 += U * G) {
            if (i0 > ib)
                load(i0);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (u > 0 && u % B == 0 && i0 + u * G >= ie)
                    break;
                const int i = i0 + u * G + ln.g;
                const float a = i < ie ? s[min(i, ie - 1)] : 0.0f;
#pragma unroll
                for (int c = 0; c < NCH; ++c)
                    add_unit<FMT>(w[u][c], a, acc[c]);
            }
        }
    }
    merge_store<FMT, T, LG, NCH, W>(acc, ln, m, l, stat, part, H + (size_t)n * d, c0 * CW, d, wave,
                                    lane);
}

// Full-rank keys: each group scores a batch of four sources from the codes in
// registers, and they join its online softmax; the four scores are formed by
// four lanes at once.  W = 0: every group its own token, kWaves waves a
// workgroup.  Else a workgroup of W waves has one token, whose sources its groups
// share; o_new as in cache_fwd_lr_wg.
template <int FMT, typename T, int LG, int NCH, int W>
__global__ void __launch_bounds__(W == 0 ? kBlock : W * kWaveSize)
cache_fwd_full(uint8_t *codes, uint8_t *scales, const float *__restrict__ q,
               const T *__restrict__ o_new, T *__restrict__ H, int S, int N, int d, float eps)
{
    constexpr int G = kWaveSize / LG, CW = unit_cols<FMT>();
    constexpr int per_block = kCacheBlock / CW;
    extern __shared__ float lds[];
    const int lane = threadIdx.x & (kWaveSize - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWaveSize);
    const int bx = xcd_block().x;
    const int n0 = W == 0 ? (bx * kWaves + wave) * G : bx;
    if (W == 0 && n0 >= N)
        return;  // wave-uniform; no workgroup barrier on this path
    const Lanes<FMT, LG, NCH> ln(lane, d);
    const int n = W == 0 ? min(n0 + ln.g, N - 1) : n0;
    const int per = W == 0 ? S : (S + W - 1) / W;
    const int ib = W == 0 ? 0 : min(S, wave * per), ie = min(S, ib + per);
    constexpr int step = W == 0 ? 1 : G;  // from a group's source to its next
    const int i1 = W == 0 ? 0 : ln.g;     // a group's first source
    const size_t first = (size_t)n0 * ln.nu, plane = (size_t)N * ln.nu;
    unsigned at[NCH];
    float qv[NCH][CW], acc[NCH][CW];
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        at[c] = ln.at[c] + (unsigned)((n - n0) * ln.nu);
#pragma unroll
        for (int e = 0; e < CW; ++e) {
            const int j = ln.col(c) + e;
            qv[c][e] = j < d ? q[j] : 0.0f;
            acc[c][e] = 0.0f;
        }
    }
    if (W != 0 && o_new && ie == S && ib < ie) {
        if (ln.g == 0) {
            const size_t b = (size_t)(S - 1) * plane + first;
#pragma unroll
            for (int c = 0; c < NCH; ++c) {
                float x[CW];
#pragma unroll
                for (int h = 0; h < CW / 8; ++h) {
                    float y[8];
                    load8(o_new + (size_t)n * d, ln.col(c) + 8 * h, d, y);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        x[8 * h + e] = y[e];
                }
                UnitRaw<FMT> z;
                encode_unit<FMT>(x, z);
                if (ln.in[c])
                    store_unit<FMT>(codes + b * 16, scales + b / per_block, ln.at[c], z);
            }
        }
        __threadfence_block();
    }
    const float inv_d = 1.0f / (float)d;
    float m = -INFINITY, l = 0.0f;
    typedef UnitRaw<FMT> Trip[4][NCH];
    auto load = [&](Trip &w, int i0) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const size_t b = min(i0 + u * step + i1, ie - 1) * plane + first;
#pragma unroll
            for (int c = 0; c < NCH; ++c)
                load_unit<FMT>(codes + b * 16, scales + b / per_block, at[c], w[u][c]);
        }
    };
    auto add = [&](const Trip &w, int i0) {
        float ss[4], dot[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            ss[u] = dot[u] = 0.0f;
#pragma unroll
            for (int c = 0; c < NCH; ++c) {
                float a = 0.0f;
#pragma unroll
                for (int h = 0; h < CW / 16; ++h) {
                    float x[16];
                    unit_values<FMT>(w[u][c], h, x);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        a = fmaf(x[e], x[e], a);
                        dot[u] = fmaf(qv[c][16 * h + e], x[e], dot[u]);
                    }
                }
                ss[u] += ln.in[c] ? a : 0.0f;
            }
        }
        const float tss = four_sums<LG>(ss, lane), tdot = four_sums<LG>(dot, lane);
        float sc = tdot * rsqrtf(tss * inv_d + eps);  // of source four_index(lane)
        if (i0 + four_index<LG>(lane) * step + i1 >= ie)
            sc = -INFINITY;
        float mb = m;
#pragma unroll
        for (int u = 0; u < 4; ++u)
            mb = fmaxf(mb, four_value<LG>(sc, lane, u));
        if (mb > m) {
            const float scale = expf(m - mb);
            l *= scale;
#pragma unroll
            for (int c = 0; c < NCH; ++c)
#pragma unroll
                for (int e = 0; e < CW; ++e)
                    acc[c][e] *= scale;
            m = mb;
        }
        // A group that has no source in the batch adds nothing (m may be -inf).
        const float wt = sc == -INFINITY ? 0.0f : expf(sc - m);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float a = four_value<LG>(wt, lane, u);
            l += a;
#pragma unroll
            for (int c = 0; c < NCH; ++c)
                add_unit<FMT>(w[u][c], a, acc[c]);
        }
    };
    if constexpr (NCH == 1) {  // (more units: no registers for a second buffer)
        if (ib < ie) {  // wave-uniform
            Trip w;
            load(w, ib);
            pipelined(ib, ie, 4 * step, w, load, add);
        }
    } else {
        for (int i0 = ib; i0 < ie; i0 += 4 * step) {
            Trip w;
            load(w, i0);
            __builtin_amdgcn_sched_barrier(0);
            add(w, i0);
        }
    }
    if constexpr (W != 0) {
        if constexpr (G > 1) {  // the groups' states on one maximum
            float mw = m;
#pragma unroll
            for (int x = LG; x < kWaveSize; x <<= 1)
                mw = fmaxf(mw, __shfl_xor(mw, x, kWaveSize));
            const float scale = m == -INFINITY ? 0.0f : expf(m - mw);
            l *= scale;
#pragma unroll
            for (int c = 0; c < NCH; ++c)
#pragma unroll
                for (int e = 0; e < CW; ++e)
                    acc[c][e] *= scale;
#pragma unroll
            for (int x = LG; x < kWaveSize; x <<= 1)
                l += __shfl_xor(l, x, kWaveSize);
            m = mw;
        }
        merge_store<FMT, T, LG, NCH, W>(acc, ln, m, l, lds, lds + 2 * W, H + (size_t)n * d, 0, d, wave,
                                        lane);
    } else {
        const float inv = 1.0f / l;
#pragma unroll
        for (int c = 0; c < NCH; ++c)
#pragma unroll
            for (int e = 0; e < CW; ++e)
                acc[c][e] *= inv;
        if (n0 + ln.g < N)
            store_h<FMT, T, LG, NCH>(H + (size_t)n * d, ln, 0, d, acc);
    }
}

namespace {

constexpr int64_t kMaxSourcesFwd = 1024, kMaxSourcesBwd = 512, kMaxRankBwd = 256;
constexpr int64_t kMaxRow = 4096;            // columns that a wave holds
constexpr int64_t kMaxColumns = 1 << 20;     // of a row in column blocks

// Tokens up to which a token's sources are split over a workgroup: one number for all
// widths, at which wide rows are about level; rows of few columns, several tokens of
// which share a wave, would gain from more.  Split / one wave a token, 1024 tokens:
// e4m3, 64 sources, d = 2048 24.6 / 26.6 us, 49 sources, d = 1024 13.3 / 12.0; e2m1, 33
// sources, d = 500 10.6 / 17.1, d = 1024 11.5 / 11.8, at 1500 tokens 15.9 / 12.5.  Full
// rank: e2m1, 49 sources, d = 1024: 512 tokens 14.1 / 22.4, 700 tokens 19.9 / 22.6, 850
// tokens 23.8 / 22.7; e4m3, 33 sources, d = 2048: 700 tokens 25.0 / 23.0.
constexpr int64_t kSplitTokens = 1024, kSplitFull = 768;

// Waves from which a wave of the low-rank forward takes several tokens a group
// (two a SIMD; their chain of trips is four times as long), and the sources up to
// which their scores fit LDS.  One token / four: e4m3, 49 sources, d = 1024: 4099
// tokens 40 / 54 us, 8192 tokens 75 / 70; 64 sources, d = 2048: 8192 tokens 192 / 175;
// e2m1, 33 sources, d = 1024 (two tokens / eight a wave): 8192 tokens 36 / 53, 16384
// tokens 69 / 69; 64 sources, d = 2048: 9000 tokens 123 / 163, 16384 tokens 244 / 220.
constexpr int64_t kManyWaves = 2048, kManySources = 128;

bool split_tokens(const CacheProblem &p)
{
    return p.N <= (p.mode == LRAR_MODE_FULL ? kSplitFull : kSplitTokens) && p.S > 1;
}

template <int FMT, typename T>
hipError_t launch_fwd_as(const CacheProblem &p, const void *o_new, void *H, hipStream_t st)
{
    T *h = static_cast<T *>(H);
    const T *o = static_cast<const T *>(o_new);
    uint8_t *codes = const_cast<uint8_t *>(p.codes), *scales = const_cast<uint8_t *>(p.scales);
    const int S = (int)p.S, N = (int)p.N, d = (int)p.d, r = (int)p.r;
    constexpr int W = kWaves;
    const bool split = split_tokens(p);
    return dispatch_lanes<FMT>(p.d, [&](auto lg, auto nc) -> hipError_t {
        constexpr int LG = decltype(lg)::value, NCH = decltype(nc)::value;
        constexpr int G = kWaveSize / LG, cols = NCH * LG * unit_cols<FMT>();
        const unsigned gy = (unsigned)((d + cols - 1) / cols);
        const size_t meet = (2 * W + W * cols) * sizeof(float);
        if (p.mode == LRAR_MODE_FULL) {
            if (split)
                hipLaunchKernelGGL((cache_fwd_full<FMT, T, LG, NCH, W>), dim3((unsigned)N),
                                   dim3(kBlock), meet, st, codes, scales, p.q, o, h, S, N, d, p.eps);
            else
                hipLaunchKernelGGL((cache_fwd_full<FMT, T, LG, NCH, 0>),
                                   dim3((unsigned)((N + kWaves * G - 1) / (kWaves * G))),
                                   dim3(kBlock), 0, st, codes, scales, p.q, o, h, S, N, d, p.eps);
            return hipGetLastError();
        }
        auto launch = [&](auto sliced) {
            constexpr bool SL = decltype(sliced)::value;
            if (split) {
                const int s_pad = (S + W - 1) / W;
                hipLaunchKernelGGL((cache_fwd_lr_wg<FMT, T, LG, NCH, SL, W>), dim3((unsigned)N, gy),
                                   dim3(kBlock), meet + W * s_pad * sizeof(float), st, codes,
                                   scales, p.K, p.q, o, h, S, N, d, r, p.eps, s_pad);
            } else {
                auto many = [&](auto tw, auto sb) {
                    constexpr int TW = decltype(tw)::value, SB = decltype(sb)::value;
                    const int tokens = kWaves * G * TW;
                    hipLaunchKernelGGL((cache_fwd_lr<FMT, T, LG, NCH, SL, TW, SB>),
                                       dim3((unsigned)((N + tokens - 1) / tokens), gy), dim3(kBlock),
                                       tokens * S * sizeof(float), st, codes, scales, p.K, p.q, h,
                                       S, N, d, r, p.eps, S);
                };
                constexpr int TWB = LG == 16 || cols > 2048 ? 2 : 4;  // (cols: registers)
                if (N >= kManyWaves * G * TWB && S <= kManySources)
                    many(std::integral_constant<int, TWB>{}, std::integral_constant<int, LG == 16 ? 2 : 1>{});
                else
                    many(std::integral_constant<int, 1>{}, std::integral_constant<int, 4>{});
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
    if (p.N > (1 << 25)) {  // a launch's threads
        *why = "N exceeds 2^25 tokens";
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
    // Sliced keys of a row in several column blocks read what another block writes.
    const bool fused = o_new && split_tokens(p) && p.d <= kMaxRow;
    if (o_new && !fused) {
        const int64_t first = (p.S - 1) * p.N;
        const int rc = launch_cache_write(
            o_new, const_cast<uint8_t *>(p.codes) + first * cache_row_bytes(p.d, p.format),
            const_cast<uint8_t *>(p.scales) + first * cache_blocks(p.d), p.N, p.d, p.format,
            p.dtype, st, err);
        if (rc)
            return rc;
        o_new = nullptr;
    }
    hipError_t e;
    if (p.dtype == LRAR_DTYPE_BF16)
        e = p.format == LRAR_CACHE_FP8 ? launch_fwd_as<LRAR_CACHE_FP8, uint16_t>(p, o_new, H, st)
                                       : launch_fwd_as<LRAR_CACHE_FP4, uint16_t>(p, o_new, H, st);
    else
        e = p.format == LRAR_CACHE_FP8 ? launch_fwd_as<LRAR_CACHE_FP8, float>(p, o_new, H, st)
                                       : launch_fwd_as<LRAR_CACHE_FP4, float>(p, o_new, H, st);
    return hip_status(e, "cache_route_fwd launch", err);
}

}  // namespace lrar

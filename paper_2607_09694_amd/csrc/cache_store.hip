// Quantising rows into the 8- or 4-bit source stack and reading them back.  Both are
// bound by their bytes: reading 49 x 2048 rows of 1024 columns back from e4m3 to bf16
// takes 45 us (311 MB, 6.9 TB/s), writing 12289 rows of 2000 columns as e2m1 11 us
// (60 MB).
#include "cache_device.h"

#include <algorithm>

namespace lrar {

// Both kernels walk the rows in slots of 8 columns, four lanes to a block of 32
// columns: one 16-byte access of bf16 (two of fp32), 8 or 4 bytes of codes, and
// for the write the block's maximum over four lanes by two register moves.  A
// workgroup takes `rpb` whole rows, whose slots are contiguous in the codes;
// magic = ceil(2^32 / slots a row) turns a slot of the workgroup (at most
// kSlotsPerBlock, or one row) into its row without a division.
struct RowSlots {
    int slots, rpb;
    unsigned magic;
};

template <int FMT, typename T>
__global__ void __launch_bounds__(kBlock)
cache_write(const T *__restrict__ O, uint8_t *__restrict__ codes, uint8_t *__restrict__ scales,
            int64_t rows, int d, RowSlots rs)
{
    typedef typename Codes<FMT>::key_t key_t;
    for (int64_t r0 = (int64_t)blockIdx.x * rs.rpb; r0 < rows; r0 += (int64_t)gridDim.x * rs.rpb) {
        const int n = (int)min((int64_t)rs.rpb, rows - r0) * rs.slots;
        key_t *crow = reinterpret_cast<key_t *>(codes) + r0 * rs.slots;
        uint8_t *erow = scales + r0 * (rs.slots / 4);
        // n is a multiple of 4, and so is every stride: the four lanes of a block
        // are in or out together.
        for (int s = threadIdx.x; s < n; s += kBlock) {
            const int rl = rs.rpb == 1 ? 0 : (int)__umulhi((unsigned)s, rs.magic);
            const int col = (s - rl * rs.slots) * 8;
            float x[8];
            load8(O + (r0 + rl) * d, col, d, x);
            float top = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                top = max_magnitude(top, x[e]);
            top = max_magnitude(top, dpp_move<kDppXor1>(top));
            top = max_magnitude(top, dpp_move<kDppXor2>(top));
            const unsigned e = scale_byte<FMT>(top);
            crow[s] = encode<FMT>(x, e);
            if ((s & 3) == 0)
                erow[s >> 2] = (uint8_t)e;
        }
    }
}

template <int FMT, typename T>
__global__ void __launch_bounds__(kBlock)
cache_read(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales,
           T *__restrict__ O, int64_t rows, int d, RowSlots rs)
{
    typedef typename Codes<FMT>::key_t key_t;
    for (int64_t r0 = (int64_t)blockIdx.x * rs.rpb; r0 < rows; r0 += (int64_t)gridDim.x * rs.rpb) {
        const int n = (int)min((int64_t)rs.rpb, rows - r0) * rs.slots;
        const key_t *crow = reinterpret_cast<const key_t *>(codes) + r0 * rs.slots;
        const uint8_t *erow = scales + r0 * (rs.slots / 4);
        for (int s = threadIdx.x; s < n; s += kBlock) {
            const int rl = rs.rpb == 1 ? 0 : (int)__umulhi((unsigned)s, rs.magic);
            const int col = (s - rl * rs.slots) * 8;
            float x[8];
            decode<FMT>(crow[s], block_scale(erow[s >> 2]), x);
            store8<T, true>(O + (r0 + rl) * d, col, d, x);
        }
    }
}

namespace {

// Slots a workgroup, about: rows of few columns share one.
constexpr int kSlotsPerBlock = 1024;

RowSlots row_slots(int64_t rows, int64_t d, int64_t *nblocks)
{
    RowSlots rs;
    rs.slots = (int)cache_blocks(d) * 4;
    rs.rpb = rs.slots >= kSlotsPerBlock ? 1 : kSlotsPerBlock / rs.slots;
    rs.magic = (unsigned)((((uint64_t)1 << 32) + rs.slots - 1) / rs.slots);
    *nblocks = (rows + rs.rpb - 1) / rs.rpb;
    return rs;
}

constexpr int64_t kMaxBlocks = (int64_t)1 << 31;   // of rows.rpb rows; refused from here on
constexpr int64_t kGridBlocks = (int64_t)1 << 20;  // launched; they walk the rest

template <typename F> hipError_t by_format(int format, int dtype, F &&f)
{
    constexpr auto e8 = std::integral_constant<int, LRAR_CACHE_FP8>{};
    constexpr auto e4 = std::integral_constant<int, LRAR_CACHE_FP4>{};
    if (dtype == LRAR_DTYPE_BF16)
        return format == LRAR_CACHE_FP8 ? f(e8, uint16_t{}) : f(e4, uint16_t{});
    return format == LRAR_CACHE_FP8 ? f(e8, float{}) : f(e4, float{});
}

}  // namespace

int launch_cache_write(const void *O, uint8_t *codes, uint8_t *scales, int64_t rows, int64_t d,
                       int format, int dtype, hipStream_t st, std::string *err)
{
    if (rows == 0)
        return LRAR_OK;
    int64_t nb;
    const RowSlots rs = row_slots(rows, d, &nb);
    if (nb >= kMaxBlocks) {
        *err = "too many rows for one launch";
        return LRAR_EUNSUPPORTED;
    }
    const hipError_t e = by_format(format, dtype, [&](auto fmt, auto t) -> hipError_t {
        typedef decltype(t) T;
        hipLaunchKernelGGL((cache_write<decltype(fmt)::value, T>), dim3((unsigned)std::min(nb, kGridBlocks)),
                           dim3(kBlock), 0, st, static_cast<const T *>(O), codes, scales, rows,
                           (int)d, rs);
        return hipGetLastError();
    });
    return hip_status(e, "cache_write launch", err);
}

int launch_cache_read(const uint8_t *codes, const uint8_t *scales, void *O, int64_t rows,
                      int64_t d, int format, int dtype, hipStream_t st, std::string *err)
{
    if (rows == 0)
        return LRAR_OK;
    int64_t nb;
    const RowSlots rs = row_slots(rows, d, &nb);
    if (nb >= kMaxBlocks) {
        *err = "too many rows for one launch";
        return LRAR_EUNSUPPORTED;
    }
    const hipError_t e = by_format(format, dtype, [&](auto fmt, auto t) -> hipError_t {
        typedef decltype(t) T;
        hipLaunchKernelGGL((cache_read<decltype(fmt)::value, T>), dim3((unsigned)std::min(nb, kGridBlocks)),
                           dim3(kBlock), 0, st, codes, scales, static_cast<T *>(O), rows, (int)d,
                           rs);
        return hipGetLastError();
    });
    return hip_status(e, "cache_read launch", err);
}

}  // namespace lrar

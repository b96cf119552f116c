// The paged 4-bit cache of keys and values: sq_cache_append quantizes new rows into their pages, sq_cache_read gives rows
// back as fp16.
#include "sq_cache.h"
#include "sq_quant4.h"

namespace sq {

namespace {

// Where a new row lives: its page (nullptr: none) and its slot in it.
__device__ __forceinline__ uint8_t *place_of_row(const CacheView &c, int64_t row, int &slot)
{
    const int b = sequence_of_row(c.row_start, c.B, row);
    if (b < 0) return nullptr;
    const int64_t at = (int64_t)c.cached[b] + (row - c.row_start[b]);
    if (c.cached[b] < 0 || at >= ((int64_t)c.per_sequence << c.page_shift)) return nullptr;
    slot = (int)at & ((1 << c.page_shift) - 1);
    const int number = cache_page(c, b, (int)(at >> c.page_shift));
    return number < 0 ? nullptr : c.base + (int64_t)number * c.page_bytes;
}

// One workgroup per row; a lane takes eight channels of a head of K or V, D / 8 neighbouring lanes a head.  Every wave
// finds the row's place by itself (two dependent loads and the table's), which is what a decode step's few rows cost.
template <int D>
__global__ __launch_bounds__(256) void cache_append_kernel(const CacheView c, const __half *__restrict__ K, int64_t ldk,
                                                           const __half *__restrict__ V, int64_t ldv)
{
    constexpr int LANES = D / 8;
    const int64_t row = blockIdx.x;
    int slot;
    uint8_t *page = place_of_row(c, row, slot);
    if (!page) return;
    const int rows_of_page = 1 << c.page_shift, half_codes = rows_of_page * (D / 2);
    __half *steps = reinterpret_cast<__half *>(page + cache_steps_at(c.Hk, D, rows_of_page));
    const int units = 2 * c.Hk * LANES;
    for (int u0 = 0; u0 < units; u0 += 256) {
        const int u = u0 + (int)threadIdx.x, unit = min(u, units - 1);         // whole waves: the maxima need every lane
        const int head = unit / LANES, piece = unit % LANES;
        const bool is_v = head >= c.Hk;
        const int h = is_v ? head - c.Hk : head;
        const __half *src = is_v ? V + row * ldv : K + row * ldk;
        const uint4 x = *reinterpret_cast<const uint4 *>(src + h * D + 8 * piece);
        const __half s = run_step(run_max<LANES>(x));
        const uint32_t codes = run_codes_plus8(x, __builtin_amdgcn_rcpf(__half2float(s)));
        if (u >= units) continue;
        uint8_t *dst = page + (int64_t)h * (2 * half_codes);
        if (!is_v) {
            *reinterpret_cast<uint32_t *>(dst + slot * (D / 2) + 4 * piece) = codes;
        } else {
            dst += half_codes;
            if constexpr (D == 64) {                                           // two units of two bytes
                *reinterpret_cast<uint16_t *>(dst + cache_v_unit<D>(slot, 2 * piece)) = (uint16_t)codes;
                *reinterpret_cast<uint16_t *>(dst + cache_v_unit<D>(slot, 2 * piece + 1)) = (uint16_t)(codes >> 16);
            } else if constexpr (D == 128) {
                *reinterpret_cast<uint32_t *>(dst + cache_v_unit<D>(slot, piece)) = codes;
            } else {                                                           // half a unit of eight bytes
                *reinterpret_cast<uint32_t *>(dst + cache_v_unit<D>(slot, piece / 2) + 4 * (piece & 1)) = codes;
            }
        }
        if (piece == 0) steps[(is_v ? c.Hk * rows_of_page : 0) + h * rows_of_page + slot] = s;
    }
}

template <int D>
__global__ __launch_bounds__(256) void cache_read_kernel(const CacheView c, __half *__restrict__ K, int64_t ldk,
                                                         __half *__restrict__ V, int64_t ldv)
{
    constexpr int LANES = D / 8;
    const int64_t row = blockIdx.x;
    int slot;
    const uint8_t *page = place_of_row(c, row, slot);
    if (!page) return;
    const int rows_of_page = 1 << c.page_shift, half_codes = rows_of_page * (D / 2);
    const __half *steps = reinterpret_cast<const __half *>(page + cache_steps_at(c.Hk, D, rows_of_page));
    const int units = 2 * c.Hk * LANES;
    for (int unit = (int)threadIdx.x; unit < units; unit += 256) {
        const int head = unit / LANES, piece = unit % LANES;
        const bool is_v = head >= c.Hk;
        const int h = is_v ? head - c.Hk : head;
        const uint8_t *src = page + (int64_t)h * (2 * half_codes);
        uint32_t codes;
        if (!is_v) {
            codes = *reinterpret_cast<const uint32_t *>(src + slot * (D / 2) + 4 * piece);
        } else {
            src += half_codes;
            if constexpr (D == 64)
                codes = *reinterpret_cast<const uint16_t *>(src + cache_v_unit<D>(slot, 2 * piece)) |
                        ((uint32_t) * reinterpret_cast<const uint16_t *>(src + cache_v_unit<D>(slot, 2 * piece + 1)) << 16);
            else if constexpr (D == 128)
                codes = *reinterpret_cast<const uint32_t *>(src + cache_v_unit<D>(slot, piece));
            else
                codes = *reinterpret_cast<const uint32_t *>(src + cache_v_unit<D>(slot, piece / 2) + 4 * (piece & 1));
        }
        const float s = __half2float(steps[(is_v ? c.Hk * rows_of_page : 0) + h * rows_of_page + slot]);
        uint4 out;
        uint32_t *w = &out.x;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            // code * step: 15 bits, rounded once to fp16
            const v2h p = {(_Float16)((float)((int)((codes >> (8 * e)) & 15) - 8) * s),
                           (_Float16)((float)((int)((codes >> (8 * e + 4)) & 15) - 8) * s)};
            w[e] = __builtin_bit_cast(uint32_t, p);
        }
        *reinterpret_cast<uint4 *>((is_v ? V + row * ldv : K + row * ldk) + h * D + 8 * piece) = out;
    }
}

sq_status check_rows(const void *K, int64_t ldk, const void *V, int64_t ldv, int64_t T, int32_t Hk, int32_t D,
                     const int32_t *row_start, const int32_t *cached, int32_t B, const int32_t *table, int32_t per_sequence,
                     int32_t page, const void *cache, int32_t pages)
{
    const sq_status s = check_cache(Hk, D, page, B, per_sequence, pages);
    if (s != SQ_OK) return s;
    if (T < 0 || T > SQ_MAX_ROWS || ldk < (int64_t)Hk * D || ldv < (int64_t)Hk * D) return SQ_ERR_SHAPE;
    if (T == 0 || B == 0 || per_sequence == 0 || pages == 0) return SQ_OK;
    if (!K || !V || !row_start || !cached || !table || !cache) return SQ_ERR_NULL;
    if (((uintptr_t)K & 15) || ((uintptr_t)V & 15) || (ldk % 8) != 0 || (ldv % 8) != 0 || ((uintptr_t)cache & 15) ||
        (((uintptr_t)row_start | (uintptr_t)cached | (uintptr_t)table) & 3))
        return SQ_ERR_ALIGN;
    return SQ_OK;
}

}  // namespace

}  // namespace sq

extern "C" int64_t sq_cache_page_bytes(int32_t Hk, int32_t D, int32_t page)
{
    if (sq::check_cache(Hk, D, page, 0, 0, 0) != SQ_OK) return 0;
    return ((int64_t)Hk * page * (D + 4) + 255) / 256 * 256;
}

extern "C" sq_status sq_cache_append(const void *K, int64_t ldk, const void *V, int64_t ldv, int64_t T, int32_t Hk, int32_t D,
                                     const int32_t *row_start, const int32_t *cached, int32_t B, const int32_t *table,
                                     int32_t per_sequence, int32_t page, void *cache, int32_t pages, void *stream)
{
    const sq_status s = sq::check_rows(K, ldk, V, ldv, T, Hk, D, row_start, cached, B, table, per_sequence, page, cache, pages);
    if (s != SQ_OK || T == 0 || B == 0 || per_sequence == 0 || pages == 0) return s;
    const sq::CacheView c = sq::cache_view(cache, pages, Hk, D, page, table, per_sequence, row_start, cached, B);
    auto kernel = D == 64 ? sq::cache_append_kernel<64> : D == 128 ? sq::cache_append_kernel<128> : sq::cache_append_kernel<256>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)T), dim3(256), 0, static_cast<hipStream_t>(stream), c,
                       static_cast<const __half *>(K), ldk, static_cast<const __half *>(V), ldv);
    return hipGetLastError() == hipSuccess ? SQ_OK : SQ_ERR_LAUNCH;
}

extern "C" sq_status sq_cache_read(const void *cache, int32_t pages, int32_t Hk, int32_t D, const int32_t *row_start,
                                   const int32_t *cached, int32_t B, const int32_t *table, int32_t per_sequence, int32_t page,
                                   void *K, int64_t ldk, void *V, int64_t ldv, int64_t T, void *stream)
{
    const sq_status s = sq::check_rows(K, ldk, V, ldv, T, Hk, D, row_start, cached, B, table, per_sequence, page, cache, pages);
    if (s != SQ_OK || T == 0 || B == 0 || per_sequence == 0 || pages == 0) return s;
    const sq::CacheView c = sq::cache_view(cache, pages, Hk, D, page, table, per_sequence, row_start, cached, B);
    auto kernel = D == 64 ? sq::cache_read_kernel<64> : D == 128 ? sq::cache_read_kernel<128> : sq::cache_read_kernel<256>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)T), dim3(256), 0, static_cast<hipStream_t>(stream), c, static_cast<__half *>(K),
                       ldk, static_cast<__half *>(V), ldv);
    return hipGetLastError() == hipSuccess ? SQ_OK : SQ_ERR_LAUNCH;
}

// The paged 4-bit cache of keys and values: sq_cache_append quantizes new rows into their pages, sq_cache_read gives rows
// back as fp16.
#include "sq_cache.h"
#include "sq_quant4.h"

namespace sq {

namespace {

// Where a new row lives: its page (nullptr: none) and its slot in it.
__device__ __forceinline__ uint8_t *place_of_row(const CacheView &c, int64_t row, int &slot)
{
    const RowOwner r = owner_of_row(c, row);
    if (r.b < 0 || r.first < 0 || r.cached < 0) return nullptr;
    const int64_t at = (int64_t)r.cached + (row - r.first);
    if (at >= ((int64_t)c.per_sequence << c.page_shift)) return nullptr;
    slot = (int)at & ((1 << c.page_shift) - 1);
    const int number = cache_page(c, r.b, (int)(at >> c.page_shift));
    return number < 0 ? nullptr : c.base + (int64_t)number * c.page_bytes;
}

// One workgroup per row for few rows (512 rows of 8 heads of 128: append 3.4 us, 4.1 with a wave per row) and for wide ones
// (3003 rows of 32 heads of 128: 13.8 us against 16.3); otherwise a wave per row (16384 rows of 8 heads of 128: append
// 19.5 us against 21.4, read 17.0 against 22.9).
inline bool workgroup_per_row(int64_t T, int Hk, int D) { return T <= 1024 || Hk * D > 2048; }

// WAVES waves share a row; a lane takes eight channels of a head of K or V, D / 8 neighbouring lanes a head, and has
// 4 / WAVES such units under way at once.  Every wave finds the row's place by itself (three dependent loads: the sequence,
// the page's number, the codes); append asks for the first units of the row before it looks, since they are needed wherever
// the row goes.  Neighbouring rows share lines of a page, so neighbouring workgroups belong to one XCD, whose L2 joins
// their pieces of a line.  A launch for few rows is all latency (1 to 16 rows of 8 heads of 128: 3.1 us for either
// kernel), many are bound by memory: 16384 rows of 8 heads of 128, 84 MB, 19.6 us in and 17.0 out (4.3 and 4.9 TB/s).
template <int WAVES>
__device__ __forceinline__ int64_t row_of_wave(int64_t T)
{
    constexpr int ROWS = 4 / WAVES;                    // of a workgroup
    const int64_t number = block_number();
    const int groups = (int)((T + ROWS - 1) / ROWS);
    if (number >= groups) return T;
    return (int64_t)xcd_contiguous_id((int)number, groups) * ROWS + __builtin_amdgcn_readfirstlane((int)(threadIdx.x / (WAVES * kWave)));
}

template <int D, int WAVES>
__global__ __launch_bounds__(256) void cache_append_kernel(const CacheView c, const __half *__restrict__ K, int64_t ldk,
                                                           const __half *__restrict__ V, int64_t ldv, int64_t T)
{
    constexpr int LANES = D / 8, AT_ONCE = 4 / WAVES, SHARE = WAVES * kWave;
    const int lane = (int)threadIdx.x % SHARE;
    const int64_t row = row_of_wave<WAVES>(T);
    if (row >= T) return;
    const int units = 2 * c.Hk * LANES;
    uint4 x[AT_ONCE];
    auto request = [&](int u0) {
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int unit = min(u0 + k * SHARE + lane, units - 1);            // whole waves: the maxima need every lane
            const int head = unit / LANES, piece = unit % LANES;
            const __half *src = head >= c.Hk ? V + row * ldv + (head - c.Hk) * D : K + row * ldk + head * D;
            x[k] = *reinterpret_cast<const uint4 *>(src + 8 * piece);
        }
    };
    request(0);
    int slot;
    uint8_t *page = place_of_row(c, row, slot);
    if (!page) return;
    const int rows_of_page = 1 << c.page_shift, half_codes = rows_of_page * (D / 2);
    __half *steps = reinterpret_cast<__half *>(page + cache_steps_at(c.Hk, D, rows_of_page));
    for (int u0 = 0; u0 < units; u0 += AT_ONCE * SHARE) {
        if (u0 > 0) request(u0);
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int unit = u0 + k * SHARE + lane;
            // no step is infinite or NaN (either has more bits than 65504): the weight 0 of a row that is not seen gives 0
            const __half s = __ushort_as_half(min(__half_as_ushort(run_step(run_max<LANES>(x[k]))), (unsigned short)0x7BFF));
            const uint32_t codes = run_codes_plus8(x[k], __builtin_amdgcn_rcpf(__half2float(s)));
            if (unit >= units) continue;
            const int head = unit / LANES, piece = unit % LANES;
            const bool is_v = head >= c.Hk;
            const int h = is_v ? head - c.Hk : head;
            uint8_t *dst = page + (int64_t)h * (2 * half_codes);
            if (!is_v) {
                *reinterpret_cast<uint32_t *>(dst + slot * (D / 2) + 4 * piece) = codes;
            } else {
                dst += half_codes;
                if constexpr (D == 64) {                                       // two units of two bytes
                    *reinterpret_cast<uint16_t *>(dst + cache_v_unit<D>(slot, 2 * piece)) = (uint16_t)codes;
                    *reinterpret_cast<uint16_t *>(dst + cache_v_unit<D>(slot, 2 * piece + 1)) = (uint16_t)(codes >> 16);
                } else if constexpr (D == 128) {
                    *reinterpret_cast<uint32_t *>(dst + cache_v_unit<D>(slot, piece)) = codes;
                } else {                                                       // half a unit of eight bytes
                    *reinterpret_cast<uint32_t *>(dst + cache_v_unit<D>(slot, piece / 2) + 4 * (piece & 1)) = codes;
                }
            }
            if (piece == 0) steps[(is_v ? c.Hk * rows_of_page : 0) + h * rows_of_page + slot] = s;
        }
    }
}

template <int D, int WAVES>
__global__ __launch_bounds__(256) void cache_read_kernel(const CacheView c, __half *__restrict__ K, int64_t ldk,
                                                         __half *__restrict__ V, int64_t ldv, int64_t T)
{
    constexpr int LANES = D / 8, AT_ONCE = 4 / WAVES, SHARE = WAVES * kWave;
    const int lane = (int)threadIdx.x % SHARE;
    const int64_t row = row_of_wave<WAVES>(T);
    if (row >= T) return;
    int slot;
    const uint8_t *page = place_of_row(c, row, slot);
    if (!page) return;
    const int rows_of_page = 1 << c.page_shift, half_codes = rows_of_page * (D / 2);
    const __half *steps = reinterpret_cast<const __half *>(page + cache_steps_at(c.Hk, D, rows_of_page));
    const int units = 2 * c.Hk * LANES;
    for (int u0 = 0; u0 < units; u0 += AT_ONCE * SHARE) {
        uint32_t codes[AT_ONCE];
        __half step[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int unit = min(u0 + k * SHARE + lane, units - 1), head = unit / LANES, piece = unit % LANES;
            const bool is_v = head >= c.Hk;
            const int h = is_v ? head - c.Hk : head;
            const uint8_t *src = page + (int64_t)h * (2 * half_codes);
            if constexpr (D == 64) {                                           // a unit of V is two bytes
                const int64_t a = is_v ? half_codes + cache_v_unit<D>(slot, 2 * piece) : slot * (D / 2) + 4 * piece;
                const int64_t b = is_v ? half_codes + cache_v_unit<D>(slot, 2 * piece + 1) : a + 2;
                codes[k] = *reinterpret_cast<const uint16_t *>(src + a) | ((uint32_t) * reinterpret_cast<const uint16_t *>(src + b) << 16);
            } else {
                const int v = D == 128 ? cache_v_unit<D>(slot, piece) : cache_v_unit<D>(slot, piece / 2) + 4 * (piece & 1);
                codes[k] = *reinterpret_cast<const uint32_t *>(src + (is_v ? half_codes + v : slot * (D / 2) + 4 * piece));
            }
            step[k] = steps[(is_v ? c.Hk * rows_of_page : 0) + h * rows_of_page + slot];
        }
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int unit = u0 + k * SHARE + lane, head = unit / LANES, piece = unit % LANES;
            if (unit >= units) continue;
            const float s = __half2float(step[k]);
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                // code * step: 15 bits, rounded once to fp16
                const v2h p = {(_Float16)((float)((int)((codes[k] >> (8 * e)) & 15) - 8) * s),
                               (_Float16)((float)((int)((codes[k] >> (8 * e + 4)) & 15) - 8) * s)};
                w[e] = __builtin_bit_cast(uint32_t, p);
            }
            __half *dst = head >= c.Hk ? V + row * ldv + (head - c.Hk) * D : K + row * ldk + head * D;
            *reinterpret_cast<uint4 *>(dst + 8 * piece) = uint4{w[0], w[1], w[2], w[3]};
        }
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
    const bool few = sq::workgroup_per_row(T, Hk, D);
    auto kernel = few ? (D == 64 ? sq::cache_append_kernel<64, 4> : D == 128 ? sq::cache_append_kernel<128, 4> : sq::cache_append_kernel<256, 4>)
                      : (D == 64 ? sq::cache_append_kernel<64, 1> : D == 128 ? sq::cache_append_kernel<128, 1> : sq::cache_append_kernel<256, 1>);
    hipLaunchKernelGGL(kernel, sq::grid_of(few ? T : (T + 3) / 4), dim3(256), 0, static_cast<hipStream_t>(stream), c,
                       static_cast<const __half *>(K), ldk, static_cast<const __half *>(V), ldv, T);
    return hipGetLastError() == hipSuccess ? SQ_OK : SQ_ERR_LAUNCH;
}

extern "C" sq_status sq_cache_read(const void *cache, int32_t pages, int32_t Hk, int32_t D, const int32_t *row_start,
                                   const int32_t *cached, int32_t B, const int32_t *table, int32_t per_sequence, int32_t page,
                                   void *K, int64_t ldk, void *V, int64_t ldv, int64_t T, void *stream)
{
    const sq_status s = sq::check_rows(K, ldk, V, ldv, T, Hk, D, row_start, cached, B, table, per_sequence, page, cache, pages);
    if (s != SQ_OK || T == 0 || B == 0 || per_sequence == 0 || pages == 0) return s;
    const sq::CacheView c = sq::cache_view(cache, pages, Hk, D, page, table, per_sequence, row_start, cached, B);
    const bool few = sq::workgroup_per_row(T, Hk, D);
    auto kernel = few ? (D == 64 ? sq::cache_read_kernel<64, 4> : D == 128 ? sq::cache_read_kernel<128, 4> : sq::cache_read_kernel<256, 4>)
                      : (D == 64 ? sq::cache_read_kernel<64, 1> : D == 128 ? sq::cache_read_kernel<128, 1> : sq::cache_read_kernel<256, 1>);
    hipLaunchKernelGGL(kernel, sq::grid_of(few ? T : (T + 3) / 4), dim3(256), 0, static_cast<hipStream_t>(stream), c, static_cast<__half *>(K),
                       ldk, static_cast<__half *>(V), ldv, T);
    return hipGetLastError() == hipSuccess ? SQ_OK : SQ_ERR_LAUNCH;
}

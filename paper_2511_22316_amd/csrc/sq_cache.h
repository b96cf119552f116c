// Layout of a page of the 4-bit cache (public in singlequant.h) and what the kernels that write and read it share.
#pragma once

#include "sq_common.h"

namespace sq {

// A cache as the entry points take it.
struct CacheView {
    uint8_t *base;
    int64_t page_bytes;
    const int32_t *table;      // [B, per_sequence] page numbers
    const int32_t *row_start;  // [B + 1] first new row of every sequence
    const int32_t *cached;     // [B] rows a sequence had before its new ones
    int pages, per_sequence, B, Hk, page_shift;
};

// Bytes in front of the steps of a page; K's steps [Hk][page], then V's.
__host__ __device__ __forceinline__ int64_t cache_steps_at(int Hk, int D, int page) { return (int64_t)Hk * page * D; }

// Byte of the codes of unit o (channels o D / 16 .. of a head, D / 32 bytes) of V in slot `slot`, relative to the head's V
// codes: blocks of 16 slots, in a block [slot / 4 % 4][unit][slot % 4], so that a lane of the attention kernel takes the
// unit of four neighbouring slots as one run of bytes.
template <int D>
__device__ __forceinline__ int cache_v_unit(int slot, int o)
{
    return (slot >> 4) * (8 * D) + ((((slot >> 2) & 3) * 16 + o) * 4 + (slot & 3)) * (D / 32);
}

// Page number of page `index` of sequence b, or -1 where the table holds none that exists.
__device__ __forceinline__ int cache_page(const CacheView &c, int b, int index)
{
    if (index < 0 || index >= c.per_sequence) return -1;
    const int number = c.table[(int64_t)b * c.per_sequence + index];
    return number >= 0 && number < c.pages ? number : -1;
}

// Sequence of new row `row` (the same in every lane of the wave): the last b with row_start[b] <= row.  64 probes at a
// time: one memory latency up to 64 sequences, two up to 4096.  -1 for a row in front of the first or behind the last.
__device__ __forceinline__ int sequence_of_row(const int32_t *row_start, int B, int64_t row)
{
    const int lane = (int)(threadIdx.x & (kWave - 1));
    int lo = 0, count = B;                     // the answer, if there is one, is in lo .. lo + count - 1
    while (count > 0) {
        const int step = (count + kWave - 1) / kWave;
        const int at = lo + lane * step;
        const bool before = at < lo + count && (int64_t)row_start[at] <= row;
        const int hits = __popcll(__ballot(before));
        if (hits == 0) return -1;
        const int next = lo + (hits - 1) * step;
        count = min(step, lo + count - next);
        lo = next;
        if (step == 1) break;
    }
    return count > 0 && row < (int64_t)row_start[lo + 1] ? lo : -1;
}

// sizes and pointers that every entry point on a cache checks alike
inline sq_status check_cache(int32_t Hk, int32_t D, int32_t page, int32_t B, int32_t per_sequence, int32_t pages)
{
    if (Hk <= 0 || Hk > SQ_CACHE_MAX_HEADS || (D != 64 && D != 128 && D != 256)) return SQ_ERR_SHAPE;
    if (page < 16 || page > 1024 || (page & (page - 1)) != 0) return SQ_ERR_SHAPE;
    if (B < 0 || B > SQ_CACHE_MAX_SEQUENCES || per_sequence < 0 || pages < 0) return SQ_ERR_SHAPE;
    if ((int64_t)per_sequence * page > 0x7FFFFFFF) return SQ_ERR_SHAPE;          // positions are 32-bit
    return SQ_OK;
}

inline CacheView cache_view(const void *cache, int32_t pages, int32_t Hk, int32_t D, int32_t page, const int32_t *table,
                            int32_t per_sequence, const int32_t *row_start, const int32_t *cached, int32_t B)
{
    CacheView c;
    c.base = static_cast<uint8_t *>(const_cast<void *>(cache));
    c.page_bytes = sq_cache_page_bytes(Hk, D, page);
    c.table = table;
    c.row_start = row_start;
    c.cached = cached;
    c.pages = pages;
    c.per_sequence = per_sequence;
    c.B = B;
    c.Hk = Hk;
    c.page_shift = __builtin_ctz((unsigned)page);
    return c;
}

}  // namespace sq

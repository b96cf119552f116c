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

// A new row's sequence, with what the sequence's arrays say of it.
struct RowOwner {
    int b;                     // -1: none
    int first, cached;         // row_start[b], cached[b]
};

// The sequence of new row `row` (the same in every lane of the wave): the last b with row_start[b] <= row, if the row is in
// front of row_start[b + 1].  64 probes at a time, and the last ones bring the sequence's own numbers with them: one memory
// latency up to 64 sequences, two up to 4096.
__device__ __forceinline__ RowOwner owner_of_row(const CacheView &c, int64_t row)
{
    const int lane = (int)(threadIdx.x & (kWave - 1));
    const RowOwner none = {-1, 0, 0};
    int lo = 0, count = c.B;                   // the answer, if there is one, is in lo .. lo + count - 1
    while (count > kWave) {
        const int step = (count + kWave - 1) / kWave;
        const int at = lo + lane * step;
        const int hits = __popcll(__ballot(at < lo + count && (int64_t)c.row_start[at] <= row));
        if (hits == 0) return none;
        const int next = lo + (hits - 1) * step;
        count = min(step, lo + count - next);
        lo = next;
    }
    int first = 0, end = 0, cached = 0;
    const bool there = lane < count;
    if (there) {
        first = c.row_start[lo + lane];
        end = c.row_start[lo + lane + 1];
        cached = c.cached[lo + lane];
    }
    const int hits = __popcll(__ballot(there && (int64_t)first <= row));
    if (hits == 0) return none;
    const RowOwner r = {lo + hits - 1, __builtin_amdgcn_readlane(first, hits - 1), __builtin_amdgcn_readlane(cached, hits - 1)};
    return row < (int64_t)__builtin_amdgcn_readlane(end, hits - 1) ? r : none;
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

// sq_tree_attention: attention of new rows (one token a sequence, a tree of drafted tokens, or a prompt) over the paged
// 4-bit cache that holds them and everything before them.
#include "sq_cache.h"

namespace sq {

namespace {

// One wave per new row and query head.  Keys in runs of 64, a lane a key: its score, the running maximum and sum of the
// softmax over the lanes, then the values with a lane holding D / 64 channels.
template <int D>
__global__ __launch_bounds__(64) void tree_attention_row_kernel(const CacheView c, const __half *__restrict__ Q, int64_t ldq,
                                                                int Hq, const uint64_t *__restrict__ mask, int max_rows, float scale,
                                                                __half *__restrict__ O, int64_t ldo)
{
    __shared__ float q[D], p[kWave];
    __shared__ int64_t page_of[kWave];
    const int lane = threadIdx.x, hq = blockIdx.y, h = hq / (Hq / c.Hk);
    const int64_t row = blockIdx.x;
    const int b = sequence_of_row(c.row_start, c.B, row);
    if (b < 0) return;
    const int first = c.row_start[b], n = c.row_start[b + 1] - first, mine = (int)(row - first);
    if (mine >= max_rows) return;
    const int past = max(c.cached[b], 0);
    const int page = 1 << c.page_shift, half_codes = page * (D / 2);
    for (int d = lane; d < D; d += kWave) q[d] = __half2float(Q[row * ldq + hq * D + d]) * scale;
    __syncthreads();
    const uint64_t word = mask ? mask[row] : 0;
    const int64_t total = min((int64_t)past + (mask ? min(n, 64) : mine + 1), (int64_t)c.per_sequence << c.page_shift);
    float m = -1e30f, l = 0.f, acc[D / 64] = {};
    for (int64_t k0 = 0; k0 < total; k0 += kWave) {
        const int64_t key = k0 + lane;
        const bool sees = key < total && (key < past || !mask || ((word >> (key - past)) & 1));
        const int number = sees ? cache_page(c, b, (int)(key >> c.page_shift)) : -1;
        float s = -INFINITY;
        if (number >= 0) {
            const uint8_t *at = c.base + (int64_t)number * c.page_bytes;
            const int slot = (int)key & (page - 1);
            const uint8_t *codes = at + (int64_t)h * (2 * half_codes) + slot * (D / 2);
            float sum = 0.f;
            for (int d = 0; d < D / 2; ++d)
                sum += q[2 * d] * (float)((codes[d] & 15) - 8) + q[2 * d + 1] * (float)((codes[d] >> 4) - 8);
            s = sum * __half2float(reinterpret_cast<const __half *>(at + cache_steps_at(c.Hk, D, page))[h * page + slot]);
        }
        float top = s;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, kWave));
        const float m_new = fmaxf(m, top), fade = expf(m - m_new);
        float e = expf(s - m_new);
        l *= fade;
        m = m_new;
#pragma unroll
        for (int i = 0; i < D / 64; ++i) acc[i] *= fade;
        float sum = e;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, kWave);
        l += sum;
        __syncthreads();
        p[lane] = e;
        page_of[lane] = number;
        __syncthreads();
        for (int j = 0; j < kWave; ++j) {
            if (page_of[j] < 0) continue;
            const uint8_t *at = c.base + page_of[j] * c.page_bytes;
            const int slot = (int)(k0 + j) & (page - 1);
            const float w =
                p[j] * __half2float(reinterpret_cast<const __half *>(at + cache_steps_at(c.Hk, D, page))[(c.Hk + h) * page + slot]);
#pragma unroll
            for (int i = 0; i < D / 64; ++i) {
                const int d = (D / 64) * lane + i;
                const uint8_t byte = at[(int64_t)h * (2 * half_codes) + half_codes + cache_v_unit<D>(slot, d / (D / 16)) + d % (D / 16) / 2];
                acc[i] += w * (float)(((byte >> (4 * (d & 1))) & 15) - 8);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < D / 64; ++i)
        O[row * ldo + hq * D + (D / 64) * lane + i] = __float2half_rn(l > 0.f ? acc[i] / l : 0.f);
}

}  // namespace

}  // namespace sq

extern "C" int64_t sq_tree_attention_workspace_bytes(int64_t T, int32_t Hq, int32_t D)
{
    if (T < 0 || T > SQ_MAX_ROWS || Hq <= 0 || Hq > 65536 || (D != 64 && D != 128 && D != 256)) return -1;
    return 0;
}

extern "C" sq_status sq_tree_attention(const void *Q, int64_t ldq, int64_t T, int32_t Hq, int32_t Hk, int32_t D,
                                       const int32_t *row_start, const int32_t *cached, int32_t B, const uint64_t *mask,
                                       int32_t max_rows, int32_t max_keys, const int32_t *table, int32_t per_sequence,
                                       int32_t page, const void *cache, int32_t pages, float scale, void *O, int64_t ldo,
                                       void *workspace, int64_t workspace_bytes, void *stream)
{
    const sq_status s = sq::check_cache(Hk, D, page, B, per_sequence, pages);
    if (s != SQ_OK) return s;
    if (T < 0 || T > SQ_MAX_ROWS || Hq <= 0 || Hq > 65536 || (Hq % Hk) != 0) return SQ_ERR_SHAPE;
    if (ldq < (int64_t)Hq * D || ldo < (int64_t)Hq * D || !(scale > 0.f) || !(scale < 1e30f)) return SQ_ERR_SHAPE;
    if (max_rows < 0 || max_keys < 0 || (mask && max_rows > 64) || workspace_bytes < 0) return SQ_ERR_SHAPE;
    if (T == 0 || B == 0 || max_rows == 0) return SQ_OK;
    if (!Q || !O || !row_start || !cached || (!table && per_sequence > 0) || (!cache && pages > 0) || (!workspace && workspace_bytes > 0))
        return SQ_ERR_NULL;
    if (((uintptr_t)Q & 15) || ((uintptr_t)O & 15) || (ldq % 8) != 0 || (ldo % 8) != 0 || ((uintptr_t)cache & 15) ||
        ((uintptr_t)workspace & 15) || (((uintptr_t)row_start | (uintptr_t)cached | (uintptr_t)table) & 3) || ((uintptr_t)mask & 7))
        return SQ_ERR_ALIGN;
    const sq::CacheView c = sq::cache_view(cache, pages, Hk, D, page, table, per_sequence, row_start, cached, B);
    auto kernel = D == 64 ? sq::tree_attention_row_kernel<64> : D == 128 ? sq::tree_attention_row_kernel<128> : sq::tree_attention_row_kernel<256>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)T, (unsigned)Hq), dim3(64), 0, static_cast<hipStream_t>(stream), c,
                       static_cast<const __half *>(Q), ldq, Hq, mask, max_rows, scale, static_cast<__half *>(O), ldo);
    return hipGetLastError() == hipSuccess ? SQ_OK : SQ_ERR_LAUNCH;
}

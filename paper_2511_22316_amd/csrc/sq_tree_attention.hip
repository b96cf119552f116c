// sq_tree_attention: attention of new rows (one token a sequence, a tree of drafted tokens, or a prompt) over the paged
// 4-bit cache that holds them and everything before them.
#include "sq_cache.h"

namespace sq {

namespace {

constexpr int kKeysPerTile = 32;       // of one wave and step
constexpr int kWaves = 4;
constexpr int kChunkUnit = kKeysPerTile * kWaves;
constexpr int kMaxSplits = 64;         // a lane each in the kernel that joins them
constexpr float kNothing = -1e30f;     // running maximum of a row that has seen no key

// Four fp16 of one dword pair.
typedef _Float16 v4hs __attribute__((ext_vector_type(4)));

// max over the four lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float quarter_max(float v)
{
    typedef uint32_t v2u __attribute__((ext_vector_type(2)));
    const uint32_t x = __builtin_bit_cast(uint32_t, v);
    const v2u s = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    const uint32_t s0 = s[0], s1 = s[1];       // named: a bit cast of a vector's element takes element 0
    const uint32_t y = __builtin_bit_cast(uint32_t, fmaxf(__builtin_bit_cast(float, s0), __builtin_bit_cast(float, s1)));
    const v2u t = __builtin_amdgcn_permlane32_swap(y, y, false, false);
    const uint32_t t0 = t[0], t1 = t[1];
    return fmaxf(__builtin_bit_cast(float, t0), __builtin_bit_cast(float, t1));
}
__device__ __forceinline__ float quarter_sum(float v)
{
    v += __shfl_xor(v, 16, kWave);
    return v + __shfl_xor(v, 32, kWave);
}

// What a call is made of beside the cache.
struct AttentionCall {
    const __half *Q;
    __half *O;
    const uint64_t *mask;
    float *part;               // [T, Hq, splits, D] sums of a split, then [T, Hq, splits] (maximum, sum); null: one split
    int64_t ldq, ldo, T;
    int Hq, group, max_rows, splits, row_blocks, tiles_per_chunk;
    float score_scale;         // scale * log2(e) * 2^18
};

// New rows of sequence b that the call has: their number, and the first.
__device__ __forceinline__ int rows_of(const CacheView &c, const AttentionCall &a, int b, int64_t &first)
{
    first = c.row_start[b];
    if (first < 0 || first >= a.T) return 0;
    const int64_t n = min((int64_t)c.row_start[b + 1], a.T) - first;
    return (int)max((int64_t)0, n);
}

// A workgroup takes one head of K and V of one sequence, 16 R query rows (row = new row * group + query head in the group)
// and every splits-th chunk of its keys; its four waves take every fourth tile of 32 keys each and work alone until
// the end.
//
// Scores: S^T = K Q^T on v_mfma_f32_16x16x32_f16, the keys as rows of the result and the query rows as columns, so a lane has
// one query row (lane % 16) and four keys of each half of the tile (4 (lane / 16) + r); the weights it makes of them are
// already the other operand of O^T = V^T P, whose contraction runs over the keys: nothing is moved between lanes but
// the maximum (two swaps).  O^T again has the query row in the lane.
//
// Nibbles (code + 8) become fp16 without a conversion: a nibble in bits 6 to 9 of a half is the subnormal u 2^-18, which
// the matrix cores take as it is.  (They line products up by the exponents alone: a subnormal counts as 2^-14, so the low
// bits that its leading zeros push out are lost.  In bits 0 to 3 the same sums were off by 2^-14 of a step, in bits 6 to
// 9 it is 2^-20.)  For K a dword gives four pairs, one shift and one and each; V's pairs need the same channel of two keys,
// which one byte permute brings together for two channels.  The eights come off by sums: the scores' accumulators start at
// -8 * 2^-18 * sum(q), and a matrix instruction with ones in place of V gives the sum of the weights.
//
// Softmax with a running offset M per row: a weight is exp2(s - M) times the value's step, rounded to fp16 (its half step
// of rounding averages out over the keys; the normaliser keeps the weight in fp32).  M goes by the largest of score plus
// exponent of the step, so the largest product lies between 2^-1 and 2^6 whatever the steps are, and moves only when
// that is passed.
//
// Loads: K of the next tile is requested when this one's scores are done, V when its products are: one set of registers,
// all of it in flight most of the time.
template <int D, int R>
__global__ __launch_bounds__(kWaves *kWave, D == 256 ? 2 : R == 1 ? 4 : 2) void tree_attention_kernel(const CacheView c, const AttentionCall a)
{
    constexpr int KD = D / 32;                       // dwords of K (and of V) per lane and 16 keys; steps of the scores
    constexpr int VT = D / 16;                       // 16-channel tiles of the output
    constexpr int CB = D < 128 ? D : 128, LD = CB + 4;      // channels that meet in LDS at a time
    __shared__ float meet[kWaves][16][LD];
    __shared__ float2 meet_ml[kWaves][16];

    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int l16 = lane & 15, q = lane >> 4;
    int id = xcd_contiguous_id((int)blockIdx.x, (int)gridDim.x);
    const int row_block = id % a.row_blocks;
    id /= a.row_blocks;
    const int split = id % a.splits;
    id /= a.splits;
    const int h = id % c.Hk, b = id / c.Hk;

    int64_t first;
    const int n = rows_of(c, a, b, first);
    const int rows = min(n, a.max_rows) * a.group, row0 = row_block * 16 * R;
    if (row0 >= rows) return;
    const int page = 1 << c.page_shift;
    const uint32_t cap = (uint32_t)c.per_sequence << c.page_shift;
    const uint32_t past = min((uint32_t)max(c.cached[b], 0), cap);
    // keys that the rows of this workgroup see at all, and that all of them see
    const int last_row = min(n, (row0 + 16 * R - 1) / a.group + 1);
    const uint32_t limit = min(past + (uint32_t)(a.mask ? min(n, 64) : last_row), cap);
    const uint32_t all_see = a.mask ? past : min(past + (uint32_t)(row0 / a.group) + 1, limit);

    // query rows: channels (D / 4) q .. of this lane's row, in the order the nibbles come in
    v8h qf[R][KD];
    float bias[R];
    int row_of[R];
    uint64_t word[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = row0 + 16 * r + l16, i = row / a.group, hq = h * a.group + row - i * a.group;
        const bool there = row < rows;
        row_of[r] = i;
        word[r] = there && a.mask ? a.mask[first + i] : 0;
        const __half *src = a.Q + (there ? (first + i) * a.ldq + hq * D : first * a.ldq) + q * (D / 4);
        float sum = 0.f;
#pragma unroll
        for (int d = 0; d < KD; ++d) {
            const v8h x = *reinterpret_cast<const v8h *>(src + 8 * d);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += (float)x[e];
            qf[r][d] = v8h{x[0], x[4], x[1], x[5], x[2], x[6], x[3], x[7]};
        }
        bias[r] = -8.f * 0x1p-18f * quarter_sum(sum);
    }

    const int half_codes = page * (D / 2);
    const uint32_t k_lane = l16 * (D / 2) + q * (D / 8), v_lane = half_codes + lane * (D / 8);
    const int64_t head_at = (int64_t)h * (2 * half_codes), steps_at = cache_steps_at(c.Hk, D, page) + (int64_t)h * page * 2;
    const int64_t v_steps = (int64_t)c.Hk * page * 2;
    const int32_t *table = c.table + (int64_t)b * c.per_sequence;
    // page numbers of the two halves of a tile (their keys clamped to the last there is)
    auto pages_of = [&](uint32_t tile, int(&number)[2]) {
#pragma unroll
        for (int f = 0; f < 2; ++f) number[f] = table[min(tile * kKeysPerTile + 16 * f, limit - 1) >> c.page_shift];
    };
    // a page that does not exist is read as page 0, and masked
    auto page_ok = [&](int number) { return number >= 0 && number < c.pages; };
    auto page_at = [&](int number) { return c.base + (int64_t)(page_ok(number) ? number : 0) * c.page_bytes; };
    // slots of a half behind the last key lie in the same page, written or not
    auto slot_of = [&](uint32_t tile, int f) { return (int)((tile * kKeysPerTile + 16 * f) & (uint32_t)(page - 1)); };

    typedef uint32_t dwords __attribute__((ext_vector_type(KD)));
    dwords kx[2], vx[2];
    v4hs ks[2], vs[2];
    auto load_codes = [&](dwords(&x)[2], uint32_t tile, const int(&number)[2], uint32_t lane_at) {
#pragma unroll
        for (int f = 0; f < 2; ++f)
            x[f] = *reinterpret_cast<const dwords *>(page_at(number[f]) + head_at + slot_of(tile, f) * (D / 2) + lane_at);
    };
    auto load_steps = [&](uint32_t tile, const int(&number)[2]) {
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            const uint8_t *at = page_at(number[f]) + steps_at + 2 * slot_of(tile, f) + 8 * q;
            ks[f] = *reinterpret_cast<const v4hs *>(at);
            vs[f] = *reinterpret_cast<const v4hs *>(at + v_steps);
        }
    };

    v4f o[R][VT], weights[R];
    float M[R], l[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        M[r] = kNothing;
        l[r] = 0.f;
        weights[r] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < VT; ++j) o[r][j] = v4f{0.f, 0.f, 0.f, 0.f};
    }
    const v8h ones = {1, 1, 1, 1, 1, 1, 1, 1};

    uint32_t chunk_end = (uint32_t)(split + 1) * a.tiles_per_chunk;
    const uint32_t to_next_chunk = (uint32_t)(a.splits - 1) * a.tiles_per_chunk, tiles = (limit + kKeysPerTile - 1) / kKeysPerTile;
    auto following = [&](uint32_t tile) {
        tile += kWaves;
        if (tile >= chunk_end) {
            tile += to_next_chunk;
            chunk_end += to_next_chunk + a.tiles_per_chunk;
        }
        return tile;
    };
    uint32_t tile = (uint32_t)split * a.tiles_per_chunk + wave;
    if (tile < tiles) {
        int number[2], number_n[2];
        pages_of(tile, number);
        uint32_t tile_n = following(tile);
        pages_of(min(tile_n, tiles - 1), number_n);
        load_codes(kx, tile, number, k_lane);
        load_steps(tile, number);
        load_codes(vx, tile, number, v_lane);
        while (true) {
            const bool more = tile_n < tiles;
            const uint32_t tile_l = more ? tile_n : tile;              // behind the last tile: that one again, unused
            const int number_l[2] = {more ? number_n[0] : number[0], more ? number_n[1] : number[1]};
            // scores
            v4f s[R][2];
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int f = 0; f < 2; ++f) s[r][f] = v4f{bias[r], bias[r], bias[r], bias[r]};
#pragma unroll
            for (int d = 0; d < KD; ++d)
#pragma unroll
                for (int f = 0; f < 2; ++f) {
                    const uint32_t x = kx[f][d];
                    const v4i w = {(int)((x << 6) & 0x03C003C0u), (int)((x << 2) & 0x03C003C0u), (int)((x >> 2) & 0x03C003C0u),
                                   (int)((x >> 6) & 0x03C003C0u)};
#pragma unroll
                    for (int r = 0; r < R; ++r)
                        s[r][f] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, w), qf[r][d], s[r][f], 0, 0, 0);
                }
            load_codes(kx, tile_l, number_l, k_lane);
            const uint32_t tile_2 = following(tile_l);
            int number_2[2];
            pages_of(min(tile_2, tiles - 1), number_2);

            // scores times steps; keys that a row does not see
            const uint32_t key0 = tile * kKeysPerTile;
            const bool cut = key0 + kKeysPerTile > all_see || !page_ok(number[0]) || !page_ok(number[1]);
            float step_v[2][4];
#pragma unroll
            for (int f = 0; f < 2; ++f)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    step_v[f][e] = (float)vs[f][e];
#pragma unroll
                    for (int r = 0; r < R; ++r) s[r][f][e] *= (float)ks[f][e] * a.score_scale;
                }
            float step_exponent[2][4];                   // 2^ of it is over the value's step
#pragma unroll
            for (int f = 0; f < 2; ++f)
#pragma unroll
                for (int e = 0; e < 4; ++e) step_exponent[f][e] = (float)__builtin_amdgcn_frexp_expf(step_v[f][e]);
            if (cut) {
#pragma unroll
                for (int f = 0; f < 2; ++f)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t key = key0 + 16 * f + 4 * q + e;
                        const bool in = key < limit && page_ok(number[f]);
                        const int new_row = (int)(key - past);
                        if (!in) step_v[f][e] = step_exponent[f][e] = 0.f;
#pragma unroll
                        for (int r = 0; r < R; ++r) {
                            const bool sees = in && (key < past || (a.mask ? ((word[r] >> (new_row & 63)) & 1) != 0 : new_row <= row_of[r]));
                            s[r][f][e] = sees ? s[r][f][e] : -INFINITY;
                        }
                    }
            }
            load_steps(tile_l, number_l);
            v8h p[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float want = -INFINITY;
#pragma unroll
                for (int e = 0; e < 8; ++e) want = fmaxf(want, s[r][e / 4][e % 4] + step_exponent[e / 4][e % 4]);
                want = quarter_max(want);
                if (__any(want > M[r] + 6.f)) {
                    const float M_new = fmaxf(M[r], want), fade = __builtin_amdgcn_exp2f(M[r] - M_new);
                    M[r] = M_new;
                    l[r] *= fade;
                    weights[r] *= fade;
#pragma unroll
                    for (int j = 0; j < VT; ++j) o[r][j] *= fade;
                }
                float w[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    w[e] = __builtin_amdgcn_exp2f(s[r][e / 4][e % 4] - M[r]);
                    p[r][e] = (_Float16)(w[e] * step_v[e / 4][e % 4]);
                }
                l[r] += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
                weights[r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, p[r], weights[r], 0, 0, 0);
            }
            // values: unit lane % 16 of eight keys, two keys of one channel to a dword
            auto unit_byte = [&](int f, int key, int i, uint32_t &from, int &byte) {
                const int at = key * (D / 32) + i;
                from = vx[f][at / 4];
                byte = at % 4;
            };
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                v4i even, odd;
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    uint32_t x0, x1;
                    int b0, b1;
                    unit_byte(d / 2, 2 * (d % 2), i, x0, b0);
                    unit_byte(d / 2, 2 * (d % 2) + 1, i, x1, b1);
                    const uint32_t t = __builtin_amdgcn_perm(x1, x0, 0x0C000C00u | (uint32_t)b0 | ((uint32_t)(4 + b1) << 16));
                    even[d] = (int)((t << 6) & 0x03C003C0u);
                    odd[d] = (int)((t << 2) & 0x03C003C0u);
                }
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    o[r][2 * i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, even), p[r], o[r][2 * i], 0, 0, 0);
                    o[r][2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, odd), p[r], o[r][2 * i + 1], 0, 0, 0);
                }
            }
            if (!more) break;
            load_codes(vx, tile_l, number_l, v_lane);
            tile = tile_n;
            tile_n = tile_2;
#pragma unroll
            for (int f = 0; f < 2; ++f) {
                number[f] = number_n[f];
                number_n[f] = number_2[f];
            }
        }
    }

    // the waves' sums meet, 16 rows and CB channels at a time
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (row0 + 16 * r >= rows) break;
        const float sum = quarter_sum(l[r]);
        if (q == 0) meet_ml[wave][l16] = float2{M[r], sum};
#pragma unroll
        for (int cb = 0; cb < D / CB; ++cb) {
            if (q * (D / 4) / CB == cb) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int j = 0; j < VT; j += 4) {
                        const float off = -8.f * weights[r][e];
                        *reinterpret_cast<float4 *>(&meet[wave][l16][q * (D / 4) % CB + e * VT + j]) =
                            float4{__builtin_fmaf(o[r][j][e], 0x1p18f, off), __builtin_fmaf(o[r][j + 1][e], 0x1p18f, off),
                                   __builtin_fmaf(o[r][j + 2][e], 0x1p18f, off), __builtin_fmaf(o[r][j + 3][e], 0x1p18f, off)};
                    }
            }
            __syncthreads();
            constexpr int PER = CB / 16;                               // channels per thread
            const int mine = threadIdx.x / 16, at = (threadIdx.x % 16) * PER, row = row0 + 16 * r + mine;
            if (row < rows) {
                float top = kNothing, total = 0.f, out[PER] = {};
#pragma unroll
                for (int w = 0; w < kWaves; ++w) top = fmaxf(top, meet_ml[w][mine].x);
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    const float2 ml = meet_ml[w][mine];
                    const float share = __builtin_amdgcn_exp2f(ml.x - top);
                    total = __builtin_fmaf(share, ml.y, total);
#pragma unroll
                    for (int k = 0; k < PER; ++k) out[k] = __builtin_fmaf(share, meet[w][mine][at + k], out[k]);
                }
                const int i = row / a.group, hq = h * a.group + row - i * a.group;
                if (a.splits == 1) {
                    const float scale = total > 0.f ? 1.f / total : 0.f;
                    __half *dst = a.O + (first + i) * a.ldo + hq * D + cb * CB + at;
#pragma unroll
                    for (int k = 0; k < PER; k += 4) {
                        const v4hs y = {(_Float16)(out[k] * scale), (_Float16)(out[k + 1] * scale), (_Float16)(out[k + 2] * scale),
                                        (_Float16)(out[k + 3] * scale)};
                        *reinterpret_cast<v4hs *>(dst + k) = y;
                    }
                } else {
                    const int64_t place = ((first + i) * a.Hq + hq) * a.splits + split;
                    float *dst = a.part + place * D + cb * CB + at;
#pragma unroll
                    for (int k = 0; k < PER; k += 4) *reinterpret_cast<float4 *>(dst + k) = float4{out[k], out[k + 1], out[k + 2], out[k + 3]};
                    if (cb == 0 && at == 0)
                        reinterpret_cast<float2 *>(a.part + a.T * a.Hq * (int64_t)a.splits * D)[place] = float2{top, total};
                }
            }
            __syncthreads();
        }
    }
}

// The splits of a row and head, at most kMaxSplits: one workgroup, D / 4 threads to a split, so that all sums are requested at
// once.  (One wave walking over the splits took 17.7 us for 64 of them.)
template <int D>
__global__ __launch_bounds__(256) void tree_attention_join_kernel(const CacheView c, const AttentionCall a)
{
    constexpr int LANES = D / 4, SIDE = 256 / LANES, MOST = kMaxSplits / SIDE;     // threads of a split; splits side by side; rounds of them
    __shared__ float shares[kMaxSplits], totals;
    __shared__ float4 sums[SIDE][LANES];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), mine = tid % LANES, side = tid / LANES;
    const int b = blockIdx.y, i = (int)(blockIdx.x / (unsigned)a.Hq), hq = (int)(blockIdx.x % (unsigned)a.Hq);
    int64_t first;
    const int n = rows_of(c, a, b, first);
    if (i >= min(n, a.max_rows)) return;
    const int64_t place = ((first + i) * a.Hq + hq) * a.splits;
    const float2 ml = reinterpret_cast<const float2 *>(a.part + a.T * a.Hq * (int64_t)a.splits * D)[place + min(lane, a.splits - 1)];
    float4 v[MOST];
#pragma unroll
    for (int k = 0; k < MOST; ++k) {
        v[k] = float4{0.f, 0.f, 0.f, 0.f};
        if (k * SIDE < a.splits) v[k] = reinterpret_cast<const float4 *>(a.part + (place + min(k * SIDE + side, a.splits - 1)) * D)[mine];
    }
    const bool there = lane < a.splits && ml.y > 0.f;
    float top = there ? ml.x : kNothing;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, kWave));
    const float share = there ? __builtin_amdgcn_exp2f(ml.x - top) : 0.f;
    float total = share * (there ? ml.y : 0.f);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o, kWave);
    if (tid < kWave) {
        shares[lane] = share;                              // 0 behind the last split
        if (lane == 0) totals = total;
    }
    __syncthreads();
    float4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < MOST; ++k) {
        if (k * SIDE >= a.splits) break;
        const float w = shares[k * SIDE + side];
        sum.x = __builtin_fmaf(w, v[k].x, sum.x), sum.y = __builtin_fmaf(w, v[k].y, sum.y);
        sum.z = __builtin_fmaf(w, v[k].z, sum.z), sum.w = __builtin_fmaf(w, v[k].w, sum.w);
    }
    sums[side][mine] = sum;
    __syncthreads();
    if (tid >= LANES) return;
#pragma unroll
    for (int k = 1; k < SIDE; ++k) {
        const float4 x = sums[k][mine];
        sum.x += x.x, sum.y += x.y, sum.z += x.z, sum.w += x.w;
    }
    const float scale = totals > 0.f ? 1.f / totals : 0.f;
    const v4hs y = {(_Float16)(sum.x * scale), (_Float16)(sum.y * scale), (_Float16)(sum.z * scale), (_Float16)(sum.w * scale)};
    *reinterpret_cast<v4hs *>(a.O + (first + i) * a.ldo + hq * D + 4 * mine) = y;
}

template <int D, int R>
sq_status launch_tree_attention(const CacheView &c, const AttentionCall &a, hipStream_t st)
{
    const int64_t blocks = (int64_t)a.row_blocks * a.splits * c.Hk * c.B;
    if (blocks > 0x7FFFFFFF) return SQ_ERR_SHAPE;
    hipLaunchKernelGGL((tree_attention_kernel<D, R>), dim3((unsigned)blocks), dim3(kWaves * kWave), 0, st, c, a);
    if (hipGetLastError() != hipSuccess) return SQ_ERR_LAUNCH;
    if (a.splits == 1) return SQ_OK;
    const int64_t units = (int64_t)a.max_rows * a.Hq;
    if (units > 0x7FFFFFFF) return SQ_ERR_SHAPE;
    hipLaunchKernelGGL(tree_attention_join_kernel<D>, dim3((unsigned)units, (unsigned)c.B), dim3(256), 0, st, c, a);
    return hipGetLastError() == hipSuccess ? SQ_OK : SQ_ERR_LAUNCH;
}

template <int D>
sq_status dispatch_tree_attention(const CacheView &c, AttentionCall &a, int64_t max_keys, void *workspace, int64_t workspace_bytes,
                                  hipStream_t st)
{
    const int64_t rows = (int64_t)a.max_rows * a.group;
    const int tiles = rows <= 16 ? 1 : 2;
    if (rows > (1 << 30)) return SQ_ERR_SHAPE;
    a.row_blocks = (int)((rows + 16 * tiles - 1) / (16 * tiles));
    // as many splits as give every CU four workgroups, chunks of at least 128 keys, and what the workspace holds
    const int64_t units = (int64_t)a.row_blocks * c.Hk * c.B;
    max_keys = max_keys < 1 ? 1 : max_keys;
    int64_t splits = (1024 + units - 1) / units;
    const int64_t chunks = (max_keys + kChunkUnit - 1) / kChunkUnit, room = workspace_bytes / (a.T * a.Hq * (D + 2) * 4);
    splits = splits < chunks ? splits : chunks;
    splits = splits < kMaxSplits ? splits : kMaxSplits;
    splits = splits < room ? splits : room;
    a.splits = splits < 1 ? 1 : (int)splits;
    a.part = static_cast<float *>(workspace);
    a.tiles_per_chunk = kWaves * (int)((chunks + a.splits - 1) / a.splits);
    return tiles == 1 ? launch_tree_attention<D, 1>(c, a, st) : launch_tree_attention<D, 2>(c, a, st);
}

}  // namespace

}  // namespace sq

extern "C" int64_t sq_tree_attention_workspace_bytes(int64_t T, int32_t Hq, int32_t D)
{
    if (T < 0 || T > SQ_MAX_ROWS || Hq <= 0 || Hq > 65536 || (D != 64 && D != 128 && D != 256)) return -1;
    return T * Hq * (int64_t)(D + 2) * 4 * 64;
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
    sq::CacheView c = sq::cache_view(cache, pages, Hk, D, page, table, per_sequence, row_start, cached, B);
    if (pages == 0) c.per_sequence = 0;          // no sequence has a key
    sq::AttentionCall a = {};
    a.Q = static_cast<const __half *>(Q);
    a.O = static_cast<__half *>(O);
    a.mask = mask;
    a.ldq = ldq;
    a.ldo = ldo;
    a.T = T;
    a.Hq = Hq;
    a.group = Hq / Hk;
    a.max_rows = (int)(max_rows < T ? max_rows : T);
    a.score_scale = (float)((double)scale * 1.4426950408889634 * 262144.0);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (D == 64) return sq::dispatch_tree_attention<64>(c, a, max_keys, workspace, workspace_bytes, st);
    if (D == 128) return sq::dispatch_tree_attention<128>(c, a, max_keys, workspace, workspace_bytes, st);
    return sq::dispatch_tree_attention<256>(c, a, max_keys, workspace, workspace_bytes, st);
}

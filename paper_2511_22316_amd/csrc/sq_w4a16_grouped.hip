// sq_w4a16_gemm_grouped: fp16 activations times 4-bit weight codes with one fp16 step per group of K.
//
//   Y[t, n] = fp16( sum_g s[n, g] * sum_{k in g} X[t, k] Qw[n, k] )        fp32 sums
#include "sq_w4a16_tile.h"

namespace sq {

namespace {

// ---- at most 32 tokens ------------------------------------------------------------------------
// The product is one pass over the codes.  A wave takes 16 channels (lane % 16) and slices of 128 codes, of which a lane
// loads 32 (16 bytes: quarter q = lane / 16 of the slice), and multiplies on v_mfma_f32_16x16x32_f16: four steps of 32
// codes a slice, eight of each quarter.  A group's sum has to be scaled before the next group's joins it, so the steps
// must not mix groups.  With 128 codes a group or more they do not: the four steps chain, and four multiply-adds per
// slice (a lane has one channel and four tokens) take the group's sum into the total.  With 64 the first and second pair
// of quarters belong to different groups; two swaps of dwords between the halves of the wave sort them, and two more
// between neighbouring quarters for 32:
//   step j of quarter q multiplies codes 32 q + 8 j .. (128 and more)
//   64 (j / 2) + 32 (q % 2) + 16 (q / 2) + 8 (j % 2) ..   (64)
//   32 j + 8 q ..                                          (32)
// of the slice, and the tokens' operand follows.
template <int GROUP>
__device__ __forceinline__ int slice_place(int j, int q)
{
    return GROUP >= 128 ? 32 * q + 8 * j : GROUP == 64 ? 64 * (j >> 1) + 32 * (q & 1) + 16 * (q >> 1) + 8 * (j & 1) : 32 * j + 8 * q;
}

template <int GROUP>
__device__ __forceinline__ void sort_steps(uint32_t (&w)[4])
{
    typedef uint32_t v2u __attribute__((ext_vector_type(2)));
    if constexpr (GROUP <= 64) {
        const v2u a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
        const v2u b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
        w[0] = a[0], w[1] = b[0], w[2] = a[1], w[3] = b[1];
    }
    if constexpr (GROUP == 32) {
        const v2u a = __builtin_amdgcn_permlane16_swap(w[0], w[1], false, false);
        const v2u b = __builtin_amdgcn_permlane16_swap(w[2], w[3], false, false);
        w[0] = a[0], w[1] = a[1], w[2] = b[0], w[3] = b[1];
    }
}

// The steps of a slice's groups for one channel: one fp16, or the pair or four that lie side by side (2-byte aligned).
template <int GROUP>
struct SliceSteps {
    static constexpr int COUNT = GROUP >= 128 ? 1 : 128 / GROUP;
    struct __attribute__((packed, aligned(2))) Raw {
        _Float16 s[COUNT];
    } raw;
    __device__ __forceinline__ void load(const __half *row, int slice, int group)
    {
        raw = *reinterpret_cast<const Raw *>(row + (GROUP >= 128 ? 128 * slice / group : COUNT * slice));
    }
};

// 16 NS channels per workgroup and TT blocks of 16 tokens; the NW waves deal the slices of K among themselves and add up
// through LDS.  Everything goes global -> registers, D slices ahead.
template <int GROUP, int NS, int NW, int TT, int D>
__global__ __launch_bounds__(NW *kWave) void w4a16_grouped_skinny_kernel(const __half *__restrict__ X, int64_t ldx, int T, int K,
                                                                         const uint8_t *__restrict__ Qw,
                                                                         const __half *__restrict__ steps, int group, int N,
                                                                         __half *__restrict__ Y, int64_t ldy)
{
    constexpr int SUB = SliceSteps<GROUP>::COUNT, CHAIN = 4 / SUB;       // groups of a slice, steps of one
    __shared__ float red[NW][NS][TT][4][kWave];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const int l16 = lane & 15, q = lane >> 4;
    const int col0 = blockIdx.x * (16 * NS), groups = K / group, slices = (K + 127) / 128;

    // rows past the ends are clamped: their products are never stored
    const __half *x_row[TT], *s_row[NS];
    const uint8_t *w_row[NS];
#pragma unroll
    for (int i = 0; i < TT; ++i) x_row[i] = X + (int64_t)min(16 * i + l16, T - 1) * ldx;
#pragma unroll
    for (int c = 0; c < NS; ++c) {
        const int64_t n = min(col0 + 16 * c + l16, N - 1);
        w_row[c] = Qw + n * (K / 2);
        s_row[c] = steps + n * groups;
    }
    v4f total[NS][TT];
#pragma unroll
    for (int c = 0; c < NS; ++c)
#pragma unroll
        for (int i = 0; i < TT; ++i) total[c][i] = v4f{0.f, 0.f, 0.f, 0.f};

    uint4 w[D][NS];
    SliceSteps<GROUP> s[D][NS];
    v8h x[D][TT][4];
    auto fetch = [&](int set, int slice) {
#pragma unroll
        for (int c = 0; c < NS; ++c) {
            w[set][c] = *reinterpret_cast<const uint4 *>(w_row[c] + slice * 64 + 16 * q);
            s[set][c].load(s_row[c], slice, group);
        }
#pragma unroll
        for (int i = 0; i < TT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) x[set][i][j] = *reinterpret_cast<const v8h *>(x_row[i] + slice * 128 + slice_place<GROUP>(j, q));
    };
    uint32_t magic;                                    // 1024.0 in both halves, held in a vector register
    asm volatile("v_mov_b32 %0, 0x64006400" : "=v"(magic));
    auto multiply = [&](int set) {
#pragma unroll
        for (int c = 0; c < NS; ++c) {
            uint32_t d[4] = {w[set][c].x, w[set][c].y, w[set][c].z, w[set][c].w};
            sort_steps<GROUP>(d);
#pragma unroll
            for (int g = 0; g < SUB; ++g) {
                v4f part[TT];
#pragma unroll
                for (int j = g * CHAIN; j < (g + 1) * CHAIN; ++j) {
                    const v8h b = widen_codes_f16(d[j], magic);
#pragma unroll
                    for (int i = 0; i < TT; ++i) {
                        const v8h a = __builtin_bit_cast(v8h, interleave_halves(__builtin_bit_cast(uint4, x[set][i][j])));
                        part[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, j == g * CHAIN ? v4f{0.f, 0.f, 0.f, 0.f} : part[i], 0, 0, 0);
                    }
                }
                const float step = (float)s[set][c].raw.s[g];
#pragma unroll
                for (int i = 0; i < TT; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) total[c][i][e] = __builtin_fmaf(step, part[i][e], total[c][i][e]);
            }
        }
    };
    // wave w takes slices w, w + NW, ..; behind its last one that one is requested again, and dropped
    const int whole = K / 128;
    int S = wave;
    if (S < whole) {
        const int last = S + (whole - 1 - S) / NW * NW;
#pragma unroll
        for (int k = 0; k < D - 1; ++k) fetch(k, min(S + k * NW, last));
        while (true) {
            bool more = true;
#pragma unroll
            for (int k = 0; k < D; ++k) {
                fetch((k + D - 1) % D, min(S + (D - 1) * NW, last));
                multiply(k);
                S += NW;
                if (S > last) {
                    more = false;
                    break;
                }
            }
            if (!more) break;
        }
    }
    // half a slice at the end of a row (groups of 32 or 64): its second half is read as the first and multiplied by 0
    if (GROUP < 128 && whole < slices && wave == whole % NW) {
#pragma unroll
        for (int c = 0; c < NS; ++c) {
            w[0][c] = *reinterpret_cast<const uint4 *>(w_row[c] + whole * 64 + 16 * (q & 1));
#pragma unroll
            for (int g = 0; g < SUB; ++g) s[0][c].raw.s[g] = g < SUB / 2 ? __half2float(s_row[c][SUB * whole + g]) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < TT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[0][i][j] = *reinterpret_cast<const v8h *>(x_row[i] + whole * 128 + slice_place<GROUP>(j, q) % 64);
                if (j >= 2) x[0][i][j] = v8h{0, 0, 0, 0, 0, 0, 0, 0};
            }
        multiply(0);
    }

#pragma unroll
    for (int c = 0; c < NS; ++c)
#pragma unroll
        for (int i = 0; i < TT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) red[wave][c][i][e][lane] = total[c][i][e];
    __syncthreads();
    // 16 x 16 accumulator layout: lane holds channel l % 16, register e holds token 4 (l / 16) + e
    for (int idx = tid; idx < NS * TT * 4 * kWave; idx += NW * kWave) {
        const int ln = idx & (kWave - 1), e = (idx >> 6) & 3, i = (idx >> 8) % TT, c = (idx >> 8) / TT;
        float sum = 0.f;
#pragma unroll
        for (int v = 0; v < NW; ++v) sum += red[v][c][i][e][ln];
        const int t = 16 * i + 4 * (ln >> 4) + e, n = col0 + 16 * c + (ln & 15);
        if (t < T && n < N) Y[(int64_t)t * ldy + n] = __float2half_rn(sum);
    }
}

struct GroupedArgs {
    const __half *X;
    int64_t ldx;
    int T, K;
    const uint8_t *Qw;
    const __half *steps;
    int group, N;
    __half *Y;
    int64_t ldy;
    hipStream_t st;
};

template <int GROUP, int NS, int NW, int TT, int D>
sq_status launch_grouped_skinny(const GroupedArgs &a)
{
    hipLaunchKernelGGL((w4a16_grouped_skinny_kernel<GROUP, NS, NW, TT, D>), dim3((unsigned)((a.N + 16 * NS - 1) / (16 * NS))), dim3(NW * kWave),
                       0, a.st, a.X, a.ldx, a.T, a.K, a.Qw, a.steps, a.group, a.N, a.Y, a.ldy);
    return hipGetLastError() == hipSuccess ? SQ_OK : SQ_ERR_LAUNCH;
}

template <int GROUP>
sq_status launch_grouped_few(const GroupedArgs &a)
{
    if (a.T > 16) return launch_grouped_skinny<GROUP, 1, 8, 2, 2>(a);
    if (a.N >= 16384) return launch_grouped_skinny<GROUP, 2, 4, 1, 2>(a);
    return launch_grouped_skinny<GROUP, 1, 8, 1, 2>(a);
}

// One wave per output: a lane takes every 64th run of eight codes, multiplies in fp32 and adds its sum times the group's
// step; the lanes' sums are added at the end.
__global__ __launch_bounds__(256) void w4a16_grouped_dot_kernel(const __half *__restrict__ X, int64_t ldx, int T, int K,
                                                                const uint8_t *__restrict__ Qw, const __half *__restrict__ steps,
                                                                int group, int N, __half *__restrict__ Y, int64_t ldy)
{
    const int lane = threadIdx.x & (kWave - 1);
    const int64_t id = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
    const int64_t t = id / N;
    const int n = (int)(id - t * N);
    if (t >= T) return;
    const uint32_t *q = reinterpret_cast<const uint32_t *>(Qw + (int64_t)n * (K / 2));
    const __half *s = steps + (int64_t)n * (K / group), *x = X + t * ldx;
    float sum = 0.f;
    for (int u = lane; u < K / 8; u += kWave) {
        const uint32_t w = q[u];
        const v8h a = *reinterpret_cast<const v8h *>(x + 8 * u);
        float part = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) part = __builtin_fmaf((float)a[e], (float)((int32_t)(w << (28 - 4 * e)) >> 28), part);
        sum = __builtin_fmaf(part, __half2float(s[8 * u / group]), sum);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, kWave);
    if (lane == 0) Y[t * ldy + n] = __float2half_rn(sum);
}

}  // namespace

}  // namespace sq

extern "C" sq_status sq_w4a16_gemm_grouped(const void *X, int64_t T, int32_t K, int64_t ldx, const uint8_t *Qw,
                                           const void *steps, int32_t group, int32_t N, void *Y, int64_t ldy, void *stream)
{
    if (group != 32 && group != 64 && group != 128 && group != 256) return SQ_ERR_SHAPE;
    if (T < 0 || N < 0 || K <= 0 || (K % 64) != 0 || (K % group) != 0 || K > 131072) return SQ_ERR_SHAPE;
    if (T > (1 << 24) || ldx < K || ldy < N) return SQ_ERR_SHAPE;
    if (T == 0 || N == 0) return SQ_OK;
    if (!X || !Qw || !steps || !Y) return SQ_ERR_NULL;
    if (((uintptr_t)X & 15) || (ldx % 8) != 0 || ((uintptr_t)Qw & 15) || ((uintptr_t)Y & 1) || ((uintptr_t)steps & 1))
        return SQ_ERR_ALIGN;
    if (T <= 32) {
        const sq::GroupedArgs a = {static_cast<const __half *>(X), ldx, (int)T, K, Qw, static_cast<const __half *>(steps), group, N,
                                   static_cast<__half *>(Y), ldy, static_cast<hipStream_t>(stream)};
        if (group == 32) return sq::launch_grouped_few<32>(a);
        if (group == 64) return sq::launch_grouped_few<64>(a);
        return sq::launch_grouped_few<128>(a);
    }
    const int64_t blocks = (T * N + 3) / 4;
    if (blocks > 0x7FFFFFFF) return SQ_ERR_SHAPE;
    hipLaunchKernelGGL(sq::w4a16_grouped_dot_kernel, dim3((unsigned)blocks), dim3(256), 0, static_cast<hipStream_t>(stream),
                       static_cast<const __half *>(X), ldx, (int)T, K, Qw, static_cast<const __half *>(steps), group, N,
                       static_cast<__half *>(Y), ldy);
    return hipGetLastError() == hipSuccess ? SQ_OK : SQ_ERR_LAUNCH;
}

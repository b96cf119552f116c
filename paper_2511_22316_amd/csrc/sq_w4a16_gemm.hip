// sq_w4a16_gemm: fp16 activations times 4-bit weight codes on the fp16 matrix cores of gfx950, with
// the per-output-channel step applied in the epilogue -- the weight-only setting of the paper's
// appendix (weight-only quantization table): Eq. 1 with only the weight operand quantized, the
// weight operand being Flat(W~_R) = W^T R of Sec. 4.2, one K-contiguous row of codes per channel.
//
//   Y[t, n] = fp16( sw[n] * sum_k X[t, k] * Qw[n, k] )        fp32 accumulation
//
// Three kernels: a tile kernel for many tokens (w4a16_gemm_ring_kernel, sq_w4a16_tile.h) and two decode-shaped ones,
// for at most 32 tokens (w4a16_gemm_skinny_kernel) and for at most 16 whose rows fit in LDS
// (w4a16_gemm_xlds_kernel).  All widen the codes to fp16 in registers, exactly, with the
// magic-number form described at the widening functions there.
// sq_pack_w3 / sq_w3a16_gemm (W3A16 of the same table) live here too: the decode-shaped kernels
// with the codes in three bits each, expanded to nibbles in registers (w3_nibbles).
#include "sq_w4a16_tile.h"

#include <type_traits>

namespace sq {

namespace {

// 3-bit storage (sq_pack_w3): 32 codes are three dwords a0, a1, h.  Codes 8m .. 8m + 7 have their
// two low bits (of code + 4) at bits 4i + 2 (m % 2) of a[m / 2] and their high bit at bit 4i + m of
// h.  Returned: the dword whose nibble i holds code_{8m + i} + 4, i.e. the 4-bit layout the
// widening above takes.  Two to four instructions per eight codes.
template <int M>
__device__ __forceinline__ uint32_t w3_nibbles(uint32_t a0, uint32_t a1, uint32_t h)
{
    const uint32_t a = M < 2 ? a0 : a1;
    const uint32_t low = ((M & 1) ? (a >> 2) : a) & 0x33333333u;
    const uint32_t high = M == 0 ? (h << 2) : M == 1 ? (h << 1) : M == 2 ? h : (h >> 1);
    return low | (high & 0x44444444u);
}

// Decode-shaped kernel (T <= 32, K % 256 == 0): the product is one pass over the weight codes,
// 117 MB for 8 tokens at K = 8192, N = 28672, and the tile kernel would walk K in 224
// workgroups one tile at a time.  Here a workgroup owns 16 NS output channels and one block of 16
// tokens (v_mfma_f32_16x16x32_f16: lane = token or channel l % 16, its quarter q = l / 16 of the
// 32 contraction indices of a step); its NW waves split K in slices of 256 codes dealt round-robin
// and add their partial sums through LDS at the end.  Both operands go global -> registers, the
// next slice in flight while this one is multiplied.  Per slice a lane reads the 64 codes
// [64 q, 64 q + 64) of its channel rows (two 16-byte loads each, so that the four quarters of a
// wave consume whole 128-byte lines) and the same 64 activations of its token (128 contiguous
// bytes); dword d of chunk c, widened, is the operand of step (c, d), against the activations
// 32 c + 8 d .. + 7 of the lane's 64, put into the order 0 4 1 5 2 6 3 7 the widening produces.
// W3: the codes come in the 3-bit storage, 24 bytes per lane and slice instead of 32.
template <int NS, int NW, bool W3 = false>
__global__ __launch_bounds__(NW *kWave) void w4a16_gemm_skinny_kernel(
    const __half *__restrict__ X, int64_t ldx, int T, int K, const uint8_t *__restrict__ Qw,
    const float *__restrict__ sw, int N, __half *__restrict__ Y, int64_t ldy)
{
    constexpr int BN = 16 * NS;
    static_assert(NW * NS * 4 * kWave * 4 <= 64 * 1024, "partial sums must fit in static LDS");
    __shared__ float red[NW][NS][4][kWave];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const int l16 = lane & 15, q = lane >> 4;
    const int col0 = blockIdx.x * BN, t0 = blockIdx.y * 16;
    const int Kb = W3 ? 3 * (K / 8) : K / 2;                 // bytes of a row of codes
    constexpr int LANE_BYTES = W3 ? 24 : 32;                 // 64 codes
    constexpr int NLD = W3 ? 3 : 2;                          // loads per lane, channel block and slice
    typedef typename std::conditional<W3, uint2, uint4>::type CodeLoad;

    // rows past the ends are clamped: their products are never stored
    const __half *a_ptr = X + (int64_t)min(t0 + l16, T - 1) * ldx + q * 64;
    const uint8_t *b_ptr[NS];
#pragma unroll
    for (int j = 0; j < NS; ++j) b_ptr[j] = Qw + (int64_t)min(col0 + 16 * j + l16, N - 1) * Kb + q * LANE_BYTES;

    v4f acc[NS];
#pragma unroll
    for (int j = 0; j < NS; ++j) acc[j] = v4f{0.f, 0.f, 0.f, 0.f};

    uint4 ra[2][8];
    CodeLoad rb[2][NS][NLD];
    const int slices = K / 256;
#define SQ_W16_FETCH(BUF, S)                                                                         \
    do {                                                                                             \
        _Pragma("unroll") for (int j = 0; j < NS; ++j)                                               \
            _Pragma("unroll") for (int c = 0; c < NLD; ++c)                                          \
                rb[BUF][j][c] = *reinterpret_cast<const CodeLoad *>(b_ptr[j] + (S) * (4 * LANE_BYTES) + \
                                                                    (int)sizeof(CodeLoad) * c);     \
        _Pragma("unroll") for (int u = 0; u < 8; ++u)                                                \
            ra[BUF][u] = *reinterpret_cast<const uint4 *>(a_ptr + (S) * 256 + 8 * u);                \
    } while (0)
#define SQ_W16_MULTIPLY(BUF)                                                                         \
    do {                                                                                             \
        _Pragma("unroll") for (int c = 0; c < 2; ++c)                                                \
            _Pragma("unroll") for (int d = 0; d < 4; ++d) {                                          \
                const v8h a = __builtin_bit_cast(v8h, interleave_halves(ra[BUF][4 * c + d]));        \
                _Pragma("unroll") for (int j = 0; j < NS; ++j)                                       \
                    acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, codes_of(rb[BUF][j], c, d), acc[j], 0, 0, 0); \
            }                                                                                        \
    } while (0)

    // codes 32c + 8d .. + 7 of the lane's 64 as fp16, in the order interleave_halves gives the tokens
    uint32_t magic;                                    // 1024.0 in both halves, held in a vector register
    asm volatile("v_mov_b32 %0, 0x64006400" : "=v"(magic));
    auto codes_of = [magic](const CodeLoad(&r)[NLD], int c, int d) -> v8h {
        if constexpr (W3) {
            // six dwords: (a0, a1, h) of codes 0 .. 31, then of codes 32 .. 63
            const uint32_t w[6] = {r[0].x, r[0].y, r[1].x, r[1].y, r[2].x, r[2].y};
            const uint32_t a0 = w[3 * c], a1 = w[3 * c + 1], h = w[3 * c + 2];
            const uint32_t n = d == 0 ? w3_nibbles<0>(a0, a1, h) : d == 1 ? w3_nibbles<1>(a0, a1, h)
                             : d == 2 ? w3_nibbles<2>(a0, a1, h) : w3_nibbles<3>(a0, a1, h);
            return widen_codes_f16<true>(n, magic);
        } else {
            const uint4 w4 = r[c];
            return widen_codes_f16(d == 0 ? w4.x : d == 1 ? w4.y : d == 2 ? w4.z : w4.w, magic);
        }
    };
    // wave w takes slices w, w + NW, w + 2 NW, ...; two register sets alternate
    int S = wave;
    if (S < slices) SQ_W16_FETCH(0, S);
    while (S < slices) {
        if (S + NW < slices) SQ_W16_FETCH(1, S + NW);
        SQ_W16_MULTIPLY(0);
        S += NW;
        if (S >= slices) break;
        if (S + NW < slices) SQ_W16_FETCH(0, S + NW);
        SQ_W16_MULTIPLY(1);
        S += NW;
    }
#undef SQ_W16_FETCH
#undef SQ_W16_MULTIPLY

#pragma unroll
    for (int j = 0; j < NS; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) red[wave][j][r][lane] = acc[j][r];
    __syncthreads();
    // 16 x 16 accumulator layout: lane holds channel l % 16, register r holds token 4 (l / 16) + r
    for (int idx = tid; idx < NS * 4 * kWave; idx += NW * kWave) {
        const int ln = idx & (kWave - 1), r = (idx >> 6) & 3, j = idx >> 8;
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) sum += red[w][j][r][ln];
        const int t = t0 + 4 * (ln >> 4) + r, n = col0 + 16 * j + (ln & 15);
        if (t < T && n < N) Y[(int64_t)t * ldy + n] = __float2half_rn(sum * sw[n]);
    }
}

template <int NS, int NW, bool W3 = false>
sq_status launch_w4a16_skinny(const __half *X, int64_t ldx, int T, int K, const uint8_t *Qw, const float *sw, int N,
                              __half *Y, int64_t ldy, hipStream_t st)
{
    hipLaunchKernelGGL((w4a16_gemm_skinny_kernel<NS, NW, W3>), dim3((unsigned)((N + 16 * NS - 1) / (16 * NS)), (unsigned)((T + 15) / 16)),
                       dim3(NW * kWave), 0, st, X, ldx, T, K, Qw, sw, N, Y, ldy);
    return hipGetLastError() == hipSuccess ? SQ_OK : SQ_ERR_LAUNCH;
}

// ---- at most 16 tokens whose rows fit in LDS, many channels ---------------------------------
// In the kernel above every workgroup fetches the token rows again for each slice (twice the
// bytes of its weight codes when 16-bit rows meet 4-bit codes), and the fewer channels a workgroup
// owns the more of that traffic there is.  Here a workgroup of eight waves copies the rows into
// LDS once (each 16-byte chunk already in the order the widened codes take) and every wave then
// works alone: it owns blocks of 16 channels over the whole of K, slice after slice, with the
// codes of the next D slices in flight in a ring of registers and the token chunks of the next
// slice read from LDS while this one is multiplied.  No wave waits for another after the copy:
// no partial sums, no barriers.
// One workgroup per CU (the rows take most of the LDS); block b belongs to workgroup b % grid,
// wave (b / grid) % 8.
constexpr int kXldsRowPad = 16;        // bytes; sixteen rows then start in sixteen different 16-byte bank groups
constexpr int kXldsWaves = 8;
// 16-byte chunks of the rows per thread, at most
constexpr int kXldsChunks = (kMaxDynamicLds / 16 + kXldsWaves * kWave - 1) / (kXldsWaves * kWave);

// does the walk over K begin with another round in neighbouring workgroups?  (see the kernel)
__host__ __device__ constexpr bool w4a16_xlds_turns(int K) { return K % 8192 == 0 && K < 32768; }

// TURNS: it may
template <bool W3, int D, bool TURNS>
__global__ __launch_bounds__(kXldsWaves *kWave) void w4a16_gemm_xlds_kernel(
    const __half *__restrict__ X, int64_t ldx, int T, int K, const uint8_t *__restrict__ Qw,
    const float *__restrict__ sw, int N, __half *__restrict__ Y, int64_t ldy)
{
    static_assert(D % 2 == 0, "the token chunks alternate between two register sets");
    constexpr int NT = kXldsWaves * kWave;
    extern __shared__ uint4 xlds_u4[];
    char *xs = reinterpret_cast<char *>(xlds_u4);
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const int l16 = lane & 15, q = lane >> 4;
    const int stride = 2 * K + kXldsRowPad;
    const int Kb = W3 ? 3 * (K / 8) : K / 2;                 // bytes of a row of codes
    constexpr int NLD = W3 ? 3 : 2;                          // loads per lane and slice
    typedef typename std::conditional<W3, uint2, uint4>::type CodeLoad;
    const int slices = K / 256, nblocks = (N + 15) / 16;
    const int first = blockIdx.x + gridDim.x * wave, step = gridDim.x * kXldsWaves;
    const int my_blocks = first < nblocks ? (nblocks - first + step - 1) / step : 0;

    // A lane holds the channel l16 of a block and a quarter q of a slice, codes 64 q .. 64 q + 63:
    // bytes 32q .. 32q + 31 of the slice's 128, or, in the 3-bit storage, bytes 24q .. 24q + 23
    // of its 96.  (Reading 64 contiguous bytes of a row per load instruction instead, or even
    // 1 KB contiguous per instruction from a re-tiled copy, changed nothing: 32.8 / 32.0 us.)
    // The loads of a round of D slices are issued D slices ahead, into the registers the round
    // has just consumed; slices % D == 0 (the launcher sees to it), so a round never straddles two
    // blocks and the loop body has no branch: the compiler's count of outstanding loads stays
    // exact.  Behind the last round of the last block that same round is requested once more.
    CodeLoad rb[D][NLD];
    auto row_of = [&](int bi) { return Qw + (int64_t)min(16 * (int64_t)(first + bi * step) + l16, (int64_t)N - 1) * Kb; };
    auto issue = [&](CodeLoad(&r)[NLD], const uint8_t *row, int S) {
        if constexpr (W3) {
#pragma unroll
            for (int c = 0; c < 3; ++c) r[c] = *reinterpret_cast<const uint2 *>(row + S * 96 + 24 * q + 8 * c);
        } else {
#pragma unroll
            for (int c = 0; c < 2; ++c) r[c] = *reinterpret_cast<const uint4 *>(row + S * 128 + 32 * q + 16 * c);
        }
    };

    // The token rows are requested first, 16-byte chunk by chunk (at most kXldsChunks per thread:
    // what fits in LDS), then the first D slices of codes; loads complete in order, so the rows
    // can be written to LDS while the codes are still on their way.  All requests are
    // unconditional (clamped), which keeps the compiler's count of outstanding loads exact.
    // Where rows of codes lie a multiple of 4 KB apart, every wave of the chip at the same place of its row means that the requests of
    // a moment meet in a few memory channels.  The walk over K begins with another round in neighbouring workgroups there, which
    // sit on different XCDs (N = 28672, us: T = 8, K = 8192 31.6 -> 27.7; T = 1, K = 16384 50.8 -> 46.2, K = 24576 72.4 -> 63.5; by slices
    // instead of whole rounds, or by wave: slower again).  Not from 16 KB on (T = 1: K = 32768 99 / 123, K = 65536 189 / 195), nor
    // elsewhere (T = 1, N = 32000: K = 3072 14.5 / 14.7, K = 4096 19.3 / 19.6, K = 5120 20.0 / 21.2; K = 14336, N = 16384 26.8 / 27.4).
    // The three-bit storage, whose rows of these K lie 3 KB and more apart, goes along for the same order of additions (T = 1:
    // N = 16384, K = 8192 17.4 -> 17.0, K = 24576 37.5 -> 35.8; N = 50000, K = 8192 46.7 / 48.9).
    // A channel's sum is rounded in the order of its workgroup's walk, so its last bit may depend on the channel's number there.
    const int turn = TURNS && w4a16_xlds_turns(K) ? (int)blockIdx.x % (slices / D) * D : 0;
    const int chunks_per_row = K / 8, chunks = T * chunks_per_row;
    {
        uint4 xv[kXldsChunks];
#pragma unroll
        for (int u = 0; u < kXldsChunks; ++u) {
            const int j = min(tid + NT * u, chunks - 1);
            xv[u] = *reinterpret_cast<const uint4 *>(X + (int64_t)(j / chunks_per_row) * ldx + 8 * (j % chunks_per_row));
        }
        const uint8_t *row0 = row_of(0);             // a wave without blocks requests (and drops) a valid row
#pragma unroll
        for (int i = 0; i < D; ++i) issue(rb[i], row0, turn + i);
#pragma unroll
        for (int u = 0; u < kXldsChunks; ++u) {
            const int j = tid + NT * u;
            if (j < chunks)
                *reinterpret_cast<uint4 *>(xs + (j / chunks_per_row) * stride + 16 * (j % chunks_per_row)) =
                    interleave_halves(xv[u]);
        }
    }
    __syncthreads();

    uint32_t magic;                                    // 1024.0 in both halves, held in a vector register
    asm volatile("v_mov_b32 %0, 0x64006400" : "=v"(magic));
    // this lane's token row (rows past T repeat the last one: their products are never stored)
    // and the offset of its first chunk inside a slice.  Chunk j of the lane's eight per slice:
    // codes 64 q + 8 j .. + 7 of the slice.
    const char *xa = xs + min(l16, T - 1) * stride + 128 * q;
    auto read_tokens = [&](v8h(&a)[8], int S) {
        const char *xi = xa + S * 512;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            a[j] = *reinterpret_cast<const v8h *>(xi + 16 * j);
    };
    v4f acc0, acc1;
    auto multiply = [&](const CodeLoad(&r)[NLD], const v8h(&a)[8]) {
        if constexpr (W3) {
            // (a0, a1, h) of codes 0 .. 31 and of codes 32 .. 63 of the lane's 64
            const uint32_t w[6] = {r[0].x, r[0].y, r[1].x, r[1].y, r[2].x, r[2].y};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t a0 = w[3 * h], a1 = w[3 * h + 1], hb = w[3 * h + 2];
                const uint32_t nib[4] = {w3_nibbles<0>(a0, a1, hb), w3_nibbles<1>(a0, a1, hb),
                                         w3_nibbles<2>(a0, a1, hb), w3_nibbles<3>(a0, a1, hb)};
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    v4f &acc = (m & 1) ? acc1 : acc0;
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[4 * h + m], widen_codes_f16<true>(nib[m], magic), acc, 0, 0, 0);
                }
            }
        } else {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const uint32_t w[4] = {r[c].x, r[c].y, r[c].z, r[c].w};
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    v4f &acc = (d & 1) ? acc1 : acc0;
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[4 * c + d], widen_codes_f16(w[d], magic), acc, 0, 0, 0);
                }
            }
        }
    };
    v8h ta[2][8];                                      // token chunks of this slice and of the next
    read_tokens(ta[0], TURNS ? turn : 0);
    for (int bi = 0; bi < my_blocks; ++bi) {
        const int n = 16 * (first + bi * step) + l16;
        const float step_n = sw[min(n, N - 1)];
        const uint8_t *row = row_of(bi);
        const uint8_t *row_after = row_of(bi + 1 < my_blocks ? bi + 1 : bi);
        acc0 = v4f{0.f, 0.f, 0.f, 0.f};
        acc1 = v4f{0.f, 0.f, 0.f, 0.f};
        int place = turn;
        for (int done = 0; done < slices; done += D) {
            const bool wrap = done + D >= slices;          // the round D slices ahead opens the next block
            const uint8_t *row_n = wrap ? row_after : row;
            const int S0 = TURNS ? place : done;
            const int after = S0 + D == slices ? 0 : S0 + D;       // behind the last round of a block: its first one, `turn`, again
            // (without turns the same said by `wrap`, of which the compiler makes another loop: T = 1, K = 5120, N = 32000 20.9 / 20.0 us)
            const int S_n = TURNS ? (wrap && bi + 1 == my_blocks ? S0 : after) : wrap ? (bi + 1 < my_blocks ? 0 : S0) : S0 + D;
#pragma unroll
            for (int i = 0; i < D; ++i) {
                // the slice after this one (the token rows are the same for every block)
                read_tokens(ta[(i + 1) & 1], TURNS ? (i + 1 == D ? after : S0 + i + 1) : (i + 1 == D && wrap) ? 0 : S0 + i + 1);
                multiply(rb[i], ta[i & 1]);
                issue(rb[i], row_n, S_n + i);
                // keep the requests here, one slice behind another: collected at the end of the
                // round (where the scheduler puts them) they would all be waited for at once
                __builtin_amdgcn_sched_barrier(0);
            }
            place = after;
        }
        // 16 x 16 accumulator layout: lane holds channel l16, register r holds token 4 q + r
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
            const int t = 4 * q + r4;
            if (t < T && n < N) Y[(int64_t)t * ldy + n] = __float2half_rn((acc0[r4] + acc1[r4]) * step_n);
        }
    }
}

// T <= 16, K % 1024 == 0 (rounds of at least four slices), the rows fit: T (2K + 16) bytes of LDS.
template <bool W3>
sq_status launch_w4a16_xlds(const __half *X, int64_t ldx, int T, int K, const uint8_t *Qw, const float *sw, int N,
                            __half *Y, int64_t ldy, hipStream_t st)
{
    const int nblocks = (N + 15) / 16;
    const int grid = nblocks < 256 ? nblocks : 256;
    const size_t lds = (size_t)T * (2 * K + kXldsRowPad);
    // Eight slices in flight per wave where the slices of a row come in eights (K % 2048 == 0, which holds where walks turn), else
    // four.  The kernel whose walks may turn is the faster one for four bits anyway (T = 1, N = 16384, K = 2048 9.3 -> 8.9 us,
    // K = 6144 15.9 -> 15.8), for three it is not (T = 1, N = 32000, K = 14336 41.8 / 43.8, K = 32768 94 / 100).
    auto launch = [&](auto kernel) {
        if (!allow_large_lds(reinterpret_cast<const void *>(kernel))) return SQ_ERR_LAUNCH;
        hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(kXldsWaves * kWave), lds, st, X, ldx, T, K, Qw, sw, N, Y, ldy);
        return hipGetLastError() == hipSuccess ? SQ_OK : SQ_ERR_LAUNCH;
    };
    if ((K / 256) % 8 != 0) return launch(w4a16_gemm_xlds_kernel<W3, 4, false>);
    if constexpr (W3)
        if (!w4a16_xlds_turns(K)) return launch(w4a16_gemm_xlds_kernel<W3, 8, false>);
    return launch(w4a16_gemm_xlds_kernel<W3, 8, true>);
}

// does the kernel above take the shape?  Enough blocks of 16 channels that every CU gets several waves
inline bool w4a16_xlds_covers(int64_t T, int K, int N)
{
    return T <= 16 && (K % 1024) == 0 && T * (int64_t)(2 * K + kXldsRowPad) <= kMaxDynamicLds && N >= 16 * 256 * 4;
}

// Nibble codes [N, K/2] (two's complement, every code in [-4, 3]) -> 3-bit storage [N, 3K/8].
// One thread per 32 codes: 16 bytes in, 12 bytes out.  (nibble ^ 4) & 7 is code + 4.
__global__ __launch_bounds__(256) void pack_w3_kernel(const uint8_t *__restrict__ Qw, int64_t units,
                                                      uint32_t *__restrict__ Qw3)
{
    const int64_t u = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (u >= units) return;
    const uint4 v = *reinterpret_cast<const uint4 *>(Qw + 16 * u);
    const uint32_t x0 = v.x ^ 0x44444444u, x1 = v.y ^ 0x44444444u, x2 = v.z ^ 0x44444444u, x3 = v.w ^ 0x44444444u;
    const uint32_t lo = 0x33333333u, hi = 0x44444444u;
    Qw3[3 * u + 0] = (x0 & lo) | ((x1 & lo) << 2);
    Qw3[3 * u + 1] = (x2 & lo) | ((x3 & lo) << 2);
    Qw3[3 * u + 2] = ((x0 & hi) >> 2) | ((x1 & hi) >> 1) | (x2 & hi) | ((x3 & hi) << 1);
}

}  // namespace

}  // namespace sq

extern "C" sq_status sq_pack_w3(const uint8_t *Qw, int32_t K, int32_t N, uint8_t *Qw3, void *stream)
{
    if (N < 0 || K <= 0 || (K % 64) != 0 || K > 131072) return SQ_ERR_SHAPE;
    if (N == 0) return SQ_OK;
    if (!Qw || !Qw3) return SQ_ERR_NULL;
    if (((uintptr_t)Qw & 15) || ((uintptr_t)Qw3 & 7)) return SQ_ERR_ALIGN;
    const int64_t units = (int64_t)N * (K / 32);
    hipLaunchKernelGGL(sq::pack_w3_kernel, dim3((unsigned)((units + 255) / 256)), dim3(256), 0,
                       static_cast<hipStream_t>(stream), Qw, units, reinterpret_cast<uint32_t *>(Qw3));
    return hipGetLastError() == hipSuccess ? SQ_OK : SQ_ERR_LAUNCH;
}

extern "C" sq_status sq_w3a16_gemm(const void *X, int64_t T, int32_t K, int64_t ldx, const uint8_t *Qw3,
                                   const float *sw, int32_t N, void *Y, int64_t ldy, void *stream)
{
    if (T < 0 || N < 0 || K <= 0 || (K % 256) != 0 || K > 131072) return SQ_ERR_SHAPE;
    if (T > SQ_W3A16_MAX_ROWS || ldx < K || ldy < N) return SQ_ERR_SHAPE;       // 16 tokens per grid row
    if (T == 0 || N == 0) return SQ_OK;
    if (!X || !Qw3 || !sw || !Y) return SQ_ERR_NULL;
    if (((uintptr_t)X & 15) || (ldx % 8) != 0 || ((uintptr_t)Qw3 & 7) || ((uintptr_t)Y & 1) || ((uintptr_t)sw & 3))
        return SQ_ERR_ALIGN;
    const hipStream_t s0 = static_cast<hipStream_t>(stream);
    const __half *X0 = static_cast<const __half *>(X);
    if (sq::w4a16_xlds_covers(T, K, N))
        return sq::launch_w4a16_xlds<true>(X0, ldx, (int)T, K, Qw3, sw, N, static_cast<__half *>(Y), ldy, s0);
    if (N >= 64 * 384) return sq::launch_w4a16_skinny<4, 4, true>(X0, ldx, (int)T, K, Qw3, sw, N, static_cast<__half *>(Y), ldy, s0);
    return sq::launch_w4a16_skinny<2, 8, true>(X0, ldx, (int)T, K, Qw3, sw, N, static_cast<__half *>(Y), ldy, s0);
}

extern "C" sq_status sq_w4a16_gemm(const void *X, int64_t T, int32_t K, int64_t ldx, const uint8_t *Qw,
                                   const float *sw, int32_t N, void *Y, int64_t ldy, void *stream)
{
    if (T < 0 || N < 0 || K <= 0 || (K % 64) != 0 || K > 131072) return SQ_ERR_SHAPE;
    if (T > (1 << 24) || ldx < K || ldy < N) return SQ_ERR_SHAPE;
    if (T == 0 || N == 0) return SQ_OK;
    if (!X || !Qw || !sw || !Y) return SQ_ERR_NULL;
    if (((uintptr_t)X & 15) || (ldx % 8) != 0 || ((uintptr_t)Qw & 15) || ((uintptr_t)Y & 1) || ((uintptr_t)sw & 3))
        return SQ_ERR_ALIGN;
    // At most 32 tokens: one pass over the weights (two token blocks above 16 tokens read them twice,
    // the second time mostly out of the caches; beyond that the tile kernel is the better choice).
    // Launch shapes as in the W4A4 decode-shaped kernel: about eight waves on every CU.
    if (T <= 32 && (K % 256) == 0 && sq::debug_option(SQ_DEBUG_W4A16_LAUNCH_SHAPE) == 0) {
        const hipStream_t s0 = static_cast<hipStream_t>(stream);
        const __half *X0 = static_cast<const __half *>(X);
        if (sq::w4a16_xlds_covers(T, K, N))
            return sq::launch_w4a16_xlds<false>(X0, ldx, (int)T, K, Qw, sw, N, static_cast<__half *>(Y), ldy, s0);
        if (N >= 64 * 384) return sq::launch_w4a16_skinny<4, 4>(X0, ldx, (int)T, K, Qw, sw, N, static_cast<__half *>(Y), ldy, s0);
        return sq::launch_w4a16_skinny<2, 8>(X0, ldx, (int)T, K, Qw, sw, N, static_cast<__half *>(Y), ldy, s0);
    }
    // Many tokens: 256 x 256 tiles (eight waves) when there are enough of them to fill the CUs, else
    // 128 x 256 tiles (four multiplying waves and four loading waves: with the loads in the multiplying
    // waves this tile took 69.1 instead of 67.2 us on 2048 x 4096 x 4096 and 177 instead of 165 us at
    // K = 11008).
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const __half *Xh = static_cast<const __half *>(X);
    __half *Yh = static_cast<__half *>(Y);
    const int shape = sq::debug_option(SQ_DEBUG_W4A16_LAUNCH_SHAPE);
    const int64_t tiles_large = ((T + 255) / 256) * ((N + 255) / 256);
    // Few tiles: 64 x 128, then 128 x 128 tiles with two K groups of four waves while one workgroup per CU takes the whole
    // product (us, 128 x 256 tiles / here: T = 100, K = N = 4096 40.2 / 19.9; T = 333 42.1 / 22.5; T = 100, K = 11008, N = 13824
    // 100 / 57.5; T = 600, K = N = 4096 42.0 / 30.9; T = 333, N = 9000 44.3 / 35.8; T = 1000, N = 4096 45.0 / 39.9; from the next
    // round of workgroups on the larger tiles win: T = 600, N = 9000 53.4 / 67.2).  A K tile costs such a wave what its
    // widening takes to issue, so its fragments are tall (two or four token blocks to one of channels: T = 333, K = N = 4096 with
    // the fragments of the 64 x 128 tile the other way round 29.9), and two waves per SIMD share it; four K groups gain
    // little more (22.2).
    const int64_t tiles_64x128 = ((T + 63) / 64) * ((N + 127) / 128), tiles_128 = ((T + 127) / 128) * ((N + 127) / 128);
    const bool two_k_groups = K % 128 == 0;
    if (two_k_groups && (shape == 3 || (shape == 0 && tiles_64x128 <= 256)))
        return sq::launch_w4a16_ring<1, 4, 2, 1, 1, 64, 0, 2>(Xh, ldx, (int)T, K, Qw, sw, N, Yh, ldy, st);
    if (two_k_groups && (shape == 4 || (shape == 0 && tiles_128 <= 256)))
        return sq::launch_w4a16_ring<1, 4, 4, 1, 1, 64, 0, 2>(Xh, ldx, (int)T, K, Qw, sw, N, Yh, ldy, st);
    if (shape == 2 || (shape != 1 && tiles_large >= 192))
        return sq::launch_w4a16_ring<2, 4, 4, 2, 1, 64>(Xh, ldx, (int)T, K, Qw, sw, N, Yh, ldy, st);
    return sq::launch_w4a16_ring<1, 4, 4, 2, 1, 64, 4>(Xh, ldx, (int)T, K, Qw, sw, N, Yh, ldy, st);
}

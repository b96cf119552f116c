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

// 16 NS channels and TT blocks of 16 tokens per workgroup; the NW waves deal the slices of K among themselves and add up
// through LDS.  Everything goes global -> registers, one unit of H slices ahead.  The steps of a unit are one load: every
// load of a wave touches 16 rows, and their number is what this kernel costs beside the bytes.
template <int GROUP, int NS, int NW, int TT, int H>
__global__ __launch_bounds__(NW *kWave) void w4a16_grouped_skinny_kernel(const __half *__restrict__ X, int64_t ldx, int T, int K,
                                                                         const uint8_t *__restrict__ Qw,
                                                                         const __half *__restrict__ steps, int N,
                                                                         __half *__restrict__ Y, int64_t ldy)
{
    constexpr int SUB = GROUP >= 128 ? 1 : 128 / GROUP, CHAIN = 4 / SUB;       // groups of a slice, steps of one
    constexpr int SPU = H * 128 < GROUP ? 1 : H * 128 / GROUP;                 // groups of a unit
    struct __attribute__((packed, aligned(2))) UnitSteps {
        _Float16 s[SPU];
    };
    __shared__ float red[NW][NS][TT][4][kWave];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const int l16 = lane & 15, q = lane >> 4;
    const int col0 = blockIdx.x * (16 * NS), t0 = blockIdx.y * (16 * TT), groups = K / GROUP, units = (K + 128 * H - 1) / (128 * H);

    // rows past the ends are clamped: their products are never stored
    const __half *x_row[TT], *s_row[NS];
    const uint8_t *w_row[NS];
#pragma unroll
    for (int i = 0; i < TT; ++i) x_row[i] = X + (int64_t)min(t0 + 16 * i + l16, T - 1) * ldx;
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

    auto step_at = [&](int unit) { return unit * (128 * H) / GROUP; };
    uint4 w[2][NS][H];
    UnitSteps s[2][NS];
    v8h x[2][TT][H][4];
    auto fetch = [&](int set, int unit) {
#pragma unroll
        for (int c = 0; c < NS; ++c) {
#pragma unroll
            for (int h = 0; h < H; ++h) w[set][c][h] = *reinterpret_cast<const uint4 *>(w_row[c] + unit * (64 * H) + 64 * h + 16 * q);
            s[set][c] = *reinterpret_cast<const UnitSteps *>(s_row[c] + step_at(unit));
        }
#pragma unroll
        for (int i = 0; i < TT; ++i)
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
                for (int j = 0; j < 4; ++j) x[set][i][h][j] = *reinterpret_cast<const v8h *>(x_row[i] + unit * (128 * H) + 128 * h + slice_place<GROUP>(j, q));
    };
    // the unit that ends behind the row: codes from inside it, tokens and steps of zero
    auto fetch_last = [&](int unit) {
#pragma unroll
        for (int c = 0; c < NS; ++c) {
#pragma unroll
            for (int h = 0; h < H; ++h) w[0][c][h] = *reinterpret_cast<const uint4 *>(w_row[c] + min(unit * (64 * H) + 64 * h + 16 * q, K / 2 - 16));
#pragma unroll
            for (int g = 0; g < SPU; ++g)
                s[0][c].s[g] = step_at(unit) + g < groups ? (_Float16)__half2float(s_row[c][step_at(unit) + g]) : (_Float16)0.f;
        }
#pragma unroll
        for (int i = 0; i < TT; ++i)
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int at = unit * (128 * H) + 128 * h + slice_place<GROUP>(j, q);
                    x[0][i][h][j] = v8h{0, 0, 0, 0, 0, 0, 0, 0};
                    if (at < K) x[0][i][h][j] = *reinterpret_cast<const v8h *>(x_row[i] + at);
                }
    };
    uint32_t magic;                                    // 1024.0 in both halves, held in a vector register
    asm volatile("v_mov_b32 %0, 0x64006400" : "=v"(magic));
    auto multiply = [&](int set) {
#pragma unroll
        for (int h = 0; h < H; ++h) {
            v8h a[TT][4];
#pragma unroll
            for (int i = 0; i < TT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) a[i][j] = __builtin_bit_cast(v8h, interleave_halves(__builtin_bit_cast(uint4, x[set][i][h][j])));
#pragma unroll
            for (int c = 0; c < NS; ++c) {
                uint32_t d[4] = {w[set][c][h].x, w[set][c][h].y, w[set][c][h].z, w[set][c][h].w};
                sort_steps<GROUP>(d);
#pragma unroll
                for (int g = 0; g < SUB; ++g) {
                    v4f part[TT];
#pragma unroll
                    for (int j = g * CHAIN; j < (g + 1) * CHAIN; ++j) {
                        const v8h b = widen_codes_f16(d[j], magic);
#pragma unroll
                        for (int i = 0; i < TT; ++i)
                            part[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[i][j], b, j == g * CHAIN ? v4f{0.f, 0.f, 0.f, 0.f} : part[i], 0, 0, 0);
                    }
                    const float step = (float)s[set][c].s[h * SPU / H + g];
#pragma unroll
                    for (int i = 0; i < TT; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) total[c][i][e] = __builtin_fmaf(step, part[i][e], total[c][i][e]);
                }
            }
        }
    };
    // wave w takes units w, w + NW, ..; two register sets alternate
    const int whole = K / (128 * H);
    int P = wave;
    if (P < whole) fetch(0, P);
    while (P < whole) {
        if (P + NW < whole) fetch(1, P + NW);
        multiply(0);
        P += NW;
        if (P >= whole) break;
        if (P + NW < whole) fetch(0, P + NW);
        multiply(1);
        P += NW;
    }
    if (whole < units && wave == whole % NW) {
        fetch_last(whole);
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
        const int t = t0 + 16 * i + 4 * (ln >> 4) + e, n = col0 + 16 * c + (ln & 15);
        if (t < T && n < N) Y[(int64_t)t * ldy + n] = __float2half_rn(sum);
    }
}

// ---- at most 16 tokens whose rows fit in LDS ------------------------------------------------------
// In the kernel above every workgroup fetches the token rows for itself, twice to sixteen times the bytes of the codes it
// reads.  Here a workgroup copies the rows into LDS once (each 16-byte chunk already in the order the widened codes
// take).  It owns blocks of 16 channels (b % grid), whose rounds of NR slices its NW waves share evenly, one run of rounds
// each; what a run leaves of a block is added up at the end, in the order of the waves.  A slice of the next round is
// requested when this round's is done, so a wave has NR KB of codes in flight at all times, across the ends of blocks too.
// The steps of a round are one load: every quarter of a wave takes a quarter of them, and swaps hand them to the others.
// (A step load per slice touches 16 cache lines for two bytes of each, which the codes have pushed out of the CU's cache
// again by the next slice: 43 us at T = 8, K = 8192, N = 28672, groups of 128; all steps of a round in every quarter
// 33.5, and 46 with groups of 32.)  Where K is no whole number of rounds the rows go on with zeros, and the last slice of codes is taken
// again with them and with steps of zero.
constexpr int kRowPad = 16;            // bytes; sixteen rows then start in sixteen different 16-byte bank groups
inline __host__ __device__ int row_bytes(int K, int per_round) { return 2 * ((K + per_round - 1) / per_round * per_round) + kRowPad; }

// A dword of every quarter of the wave, in all of them.
__device__ __forceinline__ void all_quarters(uint32_t v, uint32_t (&of)[4])
{
    typedef uint32_t v2u __attribute__((ext_vector_type(2)));
    const v2u halves = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    const uint32_t lower = halves[0], upper = halves[1];
    const v2u a = __builtin_amdgcn_permlane16_swap(lower, lower, false, false);
    const v2u b = __builtin_amdgcn_permlane16_swap(upper, upper, false, false);
    of[0] = a[0], of[1] = a[1], of[2] = b[0], of[3] = b[1];
}

template <int GROUP, int NW, int NR>
__global__ __launch_bounds__(NW *kWave) void w4a16_grouped_rows_kernel(const __half *__restrict__ X, int64_t ldx, int T, int K,
                                                                       const uint8_t *__restrict__ Qw, const __half *__restrict__ steps,
                                                                       int N, __half *__restrict__ Y, int64_t ldy)
{
    static_assert(NR % 2 == 0, "the token chunks alternate between two register sets");
    constexpr int NT = NW * kWave, SUB = GROUP >= 128 ? 1 : 128 / GROUP, CHAIN = 4 / SUB;
    constexpr int SPR = NR * 128 / GROUP, PIECE = SPR < 4 ? 1 : SPR / 4;       // steps per round, and of a quarter
    constexpr int CHUNKS = (kMaxDynamicLds / 16 + NT - 1) / NT;                // 16-byte chunks of the rows per thread, at most
    struct __attribute__((packed, aligned(2))) Piece {
        unsigned short s[PIECE];
    };
    extern __shared__ uint4 rows_u4[];
    char *xs = reinterpret_cast<char *>(rows_u4);
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int l16 = lane & 15, q = lane >> 4;
    const int stride = row_bytes(K, NR * 128), slices = K / 128, groups = K / GROUP, rounds = (slices + NR - 1) / NR;
    const int blocks = (N + 15) / 16, mine = (blocks - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x;
    // this wave's run: rounds [begin, end) of the workgroup's mine * rounds, numbered block after block
    const int64_t all = (int64_t)mine * rounds;
    const int begin = (int)(all * wave / NW), end = (int)(all * (wave + 1) / NW);
    // Neighbouring workgroups begin their blocks with another round: the requests of a moment would meet in a few memory
    // channels where rows of codes lie a multiple of 4 KB apart (T = 8, K = 8192, N = 28672, groups of 128: 33.4 -> 30.7 us),
    // and elsewhere it costs nothing (T = 1, K = 11008, N = 57344: 69.7 -> 68.0).  The order of a channel's additions goes
    // with it.
    const int turn = (int)blockIdx.x % rounds;

    // what is requested next; behind the run's end its last round again, dropped
    auto channel = [&](int block) { return (int64_t)min(16 * ((int)blockIdx.x + block * (int)gridDim.x) + l16, N - 1); };
    int ask = min(begin, (int)all - 1), ask_block = ask / rounds, ask_round;
    const uint8_t *w_row;
    const __half *s_row;
    auto aim = [&]() {
        const int r = ask - ask_block * rounds + turn;
        ask_round = r >= rounds ? r - rounds : r;
    };
    auto aim_block = [&]() {
        w_row = Qw + channel(ask_block) * (K / 2) + 16 * q;
        s_row = steps + channel(ask_block) * groups;
    };
    aim();
    aim_block();
    auto advance = [&]() {
        if (ask + 1 >= end) return;
        ++ask;
        if (ask == (ask_block + 1) * rounds) {
            ++ask_block;
            aim_block();
        }
        aim();
    };
    uint4 w[NR];
    Piece s;                                           // of the round that is requested
    auto ask_codes = [&](int k) { w[k] = *reinterpret_cast<const uint4 *>(w_row + min(NR * ask_round + k, slices - 1) * 64); };
    auto ask_steps = [&]() {
        const int at = ask_round * SPR + q * PIECE;
        if (ask_round * SPR + 4 * PIECE <= groups) {
            s = *reinterpret_cast<const Piece *>(s_row + at);
        } else {
#pragma unroll
            for (int g = 0; g < PIECE; ++g) {
                const unsigned short v = __half_as_ushort(s_row[min(at + g, groups - 1)]);
                s.s[g] = at + g < groups ? v : 0;
            }
        }
    };

    // the token rows are requested first, then the first round; loads complete in order, so the rows go to LDS while the
    // codes are on their way
    const int chunks_per_row = K / 8, chunks = T * chunks_per_row;
    {
        uint4 xv[CHUNKS];
#pragma unroll
        for (int u = 0; u < CHUNKS; ++u) {
            const int j = min(tid + NT * u, chunks - 1);
            xv[u] = *reinterpret_cast<const uint4 *>(X + (int64_t)(j / chunks_per_row) * ldx + 8 * (j % chunks_per_row));
        }
        ask_steps();
#pragma unroll
        for (int k = 0; k < NR; ++k) ask_codes(k);
#pragma unroll
        for (int u = 0; u < CHUNKS; ++u) {
            const int j = tid + NT * u;
            if (j < chunks)
                *reinterpret_cast<uint4 *>(xs + (j / chunks_per_row) * stride + 16 * (j % chunks_per_row)) = interleave_halves(xv[u]);
        }
    }
    const int tail = rounds * NR * 16 - chunks_per_row;                        // chunks of zeros behind a row
    for (int j = tid; j < T * tail; j += NT)
        *reinterpret_cast<uint4 *>(xs + (j / tail) * stride + 16 * (chunks_per_row + j % tail)) = uint4{0u, 0u, 0u, 0u};
    __syncthreads();

    uint32_t magic;                                    // 1024.0 in both halves, held in a vector register
    asm volatile("v_mov_b32 %0, 0x64006400" : "=v"(magic));
    const char *xa = xs + min(l16, T - 1) * stride;    // rows past T repeat the last one: their products are never stored
    v8h x[2][4];
    auto read_tokens = [&](int set, int slice) {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[set][j] = *reinterpret_cast<const v8h *>(xa + 256 * slice + 2 * slice_place<GROUP>(j, q));
    };
    // 16 x 16 accumulator layout: lane holds channel l16, register e holds token 4 q + e
    auto store = [&](int block, const v4f &sum) {
        const int n = 16 * ((int)blockIdx.x + block * (int)gridDim.x) + l16;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int t = 4 * q + e;
            if (t < T && n < N) Y[(int64_t)t * ldy + n] = __float2half_rn(sum[e]);
        }
    };
    v4f total = {0.f, 0.f, 0.f, 0.f}, head = total;
    int block = ask_block, round = ask_round, first_of_block = block * rounds;
    read_tokens(0, round * NR);
    advance();
    for (int at = begin; at < end; ++at) {
        const int next = round + 1 < rounds ? round + 1 : 0;          // behind a block's last round its first one, `turn`, again
        uint32_t now[(PIECE + 1) / 2][4];                             // the steps of this round, two to a dword
#pragma unroll
        for (int g = 0; g < PIECE; g += 2) all_quarters(s.s[g] | (g + 1 < PIECE ? (uint32_t)s.s[g + 1 < PIECE ? g + 1 : g] << 16 : 0u), now[g / 2]);
        ask_steps();
#pragma unroll
        for (int k = 0; k < NR; ++k) {
            read_tokens((k + 1) & 1, k + 1 == NR ? next * NR : round * NR + k + 1);
            uint32_t d[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
            sort_steps<GROUP>(d);
#pragma unroll
            for (int g = 0; g < SUB; ++g) {
                v4f part = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = g * CHAIN; j < (g + 1) * CHAIN; ++j)
                    part = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[k & 1][j], widen_codes_f16(d[j], magic), part, 0, 0, 0);
                const int step = k * SPR / NR + g, in = step % PIECE;          // of the round, of the quarter
                const uint32_t pair = now[in / 2][step / PIECE];
                const float f = __half2float(__ushort_as_half((unsigned short)(in % 2 ? pair >> 16 : pair)));
#pragma unroll
                for (int e = 0; e < 4; ++e) total[e] = __builtin_fmaf(f, part[e], total[e]);
            }
            ask_codes(k);
            // keep the requests here, one slice behind another: collected at the end of the round they would be waited for at once
            __builtin_amdgcn_sched_barrier(0);
        }
        advance();
        round = next;
        if (at + 1 == first_of_block + rounds) {
            if (first_of_block >= begin)
                store(block, total);
            else
                head = total;
            total = v4f{0.f, 0.f, 0.f, 0.f};
            ++block;
            first_of_block += rounds;
        }
    }
    // A run's last block, if it goes on in the next waves' runs: the rest of it is their `head`, or all of their sum where
    // it does not end there either.
    const bool begun = first_of_block >= begin && first_of_block < end;
    if (first_of_block < begin && begin < end) head = total;
    v4f *heads = reinterpret_cast<v4f *>(rows_u4);
    __syncthreads();                                   // all are done with the rows
    heads[wave * kWave + lane] = head;
    __syncthreads();
    if (!begun) return;
    for (int v = wave + 1; v < NW && (int)(all * v / NW) < first_of_block + rounds; ++v) {
        const v4f more = heads[v * kWave + lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) total[e] += more[e];
    }
    store(block, total);
}

// ---- at most 32 tokens whose rows do not fit in LDS -----------------------------------------------
// The rows pass through LDS in parts of 1024 channels, two of them there at a time: the next one goes to registers at a
// part's start and from there to LDS at its end.  A workgroup owns up to NW blocks of 16 channels over all of K, as many as
// make whole rounds of workgroups (T = 32, K = 8192, N = 18000: 35.4 us with all eight in each, 29.2 so); KG waves share a block,
// each with its slices of every part, and add up at the end.  A wave requests a slice of the next part when it is done with
// the same slice of this one.  Steps, and the turn by which workgroups begin with another part, as above.
// What a wave does for a slice is a chain (LDS, matrix instructions, scaling), so four waves per SIMD are better than two (us,
// T = 32, K = 8192, N = 28672, groups of 128 / 64 / 32: KG = 1 37.2 / 41.0 / 45.7, KG = 2 35.5 / 38.6 / 42.4; the kernel for few tokens
// 66 / 74 / 73).
constexpr int kPart = 1024, kPartRow = 2 * kPart + kRowPad;

template <int GROUP, int TT, int NW, int KG>
__global__ __launch_bounds__(NW *KG *kWave) void w4a16_grouped_parts_kernel(const __half *__restrict__ X, int64_t ldx, int T, int K,
                                                                        const uint8_t *__restrict__ Qw, const __half *__restrict__ steps,
                                                                        int N, __half *__restrict__ Y, int64_t ldy, int own)
{
    constexpr int NT = NW * KG * kWave, NR = kPart / 128 / KG, SUB = GROUP >= 128 ? 1 : 128 / GROUP, CHAIN = 4 / SUB;
    // codes and steps of a wave's share of a part (which may be half a group), steps of a quarter of the wave
    constexpr int SPAN = NR * 128, SPR = SPAN < GROUP ? 1 : SPAN / GROUP, PIECE = SPR < 4 ? 1 : SPR / 4;
    constexpr int SETS = TT * KG > 2 ? 1 : 2;                                  // of token chunks: what the registers hold
    constexpr int CHUNKS = 16 * TT * (kPart / 8) / NT;                         // 16-byte chunks of a part of the rows per thread
    struct __attribute__((packed, aligned(2))) Piece {
        unsigned short s[PIECE];
    };
    extern __shared__ uint4 rows_u4[];
    char *xs = reinterpret_cast<char *>(rows_u4);
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int l16 = lane & 15, q = lane >> 4;
    const int slices = K / 128, groups = K / GROUP, parts = (K + kPart - 1) / kPart;
    const int kg = wave / NW, n0 = 16 * ((int)blockIdx.x * own + wave % NW);
    const bool works = wave % NW < own;                // the others carry tokens only
    const int64_t channel = min(n0 + l16, N - 1);
    const uint8_t *w_row = Qw + channel * (K / 2) + 16 * q;
    const __half *s_row = steps + channel * groups;
    const int turn = (int)blockIdx.x % parts;
    auto part_at = [&](int p) {                        // the p-th part in this workgroup's order; behind the last its first again
        const int at = p + turn;
        return at >= parts ? at - parts : at;
    };

    uint4 xv[CHUNKS], w[NR];
    Piece s;
    auto ask_tokens = [&](int part) {
#pragma unroll
        for (int u = 0; u < CHUNKS; ++u) {
            const int j = tid + NT * u, row = j / (kPart / 8), k = part * kPart + 8 * (j % (kPart / 8));
            xv[u] = *reinterpret_cast<const uint4 *>(X + (int64_t)min(row, T - 1) * ldx + min(k, K - 8));
        }
    };
    auto put_tokens = [&](int part, int buffer) {      // zeros behind the row's end
#pragma unroll
        for (int u = 0; u < CHUNKS; ++u) {
            const int j = tid + NT * u, row = j / (kPart / 8), c = j % (kPart / 8);
            const uint4 v = interleave_halves(xv[u]);
            const bool in = part * kPart + 8 * c < K;
            *reinterpret_cast<uint4 *>(xs + (buffer * 16 * TT + row) * kPartRow + 16 * c) = uint4{in ? v.x : 0u, in ? v.y : 0u, in ? v.z : 0u, in ? v.w : 0u};
        }
    };
    auto ask_codes = [&](int part, int k) { w[k] = *reinterpret_cast<const uint4 *>(w_row + min(NR * (part * KG + kg) + k, slices - 1) * 64); };
    auto ask_steps = [&](int part) {
        const int from = (part * KG + kg) * SPAN / GROUP, at = from + q * PIECE;
        if (from + 4 * PIECE <= groups) {
            s = *reinterpret_cast<const Piece *>(s_row + at);
        } else {
#pragma unroll
            for (int g = 0; g < PIECE; ++g) {
                const unsigned short v = __half_as_ushort(s_row[min(at + g, groups - 1)]);
                s.s[g] = at + g < groups ? v : 0;
            }
        }
    };
    ask_tokens(part_at(0));
    if (works) {
        ask_steps(part_at(0));
#pragma unroll
        for (int k = 0; k < NR; ++k) ask_codes(part_at(0), k);
    }
    put_tokens(part_at(0), 0);
    __syncthreads();

    uint32_t magic;                                    // 1024.0 in both halves, held in a vector register
    asm volatile("v_mov_b32 %0, 0x64006400" : "=v"(magic));
    v4f total[TT];
#pragma unroll
    for (int i = 0; i < TT; ++i) total[i] = v4f{0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < parts; ++p) {
        const int next = part_at(p + 1 < parts ? p + 1 : p);
        ask_tokens(next);
        if (works) {
            uint32_t now[(PIECE + 1) / 2][4];                             // the steps of this part, two to a dword
#pragma unroll
            for (int g = 0; g < PIECE; g += 2) all_quarters(s.s[g] | (g + 1 < PIECE ? (uint32_t)s.s[g + 1 < PIECE ? g + 1 : g] << 16 : 0u), now[g / 2]);
            ask_steps(next);
            const char *xa = xs + ((p & 1) * 16 * TT + l16) * kPartRow;
            v8h x[SETS][TT][4];
            auto read_tokens = [&](int set, int k) {
#pragma unroll
                for (int i = 0; i < TT; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[set][i][j] = *reinterpret_cast<const v8h *>(xa + i * (16 * kPartRow) + 256 * (kg * NR + k) + 2 * slice_place<GROUP>(j, q));
            };
            if constexpr (SETS == 2) read_tokens(0, 0);
#pragma unroll
            for (int k = 0; k < NR; ++k) {
                if constexpr (SETS == 1)
                    read_tokens(0, k);
                else if (k + 1 < NR)
                    read_tokens((k + 1) & 1, k + 1);
                uint32_t d[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
                sort_steps<GROUP>(d);
#pragma unroll
                for (int g = 0; g < SUB; ++g) {
                    v4f part[TT];
#pragma unroll
                    for (int j = g * CHAIN; j < (g + 1) * CHAIN; ++j) {
                        const v8h b = widen_codes_f16(d[j], magic);
#pragma unroll
                        for (int i = 0; i < TT; ++i)
                            part[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[k % SETS][i][j], b, j == g * CHAIN ? v4f{0.f, 0.f, 0.f, 0.f} : part[i], 0, 0, 0);
                    }
                    const int step = k * SPR / NR + g, in = step % PIECE;          // of the part, of the quarter
                    const uint32_t pair = now[in / 2][step / PIECE];
                    const float f = __half2float(__ushort_as_half((unsigned short)(in % 2 ? pair >> 16 : pair)));
#pragma unroll
                    for (int i = 0; i < TT; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) total[i][e] = __builtin_fmaf(f, part[i][e], total[i][e]);
                }
                ask_codes(next, k);
                // as above: the requests stay here, one slice behind another
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        put_tokens(next, (p + 1) & 1);
        __syncthreads();
    }
    if constexpr (KG > 1) {
        v4f *sums = reinterpret_cast<v4f *>(rows_u4);
        if (kg > 0)
#pragma unroll
            for (int i = 0; i < TT; ++i) sums[((wave - NW) * TT + i) * kWave + lane] = total[i];
        __syncthreads();
        if (kg > 0) return;
#pragma unroll
        for (int v = 1; v < KG; ++v)
#pragma unroll
            for (int i = 0; i < TT; ++i) {
                const v4f more = sums[((wave + (v - 1) * NW) * TT + i) * kWave + lane];
#pragma unroll
                for (int e = 0; e < 4; ++e) total[i][e] += more[e];
            }
    }
    // 16 x 16 accumulator layout: lane holds channel l16, register e holds token 4 q + e
    const int n = n0 + l16;
#pragma unroll
    for (int i = 0; i < TT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int t = 16 * i + 4 * q + e;
            if (works && t < T && n < N) Y[(int64_t)t * ldy + n] = __float2half_rn(total[i][e]);
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

template <int GROUP, int NS, int NW, int TT, int H>
sq_status launch_grouped_skinny(const GroupedArgs &a)
{
    hipLaunchKernelGGL((w4a16_grouped_skinny_kernel<GROUP, NS, NW, TT, H>),
                       dim3((unsigned)((a.N + 16 * NS - 1) / (16 * NS)), (unsigned)((a.T + 16 * TT - 1) / (16 * TT))), dim3(NW * kWave), 0, a.st,
                       a.X, a.ldx, a.T, a.K, a.Qw, a.steps, a.N, a.Y, a.ldy);
    return hipGetLastError() == hipSuccess ? SQ_OK : SQ_ERR_LAUNCH;
}

template <int GROUP, int NW, int NR>
sq_status launch_grouped_rows(const GroupedArgs &a)
{
    const int blocks = (a.N + 15) / 16, grid = blocks < 256 ? blocks : 256;
    auto kernel = w4a16_grouped_rows_kernel<GROUP, NW, NR>;
    if (!allow_large_lds(reinterpret_cast<const void *>(kernel))) return SQ_ERR_LAUNCH;
    const size_t rows = (size_t)a.T * row_bytes(a.K, NR * 128), heads = (size_t)NW * kWave * 16;
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(NW * kWave), rows > heads ? rows : heads, a.st, a.X, a.ldx, a.T, a.K, a.Qw, a.steps, a.N,
                       a.Y, a.ldy);
    return hipGetLastError() == hipSuccess ? SQ_OK : SQ_ERR_LAUNCH;
}

template <int GROUP, int TT, int NW, int KG>
sq_status launch_grouped_parts(const GroupedArgs &a)
{
    auto kernel = w4a16_grouped_parts_kernel<GROUP, TT, NW, KG>;
    if (!allow_large_lds(reinterpret_cast<const void *>(kernel))) return SQ_ERR_LAUNCH;
    const int64_t blocks = ((int64_t)a.N + 15) / 16;
    const int64_t rounds = (blocks + 256 * NW - 1) / (256 * NW), own = (blocks + 256 * rounds - 1) / (256 * rounds);       // of workgroups; blocks of one
    hipLaunchKernelGGL(kernel, dim3((unsigned)((blocks + own - 1) / own)), dim3(NW * KG * kWave), 2 * 16 * TT * kPartRow, a.st, a.X, a.ldx, a.T, a.K,
                       a.Qw, a.steps, a.N, a.Y, a.ldy, (int)own);
    return hipGetLastError() == hipSuccess ? SQ_OK : SQ_ERR_LAUNCH;
}

// The kernels and their shapes, numbered as sq_debug_grouped_plan has them.
enum GroupedKernel {
    kChannels16 = 1, kChannels32, kChannels64, kChannels64Tokens32,        // per workgroup of the kernel for few tokens
    kRowsInLds,
    kParts8, kParts2,                                                      // blocks of channels side by side
    kTiles64x128, kTiles128x128, kTiles128x256, kTiles256x256
};

GroupedKernel choose_grouped_few(int64_t T, int K, int64_t N)
{
    const int64_t tiles = (T + 15) / 16, blocks = (N + 15) / 16;
    const bool slices = K % 128 == 0, large = K * N > ((int64_t)32 << 20) && blocks > 256;
    // Token rows in LDS where they fit and there is enough to share out evenly (us, that / the kernel for few tokens at its best,
    // T = 1, groups of 128: K = 4096, N = 8192 9.0 / 7.7, N = 9216 10.3 / 12.0; K = 8192, N = 8192 12.7 / 13.7, N = 28672 28.9 / 38.0),
    // at more than one block of channels per workgroup (K = 11008, N = 4096 10.9 / 10.1).
    if (tiles == 1 && slices && large && T * row_bytes(K, 512) <= kMaxDynamicLds) return kRowsInLds;
    // In parts where they do not fit, or are more than 16 over a K worth the two barriers of a part (us, parts / the kernel for few
    // tokens, groups of 128: T = 16, K = 8192, N = 28672 30.7 / 47.8, K = 5120, N = 13824 15.0 / 17.5, K = 8192, N = 8192 16.2 / 18.2, but
    // T = 8, K = 28672, N = 8192 42.1 / 39.3; T = 32, K = 1024, N = 28672 9.1 / 12.4, N = 16384 7.4 / 7.2; K = 2048, N = 16384 9.9 / 11.6;
    // K = 4096, N = 8192 11.9 / 13.9).
    if (slices && blocks > 256 && (tiles == 2 ? K >= (blocks > 1024 ? 1024 : 2048) : tiles == 1 && large && (T > 8 || blocks > 512)))
        return blocks > 512 ? kParts8 : kParts2;
    // The fewest channels per workgroup that need one round of workgroups on the 256 CUs (us with 16 / 32 / 64 channels, T = 1,
    // K = 4096, groups of 128: N = 4096 5.8 / 7.4 / 11.8, N = 6144 9.0 / 7.5 / 12.0, N = 9216 12.2 / 12.7 / 12.0), and both blocks of
    // 16 tokens in a workgroup before there are two rounds (T = 32, N = 11008 26.0 / 19.8).
    if (blocks * tiles <= 256) return kChannels16;
    if (blocks * tiles <= 512) return kChannels32;
    return tiles == 1 || blocks * tiles <= 1024 ? kChannels64 : kChannels64Tokens32;
}

// Many tokens: the tile kernel of sq_w4a16_gemm with the steps on the widened codes.  Us of one build with each shape, groups of 128, the
// shape taken marked:
//                            64 x 128   128 x 128   128 x 256   256 x 256
//                               two K groups
//   T = 333, K = N = 4096      28.7 *     35.4        47.6        88.8
//   T = 333, N = 9000          48.7       40.0 *      51.7        90.8
//   T = 1000, N = 4096         53.3       43.7 *      51.4        92.3
//   T = 600, N = 9000          74.9       75.5        57.1 *      92.1
//   T = 1500, N = 14336       248        228         184 *       213
//   T = 4096, K = 11008       554        418         355         332 *
//   T = 64, K = 8192, 57344   118 *      153         131         208          (64 tokens in any case)
// 256 x 256 takes 1.85 times as long per round of 256 workgroups as 128 x 256 over such shapes, and is taken where that is less.
// T = 2048, K = N = 4096 takes 72 to 76 us with groups of 32 to 128 (sq_w4a16_gemm with its step per channel 64 to 66), T = 333, K = 5120,
// N = 13824 70 to 74 (63): what the steps cost is the packed multiplication per two codes and power.
GroupedKernel choose_grouped_many(int64_t T, int K, int64_t N)
{
    auto tiles = [&](int bm, int bn) { return (T + bm - 1) / bm * ((N + bn - 1) / bn); };
    auto rounds = [&](int bm, int bn) { return (tiles(bm, bn) + 255) / 256; };
    const bool two_k_groups = K % 128 == 0;
    if (two_k_groups && (T <= 64 || tiles(64, 128) <= 256)) return kTiles64x128;
    if (two_k_groups && tiles(128, 128) <= 256) return kTiles128x128;
    return 37 * rounds(256, 256) < 20 * rounds(128, 256) ? kTiles256x256 : kTiles128x256;
}

GroupedKernel choose_grouped(int64_t T, int K, int64_t N)
{
    // Tiles of many tokens, but where the kernel for few needs one round of workgroups for them all: a workgroup there shares K
    // among eight waves, a tile is one walk over it (us, few / tiles, groups of 128: T = 64, K = 4096, N = 1024 7.8 / 23.8, T = 128,
    // N = 4096 19.4 / 24.4, K = 11008 38.8 / 62.9; two rounds: T = 48, N = 11008 33.3 / 26.1, T = 128, N = 8192 35.7 / 25.4).
    if (T > 32 && (T + 31) / 32 * ((N + 63) / 64) > 256) return choose_grouped_many(T, K, N);
    return choose_grouped_few(T, K, N);
}

template <int GROUP>
sq_status launch_grouped_few(const GroupedArgs &a, GroupedKernel kernel)
{
    const bool two = a.T > 16;
    switch (kernel) {
        case kRowsInLds: return launch_grouped_rows<GROUP, 8, 4>(a);
        case kParts8: return two ? launch_grouped_parts<GROUP, 2, 8, 2>(a) : launch_grouped_parts<GROUP, 1, 8, 2>(a);
        case kParts2: return two ? launch_grouped_parts<GROUP, 2, 2, 8>(a) : launch_grouped_parts<GROUP, 1, 2, 8>(a);
        case kChannels16: return launch_grouped_skinny<GROUP, 1, 8, 1, 2>(a);
        case kChannels32: return launch_grouped_skinny<GROUP, 2, 8, 1, 2>(a);
        // groups of 32 and 64 have more registers of steps: a slice at a time then fits
        case kChannels64: return launch_grouped_skinny<GROUP, 4, 8, 1, GROUP <= 64 ? 1 : 2>(a);
        default: return launch_grouped_skinny<GROUP, 4, 8, 2, 1>(a);
    }
}

template <int WM, int FM, int FN, int LW, int KG>
sq_status launch_grouped_tiles(const GroupedArgs &a)
{
    return launch_w4a16_ring<WM, 4, FM, FN, 1, 64, LW, KG, true>(a.X, a.ldx, a.T, a.K, a.Qw, a.steps, a.N, a.Y, a.ldy, a.st, __builtin_ctz((unsigned)a.group));
}

sq_status check_grouped(int64_t T, int32_t K, int32_t group, int32_t N)
{
    if (group != 32 && group != 64 && group != 128 && group != 256) return SQ_ERR_SHAPE;
    if (T < 0 || N < 0 || K <= 0 || (K % 64) != 0 || (K % group) != 0 || K > 131072) return SQ_ERR_SHAPE;
    if (T > (1 << 24) || N > (1 << 28)) return SQ_ERR_SHAPE;         // 2^28 channels: their numbers, padded, and the grids stay in 32 bits
    return SQ_OK;
}

}  // namespace

}  // namespace sq

extern "C" sq_status sq_w4a16_gemm_grouped(const void *X, int64_t T, int32_t K, int64_t ldx, const uint8_t *Qw,
                                           const void *steps, int32_t group, int32_t N, void *Y, int64_t ldy, void *stream)
{
    const sq_status shape = sq::check_grouped(T, K, group, N);
    if (shape != SQ_OK) return shape;
    if (ldx < K || ldy < N) return SQ_ERR_SHAPE;
    if (T == 0 || N == 0) return SQ_OK;
    if (!X || !Qw || !steps || !Y) return SQ_ERR_NULL;
    if (((uintptr_t)X & 15) || (ldx % 8) != 0 || ((uintptr_t)Qw & 15) || ((uintptr_t)Y & 1) || ((uintptr_t)steps & (group == 32 ? 3 : 1)))
        return SQ_ERR_ALIGN;
    const sq::GroupedArgs a = {static_cast<const __half *>(X), ldx, (int)T, K, Qw, static_cast<const __half *>(steps), group, N,
                               static_cast<__half *>(Y), ldy, static_cast<hipStream_t>(stream)};
    const sq::GroupedKernel kernel = sq::choose_grouped(T, K, N);
    if (kernel == sq::kTiles64x128) return sq::launch_grouped_tiles<1, 2, 1, 0, 2>(a);
    if (kernel == sq::kTiles128x128) return sq::launch_grouped_tiles<1, 4, 1, 0, 2>(a);
    if (kernel == sq::kTiles128x256) return sq::launch_grouped_tiles<1, 4, 2, 4, 1>(a);
    if (kernel == sq::kTiles256x256) return sq::launch_grouped_tiles<2, 4, 2, 0, 1>(a);
    if (group == 32) return sq::launch_grouped_few<32>(a, kernel);
    if (group == 64) return sq::launch_grouped_few<64>(a, kernel);
    if (group == 128) return sq::launch_grouped_few<128>(a, kernel);
    return sq::launch_grouped_few<256>(a, kernel);
}

extern "C" int32_t sq_debug_grouped_plan(int64_t T, int32_t K, int32_t group, int32_t N)
{
    if (T == 0 || N == 0 || sq::check_grouped(T, K, group, N) != SQ_OK) return 0;
    return (int32_t)sq::choose_grouped(T, K, N);
}

// What the 16-bit x 4-bit products share: codes widened to fp16 in registers, and the tile kernel for many tokens.
#pragma once

#include "sq_gemm_tile.h"

#include <type_traits>

namespace sq {

namespace {

// halves 0..7 of a chunk -> order 0 4 1 5 2 6 3 7 (dword d holds halves 2d, 2d+1)
__device__ __forceinline__ uint4 interleave_halves(const uint4 v)
{
    uint4 r;
    r.x = __builtin_amdgcn_perm(v.z, v.x, 0x05040100u);      // (x0, x4)
    r.y = __builtin_amdgcn_perm(v.z, v.x, 0x07060302u);      // (x1, x5)
    r.z = __builtin_amdgcn_perm(v.w, v.y, 0x05040100u);      // (x2, x6)
    r.w = __builtin_amdgcn_perm(v.w, v.y, 0x07060302u);      // (x3, x7)
    return r;
}

// eight codes of a dword as fp16, in the order 0 4 1 5 2 6 3 7.  With x = dword ^ 0x88888888 every
// nibble holds u = code + 8.  "x & 0x000F000F | 0x64006400" is the pair of halves (1024 + u_0,
// 1024 + u_4), and one packed subtraction of 1032 leaves the codes; "x & 0x00F000F0 | 0x64006400"
// is (1024 + 16 u_1, 1024 + 16 u_5), and one packed multiply-add with 1/16 and -72 leaves those
// codes, exactly (every intermediate is a small multiple of 1/16).  The upper two nibble pairs
// take the same two forms on x >> 8.  Ten instructions per dword; the and-or is written as the
// one three-operand instruction it is (its constants must come from registers in that form, which
// the compiler avoids by emitting two instructions).
// The other operand's 16-byte chunks are put into the same order (interleave_halves), which a dot
// product does not see.
// PLUS4: the nibbles already hold code + 4 (the 3-bit storage expanded by w3_nibbles below), so
// there is nothing to flip and the offsets are 1028 and 68.
template <bool PLUS4 = false>
__device__ __forceinline__ v8h widen_codes_f16(uint32_t w, uint32_t magic_vgpr)
{
    const uint32_t x = PLUS4 ? w : (w ^ 0x88888888u);
    const _Float16 off = PLUS4 ? (_Float16)-1028.f : (_Float16)-1032.f;
    const _Float16 off16 = PLUS4 ? (_Float16)-68.f : (_Float16)-72.f;
    const v2h sixteenth = {(_Float16)0.0625f, (_Float16)0.0625f};
    const v2h bias = {off, off}, bias16 = {off16, off16};
    const uint32_t x8 = x >> 8;
    uint32_t h0, h1, h2, h3;
    asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(h0) : "v"(x), "s"(0x000F000Fu), "v"(magic_vgpr));
    asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(h1) : "v"(x), "s"(0x00F000F0u), "v"(magic_vgpr));
    asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(h2) : "v"(x8), "s"(0x000F000Fu), "v"(magic_vgpr));
    asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(h3) : "v"(x8), "s"(0x00F000F0u), "v"(magic_vgpr));
    const v2h p0 = __builtin_bit_cast(v2h, h0) + bias;
    const v2h p1 = __builtin_bit_cast(v2h, h1) * sixteenth + bias16;
    const v2h p2 = __builtin_bit_cast(v2h, h2) + bias;
    const v2h p3 = __builtin_bit_cast(v2h, h3) * sixteenth + bias16;
    return v8h{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
}

// Two of the eight codes of a dword (byte M, every nibble holding code + 8) as a pair of fp16, in their own order.
// The byte is copied into both halves of a dword; "& 0x00F0000F | 0x64006400" leaves
// 1024 + (code_2M + 8) in the low half and 1024 + 16 (code_2M+1 + 8) in the high half, and one
// packed multiply-add with (1, 1/16) and (-1032, -72) the two codes, exactly.  Three
// instructions: the and-or is written as the one three-operand instruction it is (its
// constants must come from registers in that form, which the compiler avoids by emitting two).
template <int M>
__device__ __forceinline__ uint32_t widen_byte_f16(uint32_t x, uint32_t magic_vgpr, v2h scale = {(_Float16)1.f, (_Float16)0.0625f},
                                                   v2h bias = {(_Float16)-1032.f, (_Float16)-72.f})
{
    const uint32_t sel = 0x0C000C00u | (uint32_t)M | ((uint32_t)M << 16);
    uint32_t h;
    asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(h) : "v"(__builtin_amdgcn_perm(0u, x, sel)), "s"(0x00F0000Fu), "v"(magic_vgpr));
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(v2h, h) * scale + bias);
}

__device__ __forceinline__ void dma_16_if(const void *gptr, uint32_t lds_addr, int a, int b)
{
    // 16 bytes per lane, global memory -> LDS at lds_addr + 16 lane, issued only if a < b (both
    // wave-uniform); the branch lives inside the assembly so that the loop body stays one block
    asm volatile("s_cmp_lt_i32 %2, %3\n\t"
                 "s_cbranch_scc0 .Lsq16_skip_%=\n\t"
                 "s_mov_b32 m0, %1\n\t"
                 "s_nop 0\n\t"
                 "global_load_lds_dwordx4 %0, off\n"
                 ".Lsq16_skip_%=:"
                 :
                 : "v"(gptr), "s"(lds_addr), "s"(a), "s"(b)
                 : "memory", "m0", "scc");
}

// Two bytes, or four with groups of 32, of each of the first LANES lanes, global memory -> the dword at lds_addr + 4 lane
// (two are zero-extended); else as dma_16_if
template <int LANES>
__device__ __forceinline__ void dma_step_if(const void *gptr, uint32_t lds_addr, int a, int b, int group_shift)
{
    static_assert(LANES == 32 || LANES == 64, "a wave or half of it");
    if constexpr (LANES == 64)
        asm volatile("s_cmp_lt_i32 %2, %3\n\t"
                     "s_cbranch_scc0 .Lsqs_skip_%=\n\t"
                     "s_mov_b32 m0, %1\n\t"
                     "s_cmp_eq_u32 %4, 5\n\t"
                     "s_cbranch_scc1 .Lsqs_four_%=\n\t"
                     "global_load_lds_ushort %0, off\n\t"
                     "s_branch .Lsqs_skip_%=\n"
                     ".Lsqs_four_%=:\n\t"
                     "global_load_lds_dword %0, off\n"
                     ".Lsqs_skip_%=:"
                     :
                     : "v"(gptr), "s"(lds_addr), "s"(a), "s"(b), "s"(group_shift)
                     : "memory", "m0", "scc");
    else {
        uint32_t upper;
        asm volatile("s_cmp_lt_i32 %3, %4\n\t"
                     "s_cbranch_scc0 .Lsqs_skip_%=\n\t"
                     "s_mov_b32 m0, %2\n\t"
                     "s_mov_b32 %0, exec_hi\n\t"
                     "s_mov_b32 exec_hi, 0\n\t"
                     "s_cmp_eq_u32 %5, 5\n\t"
                     "s_cbranch_scc1 .Lsqs_four_%=\n\t"
                     "global_load_lds_ushort %1, off\n\t"
                     "s_branch .Lsqs_done_%=\n"
                     ".Lsqs_four_%=:\n\t"
                     "global_load_lds_dword %1, off\n"
                     ".Lsqs_done_%=:\n\t"
                     "s_mov_b32 exec_hi, %0\n"
                     ".Lsqs_skip_%=:"
                     : "=&s"(upper)
                     : "v"(gptr), "s"(lds_addr), "s"(a), "s"(b), "s"(group_shift)
                     : "memory", "m0", "scc");
    }
}

// Tile kernel for many tokens.  Block tile (WM FM 32) tokens x (WN FN 32) channels, WM x WN waves
// of FM x FN fragments of 32 x 32; K walked in tiles of 64.  Both operands travel global -> LDS
// without passing registers (16 bytes per lane), through a ring of three stages, two tiles ahead,
// completion tracked by hand: activations as they are (rows of 128 bytes, the 16-byte chunks of a
// row XOR-swizzled by (row / 2) % 8), weight codes packed (rows of 32 bytes).  A wave widens the codes
// of its own channels in registers, in order, so the activations need no reordering; one dword
// makes the operand of FM MFMAs, which is why a wave's tile is tall (FM = 4: 128 tokens x 64
// channels, 13 VALU instructions per 4 MFMAs) rather than wide.  Within a K tile lane half g takes
// elements 32g .. 32g + 31 and step s the eight elements 32g + 8s ..: chunk 4g + s of an
// activation row, dword s of chunk g of a code row.
// Operands run one step ahead of the MFMAs, also across the turn between K tiles, with the LDS reads and the widening
// written between the MFMAs: at the start of a tile nothing waits for LDS.  (All of a tile read behind its barrier, us
// before / after: T = 40, K = N = 4096 47.4 / 39.3; T = 1000, K = 3200, N = 2000 40.6 / 35.4; T = 2048, K = N = 4096 74.4 / 66.8,
// K = 11008 170 / 162; T = 2048, K = 8192, N = 14336 423 / 415.)  What bounds the large ones is power: the same products of
// zeros take 50.7 us at T = 2048, K = N = 4096 and 440 against 640 at T = 8192, N = 11008, where torch's fp16 product takes as
// long as this kernel.
// The weights are the first MFMA operand, so the 32 x 32 accumulator has the token in the lane and
// the channel in the register: register e holds channel 8 (e / 4) + 4 (lane / 32) + e % 4, four
// runs of four consecutive channels.  Two runs are traded between the half-waves (one cross-half
// swap per dword) and every lane stores 16 contiguous bytes of a row of Y.
// BK: elements of K per tile (a tile row of activations is 2 BK bytes, of codes BK / 2); 64 is what
// is built (128 was measured: 2 % faster at 2048 tokens, 10 % slower at 8192, and its 256-byte rows
// would want another swizzle).
// LW > 0: LW more waves that only request the tiles and wait for them; the multiplying waves then
// issue no memory instruction inside the loop and meet the others at the barrier of each tile.
// KG: groups of WM WN waves that walk K / KG elements each, through rings of their own, and add their sums through LDS.
// GROUPED: a step per group of 1 << group_shift >= 32 elements of K in place of one per channel.  The step of a tile, or the
// two of its halves, travel with it (a dword per channel; each is of another row, and their number is what these loads cost:
// with a load per half T = 333, K = 5120, N = 13824, groups of 32 took 73.5 us, so 69.3), and a widened code is multiplied by its step
// in fp16, rounded once: a lane's 32 elements of a tile lie in one group, so that is one packed multiplication per two codes (four
// widening instructions instead of three).  Scaling the sums instead would keep them exact, but wants as many registers again as
// the sums have.
// Eight times a step from 8192 on is no fp16.  A wave notes the channels that have such steps on its way; where a workgroup has any it
// walks over K once more (T = 2048, K = N = 4096: 75.7 us, 137 with such steps), those channels' codes taken by 1/8 and their sums by 8.
// (Sums scaled in the middle of one walk: the branch holds them twice, 60 registers more, and the large tiles spill.)
template <int WM, int WN, int FM, int FN, int OCC, int BK, int LW, int KG, bool GROUPED>
__global__ __launch_bounds__((KG * WM * WN + LW) * kWave, OCC) void w4a16_gemm_ring_kernel(
    const __half *__restrict__ X, int64_t ldx, int T, int K, const uint8_t *__restrict__ Qw,
    const typename std::conditional<GROUPED, __half, float>::type *__restrict__ sw, int N, __half *__restrict__ Y, int64_t ldy,
    int tiles_m, int tiles_n, int vec_store, int group_shift)
{
    static_assert(BK == 64, "tiles of 64 elements of K");
    constexpr int NW = WM * WN, NS = 3, STEPS = BK / 16;     // waves of a group; ring stages; MFMA steps per K tile
    static_assert(KG == 1 || LW == 0, "loading waves: one K group");
    constexpr int BM = WM * FM * 32, BN = WN * FN * 32;
    constexpr int A_ROW = 2 * BK, B_ROW = BK / 2;            // bytes of a tile row
    constexpr int A_CPR = A_ROW / 16, B_CPR = B_ROW / 16;    // 16-byte chunks per row
    constexpr int A_RPL = 64 / A_CPR, B_RPL = 64 / B_CPR;    // rows filled by one wave-wide load
    constexpr int A_BYTES = BM * A_ROW, B_BYTES = BN * B_ROW, S_BYTES = GROUPED ? BN * 4 : 0;
    constexpr int STAGE = A_BYTES + B_BYTES + S_BYTES;
    constexpr int NL = LW > 0 ? LW : NW;                     // waves that share the loads of a tile
    constexpr int A_LOADS = BM / A_RPL / NL, B_LOADS = BN / B_RPL / NL;       // wave-wide loads per loading wave and tile
    constexpr int S_LOADS = GROUPED ? 1 : 0, S_LANES = BN / NL;
    constexpr int LOADS = A_LOADS + B_LOADS + S_LOADS;
    static_assert((BM / A_RPL) % NL == 0 && (BN / B_RPL) % NL == 0 && (!GROUPED || S_LANES == 32 || S_LANES == 64),
                  "loads must split evenly over the waves");
    extern __shared__ uint4 ring[];

    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const bool loader = LW > 0 && tid / kWave >= NW;
    const int wave = (tid / kWave) % NW;                         // a loading wave counts from 0 again
    const int kg = LW > 0 ? 0 : __builtin_amdgcn_readfirstlane(tid / kWave / NW);
    const int l32 = lane & 31, g = lane >> 5;
    const int wm = wave / WN, wn = wave % WN;
    int bm, bn;
    {
        const int id = xcd_contiguous_id(blockIdx.x, tiles_m * tiles_n);
        constexpr int GM = 8;
        const int group = id / (GM * tiles_n), gm = min(GM, tiles_m - group * GM);
        const int in_group = id - group * GM * tiles_n;
        bm = group * GM + in_group % gm;
        bn = in_group / gm;
    }
    const int Kb = K / 2;
    const int kg0 = kg * (K / KG);                               // this group's elements of K
    int row0 = bm * BM, col0 = bn * BN;
    v16f acc[FM][FN];
    uint32_t eighth[FN] = {};                          // channels of a fragment whose steps are taken by 1/8, a bit each
    __shared__ uint32_t large_of[GROUPED ? KG : 1][GROUPED ? NW : 1][FN];
#pragma unroll 1
    for (int walk = 0; walk < (GROUPED ? 2 : 1); ++walk) {
        if constexpr (GROUPED) asm volatile("" : "+s"(row0), "+s"(col0));      // what follows from them is found again, not kept from walk to walk

        // global -> LDS.  One wave-wide load fills 64 consecutive chunk slots: A_RPL rows of activations
        // (lane l lands in row l / A_CPR, physical chunk l % A_CPR, which holds the logical chunk
        // (l % A_CPR) ^ ((row / 2) % 8): sixteen consecutive rows, two per 256 bytes of the 64 banks, then
        // keep the same logical chunk in sixteen different bank groups) or B_RPL rows of codes.  Rows past the ends are clamped: their
        // products are never stored.
        const __half *a_src[A_LOADS];
        const uint8_t *b_src[B_LOADS];
#pragma unroll
        for (int u = 0; u < A_LOADS; ++u) {
            const int r = A_RPL * (wave + NL * u) + lane / A_CPR;
            a_src[u] = X + (int64_t)min(row0 + r, T - 1) * ldx + kg0 + (((lane % A_CPR) ^ ((r >> 1) & 7)) * 8);
        }
#pragma unroll
        for (int u = 0; u < B_LOADS; ++u) {
            const int r = B_RPL * (wave + NL * u) + lane / B_CPR;
            b_src[u] = Qw + (int64_t)min(col0 + r, N - 1) * Kb + kg0 / 2 + (lane % B_CPR) * 16;
        }
        // steps: S_LANES channels per loading wave
        const __half *s_src = nullptr;
        if constexpr (GROUPED) s_src = sw + (int64_t)min(col0 + wave * S_LANES + lane % S_LANES, N - 1) * (K >> group_shift);
        const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint4 *)ring + kg * (NS * STAGE);
        const uint32_t wave_u = __builtin_amdgcn_readfirstlane(wave);
        auto issue_tile = [&](int kt, int stage, int limit) {
            const uint32_t sa = lds_base + (uint32_t)stage * STAGE;
#pragma unroll
            for (int u = 0; u < A_LOADS; ++u) dma_16_if(a_src[u] + kt * BK, sa + (wave_u + NL * u) * 1024, kt, limit);
#pragma unroll
            for (int u = 0; u < B_LOADS; ++u)
                dma_16_if(b_src[u] + kt * (BK / 2), sa + A_BYTES + (wave_u + NL * u) * 1024, kt, limit);
            if constexpr (GROUPED)
                dma_step_if<S_LANES>(s_src + ((kg0 + min(kt, limit - 1) * BK) >> group_shift), sa + A_BYTES + B_BYTES + wave_u * (4 * S_LANES), kt, limit,
                                     group_shift);
        };

        // LDS byte offsets of this lane's fragment chunks inside a stage: lane half g takes the elements
        // [g BK / 2, (g + 1) BK / 2) of a K tile, step s the eight elements 8 s .. of those
        int a_off[STEPS];
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
            a_off[s] = (wm * FM * 32 + l32) * A_ROW + (((STEPS * g + s) ^ ((l32 >> 1) & 7)) * 16);
        const int b_off = A_BYTES + (wn * FN * 32 + l32) * B_ROW + g * (STEPS * 4);
        const int s_off = A_BYTES + B_BYTES + (wn * FN * 32 + l32) * 4;
        const uint32_t s_half = GROUPED && group_shift == 5 && g ? 0x03020302u : 0x01000100u;       // this lane's step of the dword, twice
        const char *lds = reinterpret_cast<const char *>(ring) + kg * (NS * STAGE);

        uint32_t magic;                                    // 1024.0 in both halves, held in a vector register
        asm volatile("v_mov_b32 %0, 0x64006400" : "=v"(magic));
        const int ktiles = K / (KG * BK);
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
        int stage = 0;
        if (LW == 0 || loader) {
#pragma unroll
            for (int t = 0; t < NS - 1; ++t) issue_tile(t, t, ktiles);
            wait_tile_and_barrier<LOADS, NS>(ktiles - 1);
            issue_tile(NS - 1, NS - 1, ktiles);
        } else {
            asm volatile("s_barrier" ::: "memory");
        }
        if (LW > 0 && loader) {
            // a loading wave: the waits and requests of the loop below and nothing else; it meets the
            // multiplying waves at each of the 1 + ktiles barriers of the walk
            for (int kt = 0; kt < ktiles; ++kt) {
                wait_tile_and_barrier<LOADS, NS>(ktiles - kt - 2);
                issue_tile(kt + NS, stage, ktiles);
                stage = stage == NS - 1 ? 0 : stage + 1;
            }
            if constexpr (!GROUPED) return;
        } else {

            // Operands run one step ahead of the MFMAs: while step s is multiplied, the activations of step s + 1 are read and its
            // codes widened between the MFMAs, in the order written here.  A dword of codes per step: rb holds a tile's.
            constexpr int NM = FM * FN;
            static_assert(STEPS == 4 && NM >= 2, "four steps per tile");
            typedef uint32_t v4u __attribute__((ext_vector_type(4)));
            uint4 rb[FN];
            v8h a[2][FM];
            v4u b[2][FN];
            uint32_t flipped[FN], step2[GROUPED ? FN : 1];     // step2: the step of this lane's half of the tile, twice
            v2h scale[FN], bias[FN];                           // of the widening: codes, or codes / 8
            _Float16 largest[GROUPED ? FN : 1];                // of the steps
            if constexpr (GROUPED) {
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    const _Float16 share = (eighth[j] >> l32) & 1 ? (_Float16)0.125f : (_Float16)1.f;
                    scale[j] = v2h{share, (_Float16)0.0625f * share};
                    bias[j] = v2h{(_Float16)-1032.f * share, (_Float16)-72.f * share};
                    largest[j] = 0;
                }
            }
            auto read_codes = [&](int stage_byte) {
#pragma unroll
                for (int j = 0; j < FN; ++j) rb[j] = *reinterpret_cast<const uint4 *>(lds + stage_byte + b_off + j * (32 * B_ROW));
                if constexpr (GROUPED) {
#pragma unroll
                    for (int j = 0; j < FN; ++j) step2[j] = __builtin_amdgcn_perm(0u, *reinterpret_cast<const uint32_t *>(lds + stage_byte + s_off + j * (32 * 4)), s_half);
                }
            };
            auto read_tokens = [&](int set, int stage_byte, int s, int i) {
                a[set][i] = *reinterpret_cast<const v8h *>(lds + stage_byte + a_off[s] + i * (32 * A_ROW));
            };
            // unit u of 4 FN: byte u % 4 of the dword of step s of fragment u / 4
            auto widen_unit = [&](int set, int s, int u) {
                const int j = u / 4;
                if (u % 4 == 0) flipped[j] = (s == 0 ? rb[j].x : s == 1 ? rb[j].y : s == 2 ? rb[j].z : rb[j].w) ^ 0x88888888u;
                if constexpr (!GROUPED) {
                    b[set][j][u % 4] = u % 4 == 0   ? widen_byte_f16<0>(flipped[j], magic)
                                       : u % 4 == 1 ? widen_byte_f16<1>(flipped[j], magic)
                                       : u % 4 == 2 ? widen_byte_f16<2>(flipped[j], magic)
                                                    : widen_byte_f16<3>(flipped[j], magic);
                } else {
                    const uint32_t code2 = u % 4 == 0   ? widen_byte_f16<0>(flipped[j], magic, scale[j], bias[j])
                                           : u % 4 == 1 ? widen_byte_f16<1>(flipped[j], magic, scale[j], bias[j])
                                           : u % 4 == 2 ? widen_byte_f16<2>(flipped[j], magic, scale[j], bias[j])
                                                        : widen_byte_f16<3>(flipped[j], magic, scale[j], bias[j]);
                    b[set][j][u % 4] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(v2h, code2) * __builtin_bit_cast(v2h, step2[j]));
                }
            };
            // One step on set C; the next one's operands are step S of the tile at BYTE.  TURN: the turn into that tile comes
            // first, and its codes are read; they are widened in the second half of the step.
#define SQ_W16_STEP(C, BYTE, S, TURN)                                                                               \
    do {                                                                                                            \
        _Pragma("unroll") for (int m = 0; m < NM; ++m) {                                                            \
            const int j = m / FM, i = m % FM;                                                                       \
            constexpr int from = (TURN) ? NM / 2 : 0;                                                               \
            if ((TURN) && m == 1) {                                                                                 \
                SQ_W16_TURN();                                                                                      \
                read_codes(BYTE);                                                                                   \
            }                                                                                                       \
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, b[C][j]), a[C][i], acc[i][j], 0, 0, 0); \
            _Pragma("unroll") for (int r = 0; r < FM; ++r)                                                          \
                if (m == (r + (TURN) < NM ? r + (TURN) : NM - 1)) read_tokens(1 - (C), BYTE, S, r);                 \
            _Pragma("unroll") for (int u = 0; u < 4 * FN; ++u)                                                      \
                if (m == from + u * (NM - from) / (4 * FN)) widen_unit(1 - (C), S, u);                              \
            __builtin_amdgcn_sched_barrier(0);                                                                      \
        }                                                                                                           \
    } while (0)
            // Tile kt + 1 has landed once only the loads of the NS - 2 tiles behind it (those that exist) are outstanding.  Behind
            // the barrier every wave's share of it is in LDS and all reads of tile kt are done, so its stage takes tile kt + NS.
#define SQ_W16_TURN()                                                                                               \
    do {                                                                                                            \
        if constexpr (LW == 0) {                                                                                    \
            wait_tile_and_barrier<LOADS, NS>(ktiles - kt - 2);                                                      \
            issue_tile(kt + NS, stage, ktiles);                                                                     \
        } else {                                                                                                    \
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");                                         \
        }                                                                                                           \
    } while (0)
            read_codes(0);
#pragma unroll
            for (int i = 0; i < FM; ++i) read_tokens(0, 0, 0, i);
#pragma unroll
            for (int u = 0; u < 4 * FN; ++u) widen_unit(0, 0, u);
            for (int kt = 0; kt < ktiles; ++kt) {
                const int stage_n = stage == NS - 1 ? 0 : stage + 1;
                const int cur_byte = stage * STAGE, next_byte = stage_n * STAGE;
                if constexpr (GROUPED) {
#pragma unroll
                    for (int j = 0; j < FN; ++j) largest[j] = __builtin_fmaxf16(largest[j], __builtin_fabsf16(__builtin_bit_cast(v2h, step2[j])[0]));
                }
                SQ_W16_STEP(0, cur_byte, 1, 0);
                SQ_W16_STEP(1, cur_byte, 2, 0);
                SQ_W16_STEP(0, cur_byte, 3, 0);
                SQ_W16_STEP(1, next_byte, 0, 1);          // behind the last tile: a stale stage, never used
                stage = stage_n;
            }
#undef SQ_W16_STEP
#undef SQ_W16_TURN
            if constexpr (GROUPED) {
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    const uint64_t lanes = __ballot(largest[j] >= (_Float16)8192.f);       // both halves of the wave hold steps of the channel
                    if (lane == 0) large_of[kg][wave][j] = (uint32_t)lanes | (uint32_t)(lanes >> 32);
                }
            }
        }
        if constexpr (GROUPED) {
            __syncthreads();                               // the flags are there, and all are done with the ring
            if (walk == 1) break;
            uint32_t any = 0;
#pragma unroll
            for (int k = 0; k < KG; ++k)
#pragma unroll
                for (int w = 0; w < NW; ++w)
#pragma unroll
                    for (int j = 0; j < FN; ++j) any |= large_of[k][w][j];
            if (__builtin_amdgcn_readfirstlane(any) == 0) break;
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int k = 0; k < KG; ++k) eighth[j] = __builtin_amdgcn_readfirstlane(eighth[j] | large_of[k][wave][j]);
        }
    }
    if (LW > 0 && loader) return;

    if constexpr (KG > 1) {
        constexpr int ACC = FM * FN * 16;
        static_assert((KG - 1) * NW * ACC * kWave * 4 <= KG * NS * STAGE, "the other groups' sums fit in the dead rings");
        float *sums = reinterpret_cast<float *>(ring) + wave * (ACC * kWave) + lane;
        if constexpr (!GROUPED) __syncthreads();
        if (kg > 0) {
            float *mine = sums + (kg - 1) * (NW * ACC * kWave);
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) mine[((i * FN + j) * 16 + e) * kWave] = acc[i][j][e];
        }
        __syncthreads();
        if (kg > 0) return;
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e)
#pragma unroll
                    for (int o = 0; o < KG - 1; ++o)
                        acc[i][j][e] += sums[o * (NW * ACC * kWave) + ((i * FN + j) * 16 + e) * kWave];
    }

    typedef uint32_t v2u __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        const int nf = col0 + (wn * FN + j) * 32;            // first channel of the fragment
        float swq[4][4];
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if constexpr (GROUPED)
                    swq[q][r] = 1.f;
                else
                    swq[q][r] = sw[min(nf + 8 * q + 4 * g + r, N - 1)];
            }
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const int t = row0 + (wm * FM + i) * 32 + l32;
            if (GROUPED && eighth[j]) {
                const uint32_t mine = eighth[j] >> (4 * g);  // accumulator register e: channel 8 (e / 4) + 4 g + e % 4
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = (mine >> (8 * (e / 4) + e % 4)) & 1 ? 8.f * acc[i][j][e] : acc[i][j][e];
            }
            uint32_t run[4][2];                              // run q: channels 8q + 4g .. + 3 as two dwords
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const v2h pair = {(_Float16)__float2half_rn(acc[i][j][4 * q + 2 * h] * swq[q][2 * h]),
                                      (_Float16)__float2half_rn(acc[i][j][4 * q + 2 * h + 1] * swq[q][2 * h + 1])};
                    run[q][h] = __builtin_bit_cast(uint32_t, pair);
                }
#pragma unroll
            for (int q = 0; q < 4; q += 2) {
                // swap(a, b): result 0 = (a of lanes 0..31, b of lanes 0..31), result 1 = (a of lanes
                // 32..63, b of lanes 32..63).  With a = run q, b = run q + 1: the lower half-wave gets
                // both halves of run q (channels 8q .. 8q + 7), the upper one those of run q + 1.
                const v2u s0 = __builtin_amdgcn_permlane32_swap(run[q][0], run[q + 1][0], false, false);
                const v2u s1 = __builtin_amdgcn_permlane32_swap(run[q][1], run[q + 1][1], false, false);
                const uint32_t w[4] = {s0[0], s1[0], s0[1], s1[1]};
                const int n0 = nf + 8 * (q + g);
                if (t >= T || n0 >= N) continue;
                __half *dst = Y + (int64_t)t * ldy + n0;
                if (vec_store && n0 + 8 <= N) {
                    *reinterpret_cast<uint4 *>(dst) = uint4{w[0], w[1], w[2], w[3]};
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)              // register-only: no addressable copy of the chunk
                        if (n0 + e < N) reinterpret_cast<uint16_t *>(dst)[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
                }
            }
        }
    }
}

template <int WM, int WN, int FM, int FN, int OCC, int BK, int LW = 0, int KG = 1, bool GROUPED = false>
sq_status launch_w4a16_ring(const __half *X, int64_t ldx, int T, int K, const uint8_t *Qw,
                            const typename std::conditional<GROUPED, __half, float>::type *sw, int N, __half *Y, int64_t ldy, hipStream_t st,
                            int group_shift = 0)
{
    constexpr int BM = WM * FM * 32, BN = WN * FN * 32;
    constexpr size_t lds = (size_t)3 * KG * (BM * 2 * BK + BN * BK / 2 + (GROUPED ? BN * 4 : 0));
    static_assert(lds <= (size_t)kMaxDynamicLds, "ring does not fit in LDS");
    auto kernel = w4a16_gemm_ring_kernel<WM, WN, FM, FN, OCC, BK, LW, KG, GROUPED>;
    if ((K % (KG * BK)) != 0) return SQ_ERR_SHAPE;
    const int tiles_m = (T + BM - 1) / BM, tiles_n = (int)(((int64_t)N + BN - 1) / BN);
    if ((int64_t)tiles_m * tiles_n * ((KG * WM * WN + LW) * kWave) > 0xFFFFFFFFll) return SQ_ERR_SHAPE;       // threads of a launch
    if (!allow_large_lds(reinterpret_cast<const void *>(kernel))) return SQ_ERR_LAUNCH;
    const int vec_store = (((uintptr_t)Y & 15) == 0 && (ldy % 8) == 0) ? 1 : 0;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(tiles_m * tiles_n)), dim3((KG * WM * WN + LW) * kWave), lds, st, X, ldx, T, K, Qw,
                       sw, N, Y, ldy, tiles_m, tiles_n, vec_store, group_shift);
    return hipGetLastError() == hipSuccess ? SQ_OK : SQ_ERR_LAUNCH;
}

}  // namespace

}  // namespace sq

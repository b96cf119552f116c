// sq_rotary_fp16: rotary positions, a plane rotation of every pair of channels of a head by an angle that grows with the
// token's position; sq_rotary_table: the frequencies, scaled for long contexts (host).
#include "sq_common.h"

#include <cmath>
#include <limits>

namespace sq {

namespace {

// Cosine and sine of position * frequency.  The frequency is a 64-bit fraction of a turn, so the product modulo 2^64 is
// the fraction of a turn that is left of the angle, without error for any 32-bit position; its upper half goes to fp32
// (2^-25 of a turn at most).
__device__ __forceinline__ void rotation_of(int position, uint64_t turns, float magnitude, float &c, float &s)
{
    const uint64_t angle = (uint64_t)(int64_t)position * turns;
    const float half_turns = (float)(int32_t)(angle >> 32) * 0x1p-31f;
    sincospif(half_turns, &s, &c);
    c *= magnitude;
    s *= magnitude;
}

// a c - b s with one rounding of b s and one of the sum, which is then rounded to fp16: written out, and the sum kept from
// being rounded to fp16 in the same instruction, so that every kernel here gives the same bits.
__device__ __forceinline__ float rounded(float sum)
{
    asm("" : "+v"(sum));
    return sum;
}
__device__ __forceinline__ float turned_a(float a, float b, float c, float s) { return rounded(__builtin_fmaf(a, c, -(b * s))); }
__device__ __forceinline__ float turned_b(float a, float b, float c, float s) { return rounded(__builtin_fmaf(b, c, a * s)); }

// A lane owns one unit of 2 V channels of a token's heads: V pairs, channels V u .. and rot / 2 + V u .. (HALF) or
// 2 V u ..  It takes their cosines and sines once and then walks over the heads slot, slot + slots, ...  Behind the
// rot / (2 V) units of pairs come units that are copied (none where Y is X); they go the same way as the others and keep what
// they read, so a wave does not divide (8192 tokens, 40 heads of 128 with 64 turned: 44 us with a branch of their own,
// 39.5 us so).  One read and one write of the rows: HBM-bound, 4.2 TB/s of both with V = 8.  V is the largest of 8, 4 and 2 that
// the widths and strides allow (8192 tokens, 40 heads of 80: 40 turned 26.6 us, 20 26.3; a pair per lane took 82 and 92).
template <int V, bool HALF, bool COPIES>
__global__ __launch_bounds__(256) void rotary_kernel(const __half *X, int64_t T, int H, int D, int64_t ldx, int64_t ldh,
                                                     const int32_t *__restrict__ positions, const uint64_t *__restrict__ turns,
                                                     int rot, float magnitude, __half *Y, int64_t ldy, int64_t ldyh, int units,
                                                     int slots)
{
    typedef _Float16 Halves __attribute__((ext_vector_type(V)));
    const int64_t id = block_number() * 256 + threadIdx.x;
    const int per_token = units * slots;
    const int64_t t = id / per_token;
    if (t >= T) return;
    const int rest = (int)(id - t * per_token), u = rest % units, slot = rest / units;
    const __half *x = X + t * ldx;
    __half *y = Y + t * ldy;
    const bool turned = !COPIES || u < rot / (2 * V);
    const int d0 = HALF && turned ? V * u : 2 * V * u, d1 = HALF && turned ? rot / 2 + V * u : d0 + V;
    const bool second = !COPIES || d1 < D;                 // the last copied unit may be half a unit
    const int d2 = second ? d1 : d0;
    float c[V] = {}, s[V] = {};
    if (turned) {                                          // without turned channels there is no table, and no position is read
        const int position = positions[t];
#pragma unroll
        for (int e = 0; e < V; ++e) rotation_of(position, turns[V * u + e], magnitude, c[e], s[e]);
    }
#pragma unroll 4
    for (int h = slot; h < H; h += slots) {
        const Halves a = *reinterpret_cast<const Halves *>(x + h * ldh + d0), b = *reinterpret_cast<const Halves *>(x + h * ldh + d2);
        Halves ya, yb;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if constexpr (HALF) {
                ya[j] = (_Float16)turned_a(a[j], b[j], c[j], s[j]);
                yb[j] = (_Float16)turned_b(a[j], b[j], c[j], s[j]);
            } else {                                       // pairs of the unit's first V channels, then of the others
                const int e = j & ~1, f = e + 1, at = j / 2, bt = V / 2 + at;
                ya[j] = (_Float16)(j == e ? turned_a(a[e], a[f], c[at], s[at]) : turned_b(a[e], a[f], c[at], s[at]));
                yb[j] = (_Float16)(j == e ? turned_a(b[e], b[f], c[bt], s[bt]) : turned_b(b[e], b[f], c[bt], s[bt]));
            }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
            ya[j] = turned ? ya[j] : a[j];
            yb[j] = turned ? yb[j] : b[j];
        }
        *reinterpret_cast<Halves *>(y + h * ldyh + d0) = ya;
        if (second) *reinterpret_cast<Halves *>(y + h * ldyh + d1) = yb;
    }
}

// Any width and alignment: a lane takes one pair, or one copied channel, of one head.
__global__ __launch_bounds__(256) void rotary_pair_kernel(const __half *X, int64_t T, int H, int D, int64_t ldx, int64_t ldh,
                                                          const int32_t *__restrict__ positions,
                                                          const uint64_t *__restrict__ turns, int rot, int half,
                                                          float magnitude, __half *Y, int64_t ldy, int64_t ldyh, int units)
{
    const int64_t id = block_number() * 256 + threadIdx.x;
    const int64_t row = id / units, t = row / H;
    if (t >= T) return;
    const int u = (int)(id - row * units), h = (int)(row - t * H);
    const __half *x = X + t * ldx + h * ldh;
    __half *y = Y + t * ldy + h * ldyh;
    if (u >= rot / 2) {
        y[rot / 2 + u] = x[rot / 2 + u];
        return;
    }
    float c, s;
    rotation_of(positions[t], turns[u], magnitude, c, s);
    const int p = half ? u : 2 * u, q = half ? rot / 2 + u : 2 * u + 1;
    const float a = __half2float(x[p]), b = __half2float(x[q]);
    y[p] = __float2half_rn(turned_a(a, b, c, s));
    y[q] = __float2half_rn(turned_b(a, b, c, s));
}

template <int V>
sq_status launch_rotary(const __half *x, int64_t T, int H, int D, int64_t ldx, int64_t ldh, const int32_t *positions, const uint64_t *turns,
                        int rot, bool half, float magnitude, __half *y, int64_t ldy, int64_t ldyh, int copied, hipStream_t st)
{
    const int units = rot / (2 * V) + (copied + 2 * V - 1) / (2 * V);
    // enough lanes that every SIMD of the chip holds four waves, and at least eight heads side by side in a row
    const int64_t lanes = T * (int64_t)units;
    int64_t want = (262144 + lanes - 1) / lanes;
    if (want < 8) want = 8;
    const int slots = (int)(want < H ? want : H);
    const int64_t blocks = (lanes * slots + 255) / 256;
    if (blocks > kMaxBlocks) return SQ_ERR_SHAPE;
    auto kernel = half ? (copied ? rotary_kernel<V, true, true> : rotary_kernel<V, true, false>)
                       : (copied ? rotary_kernel<V, false, true> : rotary_kernel<V, false, false>);
    hipLaunchKernelGGL(kernel, grid_of(blocks), dim3(256), 0, st, x, T, H, D, ldx, ldh, positions, turns, rot, magnitude, y, ldy, ldyh, units,
                       slots);
    return hipGetLastError() == hipSuccess ? SQ_OK : SQ_ERR_LAUNCH;
}

}  // namespace

}  // namespace sq

extern "C" sq_status sq_rotary_table(int32_t rot, double base, sq_rotary_scaling scaling, double factor, double trained,
                                     double low, double high, uint64_t *turns)
{
    if (rot <= 0 || (rot % 2) != 0 || rot > SQ_ROTARY_MAX_CHANNELS || !(base > 1.0) || !(base <= 1e18)) return SQ_ERR_SHAPE;
    const bool scaled = scaling != SQ_ROTARY_PLAIN;
    if (scaling != SQ_ROTARY_PLAIN && scaling != SQ_ROTARY_LINEAR && scaling != SQ_ROTARY_BASE && scaling != SQ_ROTARY_PARTS)
        return SQ_ERR_SHAPE;
    if (scaled && (!(factor >= 1.0) || !(factor <= 1e9))) return SQ_ERR_SHAPE;
    if (scaling == SQ_ROTARY_BASE && rot == 2) return SQ_ERR_SHAPE;       // its exponent divides by rot - 2
    if (scaling == SQ_ROTARY_PARTS && (!(trained > 0.0) || !(low >= 0.0) || !(high > low) || !(high <= 1e18) || !(trained <= 1e18)))
        return SQ_ERR_SHAPE;
    if (!turns) return SQ_ERR_NULL;
    // 64-bit significands: an entry is then right to a few of its units, and the angle of any 32-bit position to 2^-31 of a turn
    // (in 64-bit numbers an entry is off by up to 2^9 and more, the farthest position's angle by more than the fp32 it ends in)
    typedef long double wide;
#ifndef __HIP_DEVICE_COMPILE__                         // the host's; the compiler's pass for the device takes it for 53
    static_assert(std::numeric_limits<wide>::digits >= 64, "an entry has 62 bits");
#endif
    const wide two_pi = 6.283185307179586476925286766559005768L;
    wide b = base;
    if (scaling == SQ_ROTARY_BASE) b *= std::pow((wide)factor, (wide)rot / (wide)(rot - 2));
    for (int i = 0; i < rot / 2; ++i) {
        wide f = std::pow(b, (wide)(-2 * i) / (wide)rot);
        if (scaling == SQ_ROTARY_LINEAR) f /= factor;
        if (scaling == SQ_ROTARY_PARTS) {
            wide keep = ((wide)trained * f / two_pi - low) / ((wide)high - low);
            keep = keep < 0 ? 0 : keep > 1 ? 1 : keep;
            f = f * keep + f / factor * (1 - keep);
        }
        // f <= 1 radian: below 2^62 in units of 2^-64 of a turn
        turns[i] = (uint64_t)std::nearbyint(f / two_pi * 18446744073709551616.0L);
    }
    return SQ_OK;
}

extern "C" sq_status sq_rotary_fp16(const void *X, int64_t T, int32_t H, int32_t D, int64_t ldx, int64_t ldh,
                                    const int32_t *positions, const uint64_t *turns, int32_t rot, int32_t half,
                                    float magnitude, void *Y, int64_t ldy, int64_t ldyh, void *stream)
{
    if (T < 0 || T > SQ_MAX_ROWS || H < 0 || H > 65536 || D <= 0 || D > 65536 || rot < 0 || (rot % 2) != 0 || rot > D ||
        rot > SQ_ROTARY_MAX_CHANNELS)
        return SQ_ERR_SHAPE;
    if (half != 0 && half != 1) return SQ_ERR_SHAPE;
    const int64_t rows = (int64_t)(H > 0 ? H - 1 : 0);
    if (ldh < D || ldyh < D || ldx < rows * ldh + D || ldy < rows * ldyh + D) return SQ_ERR_SHAPE;
    if (T == 0 || H == 0) return SQ_OK;
    if (!X || !Y || (rot > 0 && (!positions || !turns))) return SQ_ERR_NULL;
    if (((uintptr_t)X & 1) || ((uintptr_t)Y & 1) || ((uintptr_t)positions & 3) || ((uintptr_t)turns & 7)) return SQ_ERR_ALIGN;
    const bool in_place = X == Y;
    if (in_place && (ldx != ldy || ldh != ldyh)) return SQ_ERR_SHAPE;
    const __half *x = static_cast<const __half *>(X);
    __half *y = static_cast<__half *>(Y);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int copied = in_place ? 0 : D - rot;
    if (rot == 0 && copied == 0) return SQ_OK;
    // units of 2 V channels need every place of them on a multiple of V
    auto places = [&](int V) {
        return rot % (2 * V) == 0 && ((int64_t)D | ldx | ldh | ldy | ldyh) % V == 0 && (((uintptr_t)X | (uintptr_t)Y) & (2 * V - 1)) == 0;
    };
    if (places(8)) return sq::launch_rotary<8>(x, T, H, D, ldx, ldh, positions, turns, rot, half, magnitude, y, ldy, ldyh, copied, st);
    if (places(4)) return sq::launch_rotary<4>(x, T, H, D, ldx, ldh, positions, turns, rot, half, magnitude, y, ldy, ldyh, copied, st);
    if (places(2)) return sq::launch_rotary<2>(x, T, H, D, ldx, ldh, positions, turns, rot, half, magnitude, y, ldy, ldyh, copied, st);
    const int units = rot / 2 + copied;
    const int64_t blocks = (T * H * units + 255) / 256;
    if (blocks > sq::kMaxBlocks) return SQ_ERR_SHAPE;
    hipLaunchKernelGGL(sq::rotary_pair_kernel, sq::grid_of(blocks), dim3(256), 0, st, x, T, H, D, ldx, ldh, positions, turns, rot, half,
                       magnitude, y, ldy, ldyh, units);
    return hipGetLastError() == hipSuccess ? SQ_OK : SQ_ERR_LAUNCH;
}

// sq_quantize_grouped: rows of fp16 to 4-bit codes with one fp16 step per group of neighbouring channels.
#include "sq_quant4.h"

namespace sq {

namespace {

// One lane takes eight channels (16 bytes in, 4 bytes of codes out); a group is 4, 8, 16 or 32 lanes of a wave.  Rows are
// whole numbers of groups, so units are numbered through all rows and no group crosses a wave.  The pass is one read of X
// and one write of a quarter of that: HBM-bound, with about 60 VALU instructions per 20 bytes under it.  T = 4096, K = 11008,
// groups of 128, 113 MB: 22.0 us (5.2 TB/s), 24.3 where rows are padded and a lane divides to find its own.
template <int LANES, bool STRIDED>
__global__ __launch_bounds__(256) void quantize_grouped_kernel(const __half *__restrict__ X, int64_t units, int units_per_row,
                                                               int64_t ldx, uint32_t *__restrict__ Q,
                                                               __half *__restrict__ steps)
{
    constexpr int U = 4;                                   // units per lane, one block length apart
    const int64_t first = (int64_t)blockIdx.x * (256 * U) + threadIdx.x;
    uint4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t unit = min(first + 256 * u, units - 1);
        const int64_t row = STRIDED ? unit / units_per_row : 0;
        x[u] = *reinterpret_cast<const uint4 *>(X + row * ldx + 8 * (unit - row * units_per_row));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t unit = first + 256 * u;
        const __half s = run_step(run_max<LANES>(x[u]));
        const uint32_t codes = run_codes_plus8(x[u], __builtin_amdgcn_rcpf(__half2float(s))) ^ 0x88888888u;
        if (unit < units) {
            Q[unit] = codes;
            if (unit % LANES == 0) steps[unit / LANES] = s;
        }
    }
}

template <int LANES>
sq_status launch_quantize_grouped(const __half *X, int64_t T, int K, int64_t ldx, uint8_t *Q, __half *steps, hipStream_t st)
{
    const int64_t units = T * (K / 8), blocks = (units + 1023) / 1024;
    uint32_t *Q32 = reinterpret_cast<uint32_t *>(Q);
    if (ldx == K || T == 1)
        hipLaunchKernelGGL((quantize_grouped_kernel<LANES, false>), dim3((unsigned)blocks), dim3(256), 0, st, X, units, K / 8, ldx, Q32, steps);
    else
        hipLaunchKernelGGL((quantize_grouped_kernel<LANES, true>), dim3((unsigned)blocks), dim3(256), 0, st, X, units, K / 8, ldx, Q32, steps);
    return hipGetLastError() == hipSuccess ? SQ_OK : SQ_ERR_LAUNCH;
}

}  // namespace

}  // namespace sq

extern "C" sq_status sq_quantize_grouped(const void *X, int64_t T, int32_t K, int64_t ldx, int32_t group, uint8_t *Q,
                                         void *steps, void *stream)
{
    if (group != 32 && group != 64 && group != 128 && group != 256) return SQ_ERR_SHAPE;
    if (T < 0 || T > SQ_MAX_ROWS || K <= 0 || K > 131072 || (K % group) != 0 || ldx < K) return SQ_ERR_SHAPE;
    if (T * (int64_t)(K / 8) >= (int64_t)1024 << 24) return SQ_ERR_SHAPE;       // a launch counts 2^32 threads; so much of X fills the device
    if (T == 0) return SQ_OK;
    if (!X || !Q || !steps) return SQ_ERR_NULL;
    if (((uintptr_t)X & 15) || (ldx % 8) != 0 || ((uintptr_t)Q & 15) || ((uintptr_t)steps & 1)) return SQ_ERR_ALIGN;
    const __half *Xh = static_cast<const __half *>(X);
    __half *sh = static_cast<__half *>(steps);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (group == 32) return sq::launch_quantize_grouped<4>(Xh, T, K, ldx, Q, sh, st);
    if (group == 64) return sq::launch_quantize_grouped<8>(Xh, T, K, ldx, Q, sh, st);
    if (group == 128) return sq::launch_quantize_grouped<16>(Xh, T, K, ldx, Q, sh, st);
    return sq::launch_quantize_grouped<32>(Xh, T, K, ldx, Q, sh, st);
}

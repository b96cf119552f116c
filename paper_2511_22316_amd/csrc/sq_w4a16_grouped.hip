// sq_w4a16_gemm_grouped: fp16 activations times 4-bit weight codes with one fp16 step per group of K.
//
//   Y[t, n] = fp16( sum_g s[n, g] * sum_{k in g} X[t, k] Qw[n, k] )        fp32 sums
#include "sq_common.h"

namespace sq {

namespace {

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
    const int64_t blocks = (T * N + 3) / 4;
    if (blocks > 0x7FFFFFFF) return SQ_ERR_SHAPE;
    hipLaunchKernelGGL(sq::w4a16_grouped_dot_kernel, dim3((unsigned)blocks), dim3(256), 0, static_cast<hipStream_t>(stream),
                       static_cast<const __half *>(X), ldx, (int)T, K, Qw, static_cast<const __half *>(steps), group, N,
                       static_cast<__half *>(Y), ldy);
    return hipGetLastError() == hipSuccess ? SQ_OK : SQ_ERR_LAUNCH;
}

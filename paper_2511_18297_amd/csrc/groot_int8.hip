// Rows cut to 8 bits with a scale of their own.
#include "groot_dense_device.h"

namespace groot {

namespace {

// one row to a wavefront: its largest magnitude, then its values over scale, halves to even
template <typename T>
__global__ __launch_bounds__(kBlock) void quantize_kernel(const T *__restrict__ X, int64_t x_stride, int8_t *__restrict__ Q, int64_t q_stride,
                                                          float *__restrict__ scale_at, int64_t n, int32_t K)
{
    const int lane = threadIdx.x % kWave;
    for (int64_t row = (int64_t)blockIdx.x * kWavesPerBlock + threadIdx.x / kWave; row < n; row += (int64_t)gridDim.x * kWavesPerBlock) {
    const T *x = X + row * x_stride;
    float top = 0.f;
    bool fine = true;
    for (int32_t k = lane; k < K; k += kWave) {
        const float a = __builtin_fabsf((float)x[k]);
        fine = fine && __builtin_isfinite(a);
        top = fmaxf(top, a);
    }
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    fine = __all(fine);
    const float scale = top * (1.f / 127.f);
    for (int32_t k = lane; k < K; k += kWave)
        Q[row * q_stride + k] = fine && scale > 0.f ? (int8_t)fminf(fmaxf(rintf((float)x[k] / scale), -127.f), 127.f) : (int8_t)0;
    if (lane == 0) scale_at[row] = fine ? scale : __builtin_nanf("");
    }
}

}  // namespace

int launch_quantize_rows(int32_t dtype, const void *X, int64_t x_stride, int8_t *Q, int64_t q_stride, float *scale, int64_t n,
                         int32_t K, void *stream)
{
    const int64_t wanted = (n + kWavesPerBlock - 1) / kWavesPerBlock;
    const uint32_t blocks = wanted < (1 << 20) ? (uint32_t)wanted : 1 << 20;
    hipStream_t s = (hipStream_t)stream;
    if (dtype == GROOT_F32) quantize_kernel<float><<<blocks, kBlock, 0, s>>>((const float *)X, x_stride, Q, q_stride, scale, n, K);
    else if (dtype == GROOT_BF16) quantize_kernel<bf16_t><<<blocks, kBlock, 0, s>>>((const bf16_t *)X, x_stride, Q, q_stride, scale, n, K);
    else quantize_kernel<f16_t><<<blocks, kBlock, 0, s>>>((const f16_t *)X, x_stride, Q, q_stride, scale, n, K);
    return (int)hipGetLastError();
}

}  // namespace groot

// Rows cut to 8 bits with a scale of their own.
#include "groot_tile.h"

namespace groot {

namespace {

// kLanes lanes to a row, 16 bytes a load, kKeep loads of a lane in registers: a row that fits them is read once.  Wider rows read
// the rest a second time, from L2.  8192 rows of 4096 values, float16: 27 us for 101 MB, 3.8 TB/s: a workgroup's way from its loads over
// the maximum to its stores is what the 8 of them on a CU cannot hide.  (With a branch around every load, for its row's end, the
// loads waited for one another: 44 us.)
template <typename T, int kLanes, int kKeep, bool kShort>
__global__ __launch_bounds__(kBlock) void quantize_kernel(const T *__restrict__ X, int64_t x_stride, int8_t *__restrict__ Q, int64_t q_stride,
                                                          float *__restrict__ scale_at, int64_t n, int32_t K)
{
    constexpr int kPer = 16 / sizeof(T), kRows = kBlock / kLanes;
    __shared__ float tops[kWavesPerBlock];
    const int at = threadIdx.x % kLanes;
    const int32_t loads = (K + kPer - 1) / kPer;
    const bool whole = (((uintptr_t)Q | (uintptr_t)q_stride) & (kPer - 1)) == 0;
    for (int64_t first = (int64_t)blockIdx.x * kRows; first < n; first += (int64_t)gridDim.x * kRows) {
        const int64_t row = first + threadIdx.x / kLanes;
        const char *const x = (const char *)(X + (row < n ? row : n - 1) * x_stride);
        auto left = [&](int32_t i) { return ((int64_t)K - (int64_t)i * kPer) * (int64_t)sizeof(T); };
        auto get = [&](int32_t i) { return load16<T>(x + (int64_t)i * 16, left(i), kShort); };
        // no branch around the loads: past the row's end its last 16 bytes come, of which nothing stays
        v4i keep[kKeep];
#pragma unroll
        for (int i = 0; i < kKeep; ++i)
            keep[i] = kShort ? short16<T>(x + (int64_t)(at + i * kLanes) * 16, left(at + i * kLanes)) : raw16(x + (int64_t)(at + i * kLanes) * 16, left(at + i * kLanes));
        uint32_t seen = 0;
#pragma unroll
        for (int i = 0; i < kKeep; ++i) {
            if constexpr (!kShort) keep[i] = cut16(keep[i], left(at + i * kLanes));
            seen = row_look<T>(keep[i], seen);
        }
        for (int32_t i = at + kKeep * kLanes; i < loads; i += kLanes) seen = row_look<T>(get(i), seen);
        float top = row_top_of<(kLanes < kWave ? kLanes : kWave)>(row_top<T>(seen));
        if constexpr (kLanes > kWave) {
            __syncthreads();                                 // the row before has read the maxima
            if (threadIdx.x % kWave == 0) tops[threadIdx.x / kWave] = top;
            __syncthreads();
            static_assert(kWavesPerBlock == 4, "the maxima of four wavefronts");
            top = row_top_of<4>(tops[threadIdx.x % 4]);
        }
        if (row >= n) continue;
        const float scale = row_scale(top);
        auto put = [&](v4i v, int32_t i) {
            int8_t *const to = Q + row * q_stride + (int64_t)i * kPer;
            if (whole && (i + 1) * kPer <= K) {
                row_codes<T>(v, scale, to);
            } else {
                alignas(8) int8_t c[kPer];
                row_codes<T>(v, scale, c);
                for (int k = 0; k < kPer; ++k)
                    if (i * kPer + k < K) to[k] = c[k];
            }
        };
#pragma unroll
        for (int i = 0; i < kKeep; ++i)
            if (at + i * kLanes < loads) put(keep[i], at + i * kLanes);
        for (int32_t i = at + kKeep * kLanes; i < loads; i += kLanes) put(get(i), i);
        if (at == 0) scale_at[row] = scale;
    }
}

template <typename T>
int quantize_launch(const T *X, int64_t x_stride, int8_t *Q, int64_t q_stride, float *scale, int64_t n, int32_t K, hipStream_t stream)
{
    const int64_t loads = ((int64_t)K * sizeof(T) + 15) / 16;
    auto blocks = [&](int rows) {
        const int64_t b = (n + rows - 1) / rows;
        return (uint32_t)(b < (1 << 20) ? b : 1 << 20);
    };
    // as many lanes as a row has loads, up to the workgroup's
    if (K * sizeof(T) < 16) quantize_kernel<T, 16, 1, true><<<blocks(16), kBlock, 0, stream>>>(X, x_stride, Q, q_stride, scale, n, K);
    else if (loads <= 32) quantize_kernel<T, 16, 2, false><<<blocks(16), kBlock, 0, stream>>>(X, x_stride, Q, q_stride, scale, n, K);
    else if (loads <= 256) quantize_kernel<T, 64, 4, false><<<blocks(4), kBlock, 0, stream>>>(X, x_stride, Q, q_stride, scale, n, K);
    else quantize_kernel<T, 256, 4, false><<<blocks(1), kBlock, 0, stream>>>(X, x_stride, Q, q_stride, scale, n, K);
    return (int)hipGetLastError();
}

}  // namespace

int launch_quantize_rows(int32_t dtype, const void *X, int64_t x_stride, int8_t *Q, int64_t q_stride, float *scale, int64_t n,
                         int32_t K, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    if (dtype == GROOT_F32) return quantize_launch((const float *)X, x_stride, Q, q_stride, scale, n, K, s);
    if (dtype == GROOT_BF16) return quantize_launch((const bf16_t *)X, x_stride, Q, q_stride, scale, n, K, s);
    return quantize_launch((const f16_t *)X, x_stride, Q, q_stride, scale, n, K, s);
}

}  // namespace groot

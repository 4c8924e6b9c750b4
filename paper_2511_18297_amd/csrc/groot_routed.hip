// Rows on their way to the experts' places and back:
//   R[places[i,s]] = X[i];   out[i] = addend[i] + sum_s w[i,s] R[places[i,s]];   dR[places[i,s]] = w[i,s] dout[i], dw[i,s] = dout[i] . R[places[i,s]]
// Every kernel goes by the rows i, which know their places: no list of the other direction, no atomics; a slot's row is written by one group
// of lanes.  Bound by HBM: the n k rows at the places are read or written once, the n rows once.
//
// A piece is 16 bytes of a row.  A row's last piece is moved back to end with the row, so that it is whole too: its first values are
// copied or computed twice, alike.  Rows of less than 16 bytes go value by value.
#include "groot_tile.h"

namespace groot {

namespace {

__device__ __forceinline__ int64_t place_at(const RoutedArgs &a, int64_t row, int32_t slot)
{
    const int32_t p = a.places[row * a.k + slot];
    return p >= 0 && p < a.n_places ? p : -1;
}

// where piece `i` of a row of `bytes` begins
__device__ __forceinline__ int64_t piece_at(int64_t i, int64_t bytes) { return i * 16 + 16 <= bytes || bytes < 16 ? i * 16 : bytes - 16; }

// kLanes lanes to a row's kLanes pieces; the numbers of rows and of groups of pieces are the grid's
template <int kLanes>
__global__ __launch_bounds__(kBlock) void routed_rows_kernel(RoutedArgs a, int64_t bytes, int64_t x_bytes, int64_t r_bytes)
{
    const int lane = threadIdx.x % kLanes;
    const int64_t pieces = (bytes + 15) / 16, parts = (pieces + kLanes - 1) / kLanes;
    for (int64_t u = ((int64_t)blockIdx.x * kBlock + threadIdx.x) / kLanes; u < a.n * parts; u += (int64_t)gridDim.x * (kBlock / kLanes)) {
        const int64_t row = u / parts, i = u % parts * kLanes + lane;
        if (i >= pieces) continue;
        const char *const x = (const char *)a.X + row * x_bytes;
        const int64_t at = piece_at(i, bytes);
        v4i v;
        if (bytes >= 16) __builtin_memcpy(&v, x + at, 16);
        const float scale = a.scale_in && i == 0 ? a.scale_in[row] : 0.f;
        for (int32_t s = 0; s < a.k; ++s) {
            const int64_t p = place_at(a, row, s);
            if (p < 0) continue;
            char *const to = (char *)a.out + p * r_bytes;
            if (bytes >= 16) __builtin_memcpy(to + at, &v, 16);
            else
                for (int b = 0; b < (int)bytes; ++b) to[b] = x[b];
            if (a.scale_in && i == 0) a.scale_out[p] = scale;
        }
    }
}

template <typename T>
__device__ __forceinline__ v4i piece_of(const char *row, int64_t at, int32_t K, bool is_short)
{
    if (is_short) return short16<T>(row, K * (int64_t)sizeof(T));
    v4i v;
    __builtin_memcpy(&v, row + at, 16);
    return v;
}
template <typename T>
__device__ __forceinline__ void store_piece(char *row, int64_t at, int32_t K, bool is_short, const float (&x)[16 / sizeof(T)])
{
    constexpr int kPer = 16 / sizeof(T);
    T e[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) e[k] = (T)x[k];           // the one rounding
    if (is_short) {
        for (int k = 0; k < kPer; ++k)
            if (k < K) ((T *)row)[k] = e[k];
    } else {
        __builtin_memcpy(row + at, e, 16);
    }
}

template <typename T, int kLanes>
__global__ __launch_bounds__(kBlock) void routed_sum_kernel(RoutedArgs a)
{
    constexpr int kPer = 16 / sizeof(T);
    const int lane = threadIdx.x % kLanes;
    const int64_t bytes = (int64_t)a.K * sizeof(T), pieces = (bytes + 15) / 16, parts = (pieces + kLanes - 1) / kLanes;
    const bool is_short = bytes < 16;
    for (int64_t u = ((int64_t)blockIdx.x * kBlock + threadIdx.x) / kLanes; u < a.n * parts; u += (int64_t)gridDim.x * (kBlock / kLanes)) {
        const int64_t row = u / parts, i = u % parts * kLanes + lane;
        if (i >= pieces) continue;
        const int64_t at = piece_at(i, bytes);
        float sum[kPer];
        RowValues<T> v{};
        if (a.addend) v = row_values<T>(piece_of<T>((const char *)((const T *)a.addend + row * a.addend_stride), at, a.K, is_short));
#pragma unroll
        for (int e = 0; e < kPer; ++e) sum[e] = v.x[e];
        for (int32_t s = 0; s < a.k; ++s) {
            const int64_t p = place_at(a, row, s);
            const float w = a.weights ? a.weights[row * a.k + s] : 1.f;
            if (p >= 0) v = row_values<T>(piece_of<T>((const char *)((const T *)a.R + p * a.r_stride), at, a.K, is_short));
            else v = RowValues<T>{};                         // no place: a row of zeros, which a weight of NaN still shows in
#pragma unroll
            for (int e = 0; e < kPer; ++e) sum[e] += w * v.x[e];
        }
        store_piece<T>((char *)((T *)a.out + row * a.out_stride), at, a.K, is_short, sum);
    }
}

template <typename T, int kLanes>
__global__ __launch_bounds__(kBlock) void routed_sum_backward_kernel(RoutedArgs a)
{
    constexpr int kPer = 16 / sizeof(T);
    const int lane = threadIdx.x % kLanes;
    const int64_t bytes = (int64_t)a.K * sizeof(T), pieces = (bytes + 15) / 16;
    const bool is_short = bytes < 16;
    for (int64_t row = ((int64_t)blockIdx.x * kBlock + threadIdx.x) / kLanes; row < a.n; row += (int64_t)gridDim.x * (kBlock / kLanes)) {
        const char *const d_row = (const char *)((const T *)a.X + row * a.x_stride);
        for (int32_t s = 0; s < a.k; ++s) {
            const int64_t p = place_at(a, row, s);
            const float w = a.weights ? a.weights[row * a.k + s] : 1.f;
            const char *const r_row = (const char *)((const T *)a.R + (p < 0 ? 0 : p) * a.r_stride);
            float dot = 0.f;
            for (int64_t i = lane; i < pieces && p >= 0; i += kLanes) {
                const int64_t at = piece_at(i, bytes);
                const RowValues<T> d = row_values<T>(piece_of<T>(d_row, at, a.K, is_short));
                if (a.dweights) {
                    const RowValues<T> r = row_values<T>(piece_of<T>(r_row, at, a.K, is_short));
                    const int64_t before = (i * 16 - at) / (int64_t)sizeof(T);    // values that the piece before has counted
#pragma unroll
                    for (int e = 0; e < kPer; ++e) dot += e >= before ? d.x[e] * r.x[e] : 0.f;
                }
                if (a.out) {
                    float x[kPer];
#pragma unroll
                    for (int e = 0; e < kPer; ++e) x[e] = w * d.x[e];
                    store_piece<T>((char *)((T *)a.out + p * a.out_stride), at, a.K, is_short, x);
                }
            }
            if (a.dweights) {
#pragma unroll
                for (int m = 1; m < kLanes; m *= 2) dot += __shfl_xor(dot, m);
                if (lane == 0) a.dweights[row * a.k + s] = dot;
            }
        }
    }
}

uint32_t blocks_for(int64_t units, int lanes)
{
    const int64_t b = (units * lanes + kBlock - 1) / kBlock;
    return (uint32_t)(b < (1 << 20) ? b : 1 << 20);
}

template <typename T>
int sum_launch(const RoutedArgs &a, hipStream_t stream)
{
    const int64_t pieces = ((int64_t)a.K * sizeof(T) + 15) / 16;
    if (pieces <= 16) routed_sum_kernel<T, 16><<<blocks_for(a.n, 16), kBlock, 0, stream>>>(a);
    else routed_sum_kernel<T, 64><<<blocks_for(a.n * ((pieces + 63) / 64), 64), kBlock, 0, stream>>>(a);
    return (int)hipGetLastError();
}
template <typename T>
int sum_backward_launch(const RoutedArgs &a, hipStream_t stream)
{
    const int64_t pieces = ((int64_t)a.K * sizeof(T) + 15) / 16;
    if (pieces <= 16) routed_sum_backward_kernel<T, 16><<<blocks_for(a.n, 16), kBlock, 0, stream>>>(a);
    else routed_sum_backward_kernel<T, 64><<<blocks_for(a.n, 64), kBlock, 0, stream>>>(a);
    return (int)hipGetLastError();
}

}  // namespace

int launch_routed_rows(int32_t value_bytes, const RoutedArgs &a, void *stream)
{
    const int64_t bytes = (int64_t)a.K * value_bytes, pieces = (bytes + 15) / 16;
    hipStream_t s = (hipStream_t)stream;
    if (pieces <= 16) routed_rows_kernel<16><<<blocks_for(a.n, 16), kBlock, 0, s>>>(a, bytes, a.x_stride * value_bytes, a.out_stride * value_bytes);
    else routed_rows_kernel<64><<<blocks_for(a.n * ((pieces + 63) / 64), 64), kBlock, 0, s>>>(a, bytes, a.x_stride * value_bytes, a.out_stride * value_bytes);
    return (int)hipGetLastError();
}

int launch_routed_sum(int32_t dtype, const RoutedArgs &a, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    if (dtype == GROOT_F32) return sum_launch<float>(a, s);
    if (dtype == GROOT_BF16) return sum_launch<bf16_t>(a, s);
    return sum_launch<f16_t>(a, s);
}

int launch_routed_sum_backward(int32_t dtype, const RoutedArgs &a, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    if (dtype == GROOT_F32) return sum_backward_launch<float>(a, s);
    if (dtype == GROOT_BF16) return sum_backward_launch<bf16_t>(a, s);
    return sum_backward_launch<f16_t>(a, s);
}

}  // namespace groot

// Products grouped by node type or expert: every tile of the output belongs to one group, whose weights it takes.
#include "groot_dense_device.h"

namespace groot {

namespace {

constexpr int kTile = 64, kStep = 16;        // output tile, slice of the contraction in LDS

template <typename T>
struct Summed { typedef float type; };
template <>
struct Summed<int8_t> { typedef int32_t type; };

// out[i,:] = epilogue(A[i,:] B[g]): a workgroup takes 64 rows and 64 columns, every lane 4 x 4 of them
template <typename T, typename O, bool kNMajor>
__global__ __launch_bounds__(kBlock) void rows_kernel(const RowsProduct p, int32_t col_tiles)
{
    typedef typename Summed<T>::type S;
    __shared__ S a_s[kStep][kTile + 1], b_s[kStep][kTile + 1];
    const RowTile t = find_tile<kTile>(p.offsets, p.groups, p.n, blockIdx.x / col_tiles);
    if (t.group < 0) return;
    const int32_t j0 = (int32_t)(blockIdx.x % col_tiles) * kTile;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const T *A = (const T *)p.A, *B = (const T *)p.B + (int64_t)t.group * p.K * p.N;
    S acc[4][4] = {};
    for (int32_t k0 = 0; k0 < p.K; k0 += kStep) {
        for (int i = threadIdx.x; i < kStep * kTile; i += kBlock) {
            const int k = i % kStep, r = i / kStep;
            const int64_t row = t.begin + r;
            a_s[k][r] = row < t.end && k0 + k < p.K ? (S)A[row * p.a_stride + k0 + k] : (S)0;
            const int kb = kNMajor ? k : i / kTile, c = kNMajor ? r : i % kTile;
            b_s[kb][c] = j0 + c < p.N && k0 + kb < p.K
                             ? (S)B[kNMajor ? (int64_t)(j0 + c) * p.K + k0 + kb : (int64_t)(k0 + kb) * p.N + j0 + c] : (S)0;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kStep; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] += a_s[k][ty * 4 + i] * b_s[k][tx + 16 * j];
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i) {
        const int64_t row = t.begin + ty * 4 + i;
        if (row >= t.end) break;
        for (int j = 0; j < 4; ++j) {
            const int32_t col = j0 + tx + 16 * j;
            if (col >= p.N) break;
            const int64_t of = (int64_t)t.group * p.N + col;
            float y = (float)acc[i][j];
            if (std::is_same<T, int8_t>::value) {
                y = y * p.a_scale[row] * p.b_scale[of];
                if (p.bias) y += ((const float *)p.bias)[of];
            } else if (p.bias) y += (float)((const T *)p.bias)[of];
            if (p.relu && y < 0.f) y = 0.f;
            ((O *)p.out)[row * p.out_stride + col] = (O)y;
        }
    }
}

// dW[g] = X_g^T dY_g: a workgroup takes 64 x 64 of one group's product and walks over the group's rows
template <typename T, typename O>
__global__ __launch_bounds__(kBlock) void weights_kernel(const WeightsProduct p, int32_t k_tiles, int32_t n_tiles)
{
    __shared__ float a_s[kStep][kTile + 1], b_s[kStep][kTile + 1];
    const int32_t n0 = (int32_t)(blockIdx.x % n_tiles) * kTile, k0 = (int32_t)(blockIdx.x / n_tiles % k_tiles) * kTile;
    const int32_t g = (int32_t)(blockIdx.x / n_tiles / k_tiles);
    int64_t begin, end;
    group_rows(p.offsets, p.n, g, &begin, &end);
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    float acc[4][4] = {}, sums[4] = {};
    for (int64_t r0 = begin; r0 < end; r0 += kStep) {
        for (int i = threadIdx.x; i < kStep * kTile; i += kBlock) {
            const int r = i / kTile, c = i % kTile;
            const int64_t row = r0 + r;
            a_s[r][c] = row < end && k0 + c < p.K ? (float)((const T *)p.X)[row * p.x_stride + k0 + c] : 0.f;
            b_s[r][c] = row < end && n0 + c < p.N ? (float)((const T *)p.dY)[row * p.dy_stride + n0 + c] : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kStep; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float b = b_s[r][tx + 16 * j];
                sums[j] += b;
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i][j] += a_s[r][ty * 4 + i] * b;
            }
        __syncthreads();
    }
    for (int j = 0; j < 4; ++j) {
        const int32_t n = n0 + tx + 16 * j;
        if (n >= p.N) break;
        if (p.dbias && k0 == 0 && ty == 0) ((O *)p.dbias)[(int64_t)g * p.N + n] = (O)sums[j];
        for (int i = 0; i < 4; ++i) {
            const int32_t k = k0 + ty * 4 + i;
            if (k < p.K) ((O *)p.dW)[((int64_t)g * p.K + k) * p.N + n] = (O)acc[i][j];
        }
    }
}

template <typename T, typename O>
int rows_launch(const RowsProduct &p, void *stream)
{
    const int32_t col_tiles = (p.N + kTile - 1) / kTile;
    const int64_t tiles = ((p.n + kTile - 1) / kTile + (p.offsets ? p.groups : 0)) * col_tiles;
    if (p.b_n_major) rows_kernel<T, O, true><<<(uint32_t)tiles, kBlock, 0, (hipStream_t)stream>>>(p, col_tiles);
    else if constexpr (!std::is_same<T, int8_t>::value)
        rows_kernel<T, O, false><<<(uint32_t)tiles, kBlock, 0, (hipStream_t)stream>>>(p, col_tiles);
    return (int)hipGetLastError();
}

template <typename T, typename O>
int weights_launch(const WeightsProduct &p, void *stream)
{
    const int32_t k_tiles = (p.K + kTile - 1) / kTile, n_tiles = (p.N + kTile - 1) / kTile;
    weights_kernel<T, O><<<(uint32_t)((int64_t)p.groups * k_tiles * n_tiles), kBlock, 0, (hipStream_t)stream>>>(p, k_tiles, n_tiles);
    return (int)hipGetLastError();
}

}  // namespace

int launch_grouped_rows(int32_t dtype, const RowsProduct &p, void *stream)
{
    if (dtype == GROOT_F32) return rows_launch<float, float>(p, stream);
    if (dtype == GROOT_BF16) return rows_launch<bf16_t, bf16_t>(p, stream);
    return rows_launch<f16_t, f16_t>(p, stream);
}

int launch_int8_rows(int32_t out_dtype, const RowsProduct &p, void *stream)
{
    if (out_dtype == GROOT_F32) return rows_launch<int8_t, float>(p, stream);
    if (out_dtype == GROOT_BF16) return rows_launch<int8_t, bf16_t>(p, stream);
    return rows_launch<int8_t, f16_t>(p, stream);
}

size_t grouped_weights_workspace(int32_t, int64_t, int32_t, int32_t, int32_t) { return 0; }

int launch_grouped_weights(int32_t dtype, const WeightsProduct &p, void *stream)
{
    if (dtype == GROOT_F32) return weights_launch<float, float>(p, stream);
    if (dtype == GROOT_BF16) return p.grad_f32 ? weights_launch<bf16_t, float>(p, stream) : weights_launch<bf16_t, bf16_t>(p, stream);
    return p.grad_f32 ? weights_launch<f16_t, float>(p, stream) : weights_launch<f16_t, f16_t>(p, stream);
}

}  // namespace groot

// Products grouped by node type or expert: every tile of the output belongs to one group, whose weights it takes.
#include "groot_tile.h"

namespace groot {

namespace {

// out[i,:] = epilogue(A[i,:] B[g]): a workgroup takes kM rows of a group and kN columns, a wavefront kM / kWavesM x kN / kWavesN
template <typename T, typename O, int kM, int kN, int kWavesM, int kWavesN, bool kNMajor, bool kAligned>
__global__ __launch_bounds__(kWavesM *kWavesN *kWave) void rows_kernel(const RowsProduct p, const TileOrder order, int32_t col_tiles, bool whole)
{
    constexpr int kThreads = kWavesM * kWavesN * kWave, kI = kM / kWavesM / 32, kJ = kN / kWavesN / 32;
    typedef Stage<T, kM, kThreads, false, kAligned> StageA;
    typedef Stage<T, kN, kThreads, !kNMajor, kAligned> StageB;
    __shared__ __align__(16) char lds[2 * (StageA::kBytes + StageB::kBytes)];
    int64_t row_tile;
    int32_t col_tile;
    order.find(blockIdx.x, &row_tile, &col_tile);
    if (col_tile >= col_tiles) return;
    const RowTile t = find_tile<kM>(p.offsets, p.groups, p.n, row_tile);
    if (t.group < 0) return;
    const int32_t j0 = col_tile * kN;
    const int64_t rows = t.end - t.begin;
    const T *B = (const T *)p.B + (int64_t)t.group * p.K * p.N;
    StageA a;
    StageB b;
    a.init((const T *)p.A + t.begin * p.a_stride, p.a_stride, rows, p.K);
    if (kNMajor) b.init(B + (int64_t)j0 * p.K, p.K, p.N - j0, p.K);
    else b.init(B + j0, p.N, p.N - j0, p.K);
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int row0 = wave / kWavesN * (kM / kWavesM), col0 = wave % kWavesN * (kN / kWavesN);
    typename TileType<T>::Sum sums[kI][kJ];
    tile_product<T>(a, b, lds, (p.K + kStepValues<T> - 1) / kStepValues<T>, row0, col0, sums);
#pragma unroll
    for (int j = 0; j < kJ; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int32_t col = j0 + col0 + 32 * j + 8 * q + 4 * (lane / 32), left = p.N - col;
            if (left <= 0) continue;
            const int64_t of = (int64_t)t.group * p.N + col;
            v4f bias = {0.f, 0.f, 0.f, 0.f}, scale = {1.f, 1.f, 1.f, 1.f};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (k >= left) break;
                if (std::is_same<T, int8_t>::value) {
                    scale[k] = p.b_scale[of + k];
                    if (p.bias) bias[k] = ((const float *)p.bias)[of + k];
                } else if (p.bias) bias[k] = (float)((const O *)p.bias)[of + k];
            }
#pragma unroll
            for (int i = 0; i < kI; ++i) {
                const int64_t r = row0 + 32 * i + lane % 32;
                if (r >= rows) continue;
                const int64_t row = t.begin + r;
                v4f y;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    y[k] = (float)sums[i][j][4 * q + k];
                    if (std::is_same<T, int8_t>::value) y[k] = y[k] * p.a_scale[row] * scale[k];
                    if (p.bias) y[k] += bias[k];
                    if (p.relu && y[k] < 0.f) y[k] = 0.f;
                }
                store_quad((O *)p.out + row * p.out_stride + col, y, left, whole);
            }
        }
}

bool on16(const void *a, int64_t bytes) { return (((uintptr_t)a | (uintptr_t)bytes) & 15) == 0; }

template <typename T, typename O, int kM, int kN, int kWavesM, int kWavesN, bool kNMajor>
int rows_launch(const RowsProduct &p, void *stream)
{
    const int32_t col_tiles = (p.N + kN - 1) / kN;
    const TileOrder order((p.n + kM - 1) / kM + (p.offsets ? p.groups : 0), col_tiles);
    const int64_t b = sizeof(T);
    const bool aligned = on16(p.A, p.a_stride * b) && on16(p.B, (kNMajor ? p.K : p.N) * b) && p.K * b % 16 == 0;
    const bool whole = (((uintptr_t)p.out | (uintptr_t)(p.out_stride * sizeof(O))) & (4 * sizeof(O) - 1)) == 0;
    constexpr int kThreads = kWavesM * kWavesN * kWave;
    if (aligned) rows_kernel<T, O, kM, kN, kWavesM, kWavesN, kNMajor, true><<<order.workgroups, kThreads, 0, (hipStream_t)stream>>>(p, order, col_tiles, whole);
    else rows_kernel<T, O, kM, kN, kWavesM, kWavesN, kNMajor, false><<<order.workgroups, kThreads, 0, (hipStream_t)stream>>>(p, order, col_tiles, whole);
    return (int)hipGetLastError();
}

template <typename T, typename O, bool kNMajor>
int rows_choose(const RowsProduct &p, void *stream)
{
    const int64_t each = p.n / p.groups;                      // rows of a group, on average
    if (p.N <= 64) return rows_launch<T, O, 128, 64, 4, 1, kNMajor>(p, stream);
    if (each >= 192 && p.n * p.N >= (int64_t)256 * 256 * 128) return rows_launch<T, O, 256, 256, 2, 4, kNMajor>(p, stream);
    if (each > 32) return rows_launch<T, O, 128, 128, 2, 2, kNMajor>(p, stream);
    return rows_launch<T, O, 32, 128, 1, 4, kNMajor>(p, stream);
}

// dW[g] = X_g^T dY_g: a workgroup takes kK x kN of one group's product and walks over the group's rows
template <typename T, typename O, int kK, int kN, int kWavesK, int kWavesN, bool kAligned>
__global__ __launch_bounds__(kWavesK *kWavesN *kWave) void weights_kernel(const WeightsProduct p, int32_t k_tiles, int32_t n_tiles)
{
    constexpr int kThreads = kWavesK * kWavesN * kWave, kI = kK / kWavesK / 32, kJ = kN / kWavesN / 32;
    typedef Stage<T, kK, kThreads, true, kAligned> StageX;
    typedef Stage<T, kN, kThreads, true, kAligned> StageY;
    __shared__ __align__(16) char lds[2 * (StageX::kBytes + StageY::kBytes)];
    const int32_t n0 = (int32_t)(blockIdx.x % n_tiles) * kN, k0 = (int32_t)(blockIdx.x / n_tiles % k_tiles) * kK;
    const int32_t g = (int32_t)(blockIdx.x / n_tiles / k_tiles);
    int64_t begin, end;
    group_rows(p.offsets, p.n, g, &begin, &end);
    StageX x;
    StageY y;
    x.init((const T *)p.X + begin * p.x_stride + k0, p.x_stride, p.K - k0, end - begin);
    y.init((const T *)p.dY + begin * p.dy_stride + n0, p.dy_stride, p.N - n0, end - begin);
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int row0 = wave / kWavesN * (kK / kWavesK), col0 = wave % kWavesN * (kN / kWavesN);
    typename TileType<T>::Sum sums[kI][kJ];
    tile_product<T>(x, y, lds, (end - begin + kStepValues<T> - 1) / kStepValues<T>, row0, col0, sums);
    const bool whole = p.N % 4 == 0 && ((uintptr_t)p.dW & (4 * sizeof(O) - 1)) == 0;
#pragma unroll
    for (int i = 0; i < kI; ++i) {
        const int32_t k = k0 + row0 + 32 * i + lane % 32;
        if (k >= p.K) continue;
#pragma unroll
        for (int j = 0; j < kJ; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int32_t n = n0 + col0 + 32 * j + 8 * q + 4 * (lane / 32);
                if (n >= p.N) continue;
                const v4f v = {sums[i][j][4 * q], sums[i][j][4 * q + 1], sums[i][j][4 * q + 2], sums[i][j][4 * q + 3]};
                store_quad((O *)p.dW + ((int64_t)g * p.K + k) * p.N + n, v, p.N - n, whole);
            }
    }
}

// dbias[g] = column sums of dY_g: 64 columns to a workgroup, its wavefronts take every fourth row
template <typename T, typename O>
__global__ __launch_bounds__(kBlock) void bias_kernel(const WeightsProduct p, int32_t n_tiles)
{
    __shared__ float part[kWavesPerBlock][kWave];
    const int32_t n = (int32_t)(blockIdx.x % n_tiles) * kWave + threadIdx.x % kWave, g = (int32_t)(blockIdx.x / n_tiles);
    int64_t begin, end;
    group_rows(p.offsets, p.n, g, &begin, &end);
    float s = 0.f;
    if (n < p.N)
        for (int64_t r = begin + threadIdx.x / kWave; r < end; r += kWavesPerBlock) s += (float)((const T *)p.dY)[r * p.dy_stride + n];
    part[threadIdx.x / kWave][threadIdx.x % kWave] = s;
    __syncthreads();
    if (threadIdx.x < kWave && n < p.N) {
        for (int w = 1; w < kWavesPerBlock; ++w) s += part[w][threadIdx.x];
        ((O *)p.dbias)[(int64_t)g * p.N + n] = (O)s;
    }
}

template <typename T, typename O>
int weights_launch(const WeightsProduct &p, void *stream)
{
    constexpr int kK = 128, kN = 128;
    const int32_t k_tiles = (p.K + kK - 1) / kK, n_tiles = (p.N + kN - 1) / kN;
    const int64_t b = sizeof(T);
    const bool aligned = on16(p.X, p.x_stride * b) && on16(p.dY, p.dy_stride * b) && p.K * b % 16 == 0 && p.N * b % 16 == 0;
    const uint32_t blocks = (uint32_t)((int64_t)p.groups * k_tiles * n_tiles);
    if (aligned) weights_kernel<T, O, kK, kN, 2, 2, true><<<blocks, kBlock, 0, (hipStream_t)stream>>>(p, k_tiles, n_tiles);
    else weights_kernel<T, O, kK, kN, 2, 2, false><<<blocks, kBlock, 0, (hipStream_t)stream>>>(p, k_tiles, n_tiles);
    if (p.dbias) {
        const int32_t tiles = (p.N + kWave - 1) / kWave;
        bias_kernel<T, O><<<(uint32_t)((int64_t)p.groups * tiles), kBlock, 0, (hipStream_t)stream>>>(p, tiles);
    }
    return (int)hipGetLastError();
}

}  // namespace

int launch_grouped_rows(int32_t dtype, const RowsProduct &p, void *stream)
{
    if (dtype == GROOT_F32) return p.b_n_major ? rows_choose<float, float, true>(p, stream) : rows_choose<float, float, false>(p, stream);
    if (dtype == GROOT_BF16) return p.b_n_major ? rows_choose<bf16_t, bf16_t, true>(p, stream) : rows_choose<bf16_t, bf16_t, false>(p, stream);
    return p.b_n_major ? rows_choose<f16_t, f16_t, true>(p, stream) : rows_choose<f16_t, f16_t, false>(p, stream);
}

int launch_int8_rows(int32_t out_dtype, const RowsProduct &p, void *stream)
{
    if (out_dtype == GROOT_F32) return rows_choose<int8_t, float, true>(p, stream);
    if (out_dtype == GROOT_BF16) return rows_choose<int8_t, bf16_t, true>(p, stream);
    return rows_choose<int8_t, f16_t, true>(p, stream);
}

size_t grouped_weights_workspace(int32_t, int64_t, int32_t, int32_t, int32_t) { return 0; }

int launch_grouped_weights(int32_t dtype, const WeightsProduct &p, void *stream)
{
    if (dtype == GROOT_F32) return weights_launch<float, float>(p, stream);
    if (dtype == GROOT_BF16) return p.grad_f32 ? weights_launch<bf16_t, float>(p, stream) : weights_launch<bf16_t, bf16_t>(p, stream);
    return p.grad_f32 ? weights_launch<f16_t, float>(p, stream) : weights_launch<f16_t, f16_t>(p, stream);
}

}  // namespace groot

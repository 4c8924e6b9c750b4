// Root-mean-square norm of rows, with the residual's addition in front, an output in 8 bits behind, and its gradients.
//   h = x + residual, rounded to the type;  rstd = 1 / sqrt(mean h^2 + eps), in 64 bits and rounded once;  y = (h rstd) gain in fp32
//   scale = max |y| fl(1 / 127), codes = y / scale to the nearest
//   dx = rstd (a - h rstd^2 mean(a h)) + dh with a = dy gain;  dgain = sum over the rows of dy (h rstd)
// The sum of the squares is in 64 bits so that rstd, and with it every code, is the same whatever order the lanes add in.
// Bound by HBM: a row is read once and stays in registers as it is held.
//
// A piece is 16 bytes of a row; the last one is moved back to end with the row, so that it is whole too: its first values are computed
// twice, alike, and counted once.  Rows of less than 16 bytes go value by value.
#include "groot_tile.h"

namespace groot {

namespace {

template <typename T>
struct Piece {
    int64_t at;                              // byte of the row
    int first;                               // values that the piece before has counted; all of them where there is no such piece
    bool real;
};

template <typename T>
__device__ __forceinline__ Piece<T> piece(int32_t i, int32_t K)
{
    constexpr int kPer = 16 / sizeof(T);
    const int32_t begin = i * kPer;
    if (K < kPer) return Piece<T>{0, i == 0 ? 0 : kPer, i == 0};
    if (begin >= K) return Piece<T>{(int64_t)(K - kPer) * (int64_t)sizeof(T), kPer, false};
    const int32_t at = begin + kPer <= K ? begin : K - kPer;
    return Piece<T>{(int64_t)at * (int64_t)sizeof(T), begin - at, true};
}

template <typename T, bool kShort>
__device__ __forceinline__ v4i load_piece(const T *row, int64_t at, int32_t K)
{
    if constexpr (kShort) return short16<T>((const char *)row, (int64_t)K * (int64_t)sizeof(T));
    v4i v;
    __builtin_memcpy(&v, (const char *)row + at, 16);
    return v;
}
template <typename T, bool kShort>
__device__ __forceinline__ void store_held(T *row, int64_t at, int32_t K, v4i v)
{
    if constexpr (kShort) {
        T e[16 / sizeof(T)];
        __builtin_memcpy(e, &v, 16);
#pragma unroll
        for (int k = 0; k < (int)(16 / sizeof(T)); ++k)
            if (k < K) row[k] = e[k];
    } else {
        __builtin_memcpy((char *)row + at, &v, 16);
    }
}
template <typename T>
__device__ __forceinline__ v4i rounded(const RowValues<T> &x)
{
    constexpr int kPer = 16 / sizeof(T);
    T e[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) e[k] = (T)x.x[k];         // the one rounding
    v4i v;
    __builtin_memcpy(&v, e, 16);
    return v;
}

// Sums and maxima over the kLanes lanes of a row; every lane has them.  `lds`: a word for each wavefront of the row, twice.
template <int kLanes>
__device__ __forceinline__ double row_sum(double x, double *lds)
{
#pragma unroll
    for (int d = 1; d < (kLanes < kWave ? kLanes : kWave); d *= 2) x += __shfl_xor(x, d);
    if constexpr (kLanes > kWave) {
        __syncthreads();                                     // the row before has read its words
        if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = x;
        __syncthreads();
        x = 0;
#pragma unroll
        for (int w = 0; w < kLanes / kWave; ++w) x += lds[w];
    }
    return x;
}
template <int kLanes>
__device__ __forceinline__ float row_most(float x, double *lds)
{
    x = row_top_of<(kLanes < kWave ? kLanes : kWave)>(x);
    if constexpr (kLanes > kWave) {
        float *const tops = (float *)lds;
        __syncthreads();
        if (threadIdx.x % kWave == 0) tops[threadIdx.x / kWave] = x;
        __syncthreads();
        x = row_top_of<kLanes / kWave>(tops[threadIdx.x % (kLanes / kWave)]);
    }
    return x;
}

constexpr int block_of(int lanes) { return lanes > kBlock ? lanes : kBlock; }

template <typename T, int kLanes, int kKeep, bool kShort>
__global__ __launch_bounds__(block_of(kLanes)) void norm_kernel(NormArgs a)
{
    constexpr int kPer = 16 / sizeof(T), kThreads = block_of(kLanes), kRows = kThreads / kLanes;
    __shared__ double words[kThreads / kWave];
    const int lane = threadIdx.x % kLanes;
    const T *const gain = (const T *)a.gain;
    for (int64_t first = (int64_t)blockIdx.x * kRows; first < a.n; first += (int64_t)gridDim.x * kRows) {
        const int64_t mine = first + threadIdx.x / kLanes, row = mine < a.n ? mine : a.n - 1;   // rows beyond the last go along and store nothing
        const T *const x = (const T *)a.X + row * a.x_stride;
        v4i h[kKeep];
        double sum = 0;
#pragma unroll
        for (int i = 0; i < kKeep; ++i) h[i] = load_piece<T, kShort>(x, piece<T>(i * kLanes + lane, a.K).at, a.K);
        if (a.residual) {
            const T *const r = (const T *)a.residual + row * a.residual_stride;
#pragma unroll
            for (int i = 0; i < kKeep; ++i) {
                RowValues<T> u = row_values<T>(h[i]);
                const RowValues<T> v = row_values<T>(load_piece<T, kShort>(r, piece<T>(i * kLanes + lane, a.K).at, a.K));
#pragma unroll
                for (int e = 0; e < kPer; ++e) u.x[e] += v.x[e];
                h[i] = rounded<T>(u);
            }
        }
#pragma unroll
        for (int i = 0; i < kKeep; ++i) {
            const int counted = piece<T>(i * kLanes + lane, a.K).first;
            const RowValues<T> u = row_values<T>(h[i]);
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const double v = e >= counted ? (double)u.x[e] : 0.0;
                sum = __builtin_fma(v, v, sum);
            }
        }
        sum = row_sum<kLanes>(sum, words);
        const float rstd = (float)(1.0 / sqrt(sum / a.K + a.eps));
        const bool real = mine < a.n;
        auto values = [&](int i, int64_t at) {
            RowValues<T> u = row_values<T>(h[i]);
            const RowValues<T> g = gain ? row_values<T>(load_piece<T, kShort>(gain, at, a.K)) : RowValues<T>{};
#pragma unroll
            for (int e = 0; e < kPer; ++e) u.x[e] = gain ? (u.x[e] * rstd) * g.x[e] : u.x[e] * rstd;
            return u;
        };
        uint32_t seen = 0;
#pragma unroll
        for (int i = 0; i < kKeep; ++i) {
            const Piece<T> p = piece<T>(i * kLanes + lane, a.K);
            if (!p.real) continue;
            if (real && a.H) store_held<T, kShort>((T *)a.H + row * a.h_stride, p.at, a.K, h[i]);
            const RowValues<T> y = values(i, p.at);
            if (real && a.Y) store_held<T, kShort>((T *)a.Y + row * a.y_stride, p.at, a.K, rounded<T>(y));
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const uint32_t m = __float_as_uint(y.x[e]) & 0x7FFFFFFFu;
                if (!kShort || e < a.K) seen = m > seen ? m : seen;
            }
        }
        if (real && a.rstd && lane == 0) a.rstd[row] = rstd;
        if (a.Q) {
            const float scale = row_scale(row_most<kLanes>(__uint_as_float(seen), words));
            if (real && lane == 0) a.q_scale[row] = scale;
#pragma unroll
            for (int i = 0; i < kKeep; ++i) {
                const Piece<T> p = piece<T>(i * kLanes + lane, a.K);
                if (!p.real || !real) continue;
                const RowValues<T> y = values(i, p.at);
                alignas(8) int8_t codes[kPer];
#pragma unroll
                for (int e = 0; e < kPer; e += 4) {
                    const v4f four = {y.x[e], y.x[e + 1], y.x[e + 2], y.x[e + 3]};
                    row_codes<float>(__builtin_bit_cast(v4i, four), scale, codes + e);
                }
                int8_t *const to = a.Q + row * a.q_stride + p.at / (int64_t)sizeof(T);
                if constexpr (kShort) {
#pragma unroll
                    for (int e = 0; e < kPer; ++e)
                        if (e < a.K) to[e] = codes[e];
                } else {
                    __builtin_memcpy(to, codes, kPer);
                }
            }
        }
    }
}

// The rows of a workgroup add up their part of the gain's gradient, each lane its own columns; the parts meet in norm_gain_kernel.
template <typename T, int kLanes, int kKeep, bool kShort>
__global__ __launch_bounds__(block_of(kLanes)) void norm_backward_kernel(NormBackwardArgs a)
{
    constexpr int kPer = 16 / sizeof(T), kThreads = block_of(kLanes), kRows = kThreads / kLanes;
    __shared__ double words[kThreads / kWave];
    const int lane = threadIdx.x % kLanes;
    const T *const gain = (const T *)a.gain;
    float parts[kKeep][kPer] = {};
    for (int64_t first = (int64_t)blockIdx.x * kRows; first < a.n; first += (int64_t)gridDim.x * kRows) {
        const int64_t mine = first + threadIdx.x / kLanes, row = mine < a.n ? mine : a.n - 1;
        const bool real = mine < a.n;
        const float rstd = a.rstd[row];
        v4i h[kKeep], dy[kKeep];
#pragma unroll
        for (int i = 0; i < kKeep; ++i) {
            const int64_t at = piece<T>(i * kLanes + lane, a.K).at;
            h[i] = load_piece<T, kShort>((const T *)a.H + row * a.h_stride, at, a.K);
            dy[i] = load_piece<T, kShort>((const T *)a.dY + row * a.dy_stride, at, a.K);
        }
        auto scaled = [&](int i, int64_t at) {
            RowValues<T> u = row_values<T>(dy[i]);
            if (gain) {
                const RowValues<T> g = row_values<T>(load_piece<T, kShort>(gain, at, a.K));
#pragma unroll
                for (int e = 0; e < kPer; ++e) u.x[e] *= g.x[e];
            }
            return u;
        };
        double sum = 0;
#pragma unroll
        for (int i = 0; i < kKeep; ++i) {
            const Piece<T> p = piece<T>(i * kLanes + lane, a.K);
            const RowValues<T> u = scaled(i, p.at), x = row_values<T>(h[i]), d = row_values<T>(dy[i]);
            float here = 0.f;
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const bool counts = e >= p.first && (!kShort || e < a.K);
                here += counts ? u.x[e] * x.x[e] : 0.f;
                parts[i][e] += counts && real ? d.x[e] * (x.x[e] * rstd) : 0.f;
            }
            sum += here;
        }
        sum = row_sum<kLanes>(sum, words);
        const float c = rstd * rstd * (float)(sum / a.K);
        if (!real) continue;
#pragma unroll
        for (int i = 0; i < kKeep; ++i) {
            const Piece<T> p = piece<T>(i * kLanes + lane, a.K);
            if (!p.real) continue;
            RowValues<T> u = scaled(i, p.at);
            const RowValues<T> x = row_values<T>(h[i]);
#pragma unroll
            for (int e = 0; e < kPer; ++e) u.x[e] = rstd * (u.x[e] - x.x[e] * c);
            if (a.dH) {
                const RowValues<T> v = row_values<T>(load_piece<T, kShort>((const T *)a.dH + row * a.dh_stride, p.at, a.K));
#pragma unroll
                for (int e = 0; e < kPer; ++e) u.x[e] += v.x[e];
            }
            store_held<T, kShort>((T *)a.dX + row * a.dx_stride, p.at, a.K, rounded<T>(u));
        }
    }
    if (!a.dgain) return;
    // each group of lanes writes its own sums: [workgroups * kRows, K]
    float *const to = a.partial + ((int64_t)blockIdx.x * kRows + threadIdx.x / kLanes) * a.K;
#pragma unroll
    for (int i = 0; i < kKeep; ++i) {
        const Piece<T> p = piece<T>(i * kLanes + lane, a.K);
        const int32_t begin = (int32_t)(p.at / (int64_t)sizeof(T));
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            if (p.real && e >= p.first && begin + e < a.K) to[begin + e] = parts[i][e];
    }
}

constexpr int kGainCols = 32, kGainRows = 32;

template <typename O>
__global__ __launch_bounds__(1024) void norm_gain_kernel(const float *__restrict__ partial, int64_t groups, int32_t K, O *__restrict__ dgain)
{
    __shared__ double sums[kGainRows][kGainCols];
    const int col = threadIdx.x % kGainCols, part = threadIdx.x / kGainCols;
    const int32_t k = blockIdx.x * kGainCols + col;
    double sum = 0;
    if (k < K)
        for (int64_t g = part; g < groups; g += kGainRows) sum += (double)partial[g * K + k];
    sums[part][col] = sum;
    __syncthreads();
    if (part || k >= K) return;
    for (int p = 1; p < kGainRows; ++p) sum += sums[p][col];
    dgain[k] = (O)sum;
}

// lanes of a row, and its pieces in each, by the pieces that it has
struct NormShape {
    int lanes, keep;
    bool is_short;
};
NormShape norm_shape(int32_t K, int bytes)
{
    const int64_t pieces = ((int64_t)K * bytes + 15) / 16;
    if (K * (int64_t)bytes < 16) return {16, 1, true};
    if (pieces <= 16) return {16, 1, false};
    if (pieces <= 64) return {64, 1, false};
    if (pieces <= 256) return {64, 4, false};
    if (pieces <= 1024) return {256, 4, false};
    if (pieces <= 2048) return {256, 8, false};
    if (pieces <= 8192) return {1024, 8, false};
    return {1024, 16, false};
}

int64_t norm_blocks(int64_t n, const NormShape &s, int64_t most)
{
    const int rows = block_of(s.lanes) / s.lanes;
    const int64_t b = (n + rows - 1) / rows;
    return b < most ? b : most;
}
constexpr int64_t kBackwardBlocks = 512;

#define GROOT_NORM_SHAPES(use)                                                                                                           \
    if (s.is_short) use(16, 1, true)                                                                                                     \
    else if (s.lanes == 16) use(16, 1, false)                                                                                            \
    else if (s.lanes == 64 && s.keep == 1) use(64, 1, false)                                                                             \
    else if (s.lanes == 64) use(64, 4, false)                                                                                            \
    else if (s.lanes == 256 && s.keep == 4) use(256, 4, false)                                                                           \
    else if (s.lanes == 256) use(256, 8, false)                                                                                          \
    else if (s.keep == 8) use(1024, 8, false)                                                                                            \
    else use(1024, 16, false)

template <typename T>
int norm_launch(const NormArgs &a, hipStream_t stream)
{
    const NormShape s = norm_shape(a.K, sizeof(T));
    const uint32_t blocks = (uint32_t)norm_blocks(a.n, s, 1 << 20);
#define GROOT_NORM(lanes, keep, is_short) { norm_kernel<T, lanes, keep, is_short><<<blocks, block_of(lanes), 0, stream>>>(a); }
    GROOT_NORM_SHAPES(GROOT_NORM)
#undef GROOT_NORM
    return (int)hipGetLastError();
}

template <typename T>
int norm_backward_launch(const NormBackwardArgs &a, hipStream_t stream)
{
    const NormShape s = norm_shape(a.K, sizeof(T));
    const uint32_t blocks = (uint32_t)norm_blocks(a.n, s, kBackwardBlocks);
#define GROOT_NORM(lanes, keep, is_short) { norm_backward_kernel<T, lanes, keep, is_short><<<blocks, block_of(lanes), 0, stream>>>(a); }
    if (blocks) { GROOT_NORM_SHAPES(GROOT_NORM) }
#undef GROOT_NORM
    if (a.dgain) {
        const uint32_t cols = (a.K + kGainCols - 1) / kGainCols;
        const int64_t groups = (int64_t)blocks * (block_of(s.lanes) / s.lanes);
        if (a.grad_f32) norm_gain_kernel<<<cols, 1024, 0, stream>>>(a.partial, groups, a.K, (float *)a.dgain);
        else norm_gain_kernel<<<cols, 1024, 0, stream>>>(a.partial, groups, a.K, (T *)a.dgain);
    }
    return (int)hipGetLastError();
}

}  // namespace

size_t norm_backward_workspace(int32_t dtype, int64_t n, int32_t K)
{
    const NormShape s = norm_shape(K, dtype == GROOT_F32 ? 4 : 2);
    return (size_t)norm_blocks(n, s, kBackwardBlocks) * (block_of(s.lanes) / s.lanes) * K * sizeof(float);
}

int launch_norm(int32_t dtype, const NormArgs &a, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    if (dtype == GROOT_F32) return norm_launch<float>(a, s);
    if (dtype == GROOT_BF16) return norm_launch<bf16_t>(a, s);
    return norm_launch<f16_t>(a, s);
}

int launch_norm_backward(int32_t dtype, const NormBackwardArgs &a, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    if (dtype == GROOT_F32) return norm_backward_launch<float>(a, s);
    if (dtype == GROOT_BF16) return norm_backward_launch<bf16_t>(a, s);
    return norm_backward_launch<f16_t>(a, s);
}

}  // namespace groot

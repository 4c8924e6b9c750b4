// Few rows against weights whose rows lie along the contraction ([groups, N, K]: the 8-bit products, the input gradients): a
// workgroup takes up to 16 rows of a group and 16 columns, and its eight wavefronts share the contraction, 128 bytes of every
// weight row in turn, straight from memory into the fragments of the 16 x 16 matrix instructions.  Nothing is staged: the weights
// are read once and are nearly everything that is read.  A lane has 32 neighbouring bytes of a step (two instructions), so that
// four lanes read a row's 128 bytes.  The wavefronts' sums meet in LDS.
// groot_quantized_linear on up to four rows: every workgroup cuts the rows to 8 bits by itself, into LDS, while its first weights are
// on their way: one launch in place of two.
#include "groot_tile.h"

namespace groot {

namespace {

constexpr int kFewRows = 16, kFewCols = 16, kFewWaves = 8, kFewThreads = kFewWaves * kWave, kAhead = 4;
constexpr int kFusedRows = 4, kFusedBytes = 48 * 1024;       // rows that are cut inside, their bytes in LDS

constexpr int32_t few_tiles(int32_t N, int cols) { return (N + cols - 1) / cols; }
int64_t few_workgroups(const RowsProduct &p, int cols)
{
    return ((p.n + kFewRows - 1) / kFewRows + (p.offsets ? p.groups : 0)) * few_tiles(p.N, cols);
}

template <typename T>
struct FewType;
template <>
struct FewType<int8_t> {
    typedef v4i Sum;
    static __device__ __forceinline__ Sum mma(v4i a, v4i b, Sum c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }
};
template <>
struct FewType<bf16_t> {
    typedef v4f Sum;
    static __device__ __forceinline__ Sum mma(v4i a, v4i b, Sum c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
    }
};
template <>
struct FewType<f16_t> {
    typedef v4f Sum;
    static __device__ __forceinline__ Sum mma(v4i a, v4i b, Sum c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
    }
};
template <>
struct FewType<float> {
    typedef v4f Sum;
    static __device__ __forceinline__ Sum mma(v4i a, v4i b, Sum c)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__int_as_float(a[j]), __int_as_float(b[j]), c, 0, 0, 0);
        return c;
    }
};

// 16 bytes at offset k of a row of `bytes`, zeros behind its end
template <typename T, bool kAligned>
__device__ __forceinline__ v4i piece16(const char *row, int64_t k, int64_t bytes, bool short_row)
{
    if constexpr (kAligned) return k < bytes ? *(const v4i *)(row + k) : v4i{0, 0, 0, 0};
    else return load16<T>(row + k, bytes - k, short_row);
}

// X: the floating type of the rows where they are cut to 8 bits inside, else T
template <typename T, typename O, typename X, bool kAligned>
__global__ __launch_bounds__(kFewThreads) void few_kernel(const RowsProduct p, int32_t col_tiles)
{
#pragma clang fp contract(off)
    constexpr bool kFused = !std::is_same<X, T>::value;
    typedef typename FewType<T>::Sum Sum;
    __shared__ Sum part[kFewWaves][kWave];
    __shared__ float tops[kFusedRows][kFewWaves];
    extern __shared__ __align__(16) char cut[];              // fused: the rows in 8 bits
    const RowTile t = find_tile(p.offsets, p.groups, p.n, blockIdx.x / col_tiles, 4);
    if (t.group < 0) return;
    const int32_t n0 = (int32_t)(blockIdx.x % col_tiles) * kFewCols;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, r = lane % 16, quarter = lane / 16 * 32;
    const int rows = (int)(t.end - t.begin);
    const int64_t bytes = (int64_t)p.K * sizeof(T);
    const int32_t col = n0 + r < p.N ? n0 + r : p.N - 1;     // columns and rows that do not exist read the last one that does
    const char *const w = (const char *)((const T *)p.B + ((int64_t)t.group * p.N + col) * p.K) + quarter;
    const bool short_row = bytes < 16;
    const int32_t pieces = (int32_t)((bytes + kStepBytes - 1) / kStepBytes);

    v4i held[kAhead][2];
    auto load = [&](int32_t s, int i) {
        const int64_t k = (int64_t)s * kStepBytes;
        held[i][0] = piece16<T, kAligned>(w, k, bytes - quarter, short_row);
        held[i][1] = piece16<T, kAligned>(w, k + 16, bytes - quarter, short_row);
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
        if (wave + i * kFewWaves < pieces) load(wave + i * kFewWaves, i);

    const char *x;
    float x_scale = 1.f;
    const int32_t cut_row = (p.K + 127) / 128 * 128;
    if constexpr (kFused) {
        constexpr int kPer = 16 / sizeof(X), kKeep = 2;      // values of a load, loads of a lane that stay in registers
        const int32_t loads = (p.K + kPer - 1) / kPer;
        v4i keep[kFusedRows][kKeep];
        const auto from = [&](int m, int32_t i) { return (const char *)((const X *)p.A + (t.begin + m) * p.a_stride) + (int64_t)i * 16; };
        const auto left = [&](int32_t i) { return ((int64_t)p.K - (int64_t)i * kPer) * (int64_t)sizeof(X); };
        const auto get = [&](int m, int32_t i) { return cut16(raw16(from(m, i), left(i)), left(i)); };
        // no branch around the loads: past a row's end its last 16 bytes come, of which nothing stays
#pragma unroll
        for (int m = 0; m < kFusedRows; ++m) {
            if (m >= rows) break;
#pragma unroll
            for (int i = 0; i < kKeep; ++i) keep[m][i] = raw16(from(m, threadIdx.x + i * kFewThreads), left(threadIdx.x + i * kFewThreads));
        }
#pragma unroll
        for (int m = 0; m < kFusedRows; ++m) {
            if (m >= rows) break;
            uint32_t seen = 0;
#pragma unroll
            for (int i = 0; i < kKeep; ++i) {
                keep[m][i] = cut16(keep[m][i], left(threadIdx.x + i * kFewThreads));
                seen = row_look<X>(keep[m][i], seen);
            }
            for (int32_t i = threadIdx.x + kKeep * kFewThreads; i < loads; i += kFewThreads) seen = row_look<X>(get(m, i), seen);
            const float top = row_top_of<kWave>(row_top<X>(seen));
            if (lane == 0) tops[m][wave] = top;
        }
        __syncthreads();
#pragma unroll
        for (int m = 0; m < kFusedRows; ++m) {
            if (m >= rows) break;
            const float top = row_top_of<kFewWaves>(tops[m][lane % kFewWaves]);
            const float scale = row_scale(top);
            int8_t *const to = (int8_t *)cut + m * cut_row;
            auto put = [&](v4i v, int32_t i) { row_codes<X>(v, scale, to + (int64_t)i * kPer); };
#pragma unroll
            for (int i = 0; i < kKeep; ++i)
                if ((int)threadIdx.x + i * kFewThreads < loads) put(keep[m][i], threadIdx.x + i * kFewThreads);
            for (int32_t i = threadIdx.x + kKeep * kFewThreads; i < loads; i += kFewThreads) put(get(m, i), i);
            if (m == (int)(threadIdx.x % 256 / 16)) x_scale = scale;
        }
        __syncthreads();
        x = cut + (r < rows ? r : rows - 1) * cut_row + quarter;
    } else {
        x = (const char *)((const T *)p.A + (t.begin + (r < rows ? r : rows - 1)) * p.a_stride) + quarter;
    }

    Sum sum = {};
    for (int32_t s0 = wave; s0 < pieces; s0 += kAhead * kFewWaves) {
        v4i fa[kAhead][2], fb[kAhead][2];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int32_t s = s0 + i * kFewWaves;
            if (s >= pieces) break;
            const int64_t k = (int64_t)s * kStepBytes;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                fa[i][h] = held[i][h];
                // what lies behind the row's end in LDS meets zeros of the weights
                fb[i][h] = kFused ? *(const v4i *)(x + k + 16 * h) : piece16<T, kAligned>(x, k + 16 * h, bytes - quarter, short_row);
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (s0 + (i + kAhead) * kFewWaves < pieces) load(s0 + (i + kAhead) * kFewWaves, i);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (s0 + i * kFewWaves >= pieces) break;
#pragma unroll
            for (int h = 0; h < 2; ++h) sum = FewType<T>::mma(fa[i][h], fb[i][h], sum);
        }
    }
    part[wave][lane] = sum;
    __syncthreads();
    // a lane's four values: columns 4 (lane / 16) .. + 3 of row lane % 16
    if (threadIdx.x >= 256) return;
    const int m = threadIdx.x / 16, c = threadIdx.x % 16;
    if (m >= rows || n0 + c >= p.N) return;
    typename std::remove_reference<decltype(sum[0])>::type v = part[0][c / 4 * 16 + m][c % 4];
#pragma unroll
    for (int k = 1; k < kFewWaves; ++k) v += part[k][c / 4 * 16 + m][c % 4];
    const int64_t row = t.begin + m, of = (int64_t)t.group * p.N + n0 + c;
    float y = (float)v;
    if constexpr (std::is_same<T, int8_t>::value) {
        y = y * (kFused ? x_scale : p.a_scale[row]) * p.b_scale[of];
        if (p.bias) y += ((const float *)p.bias)[of];
    } else if (p.bias) y += (float)((const O *)p.bias)[of];
    if (p.relu && y < 0.f) y = 0.f;
    ((O *)p.out)[row * p.out_stride + n0 + c] = (O)y;
}

template <typename T, typename O, typename X>
int few_launch(const RowsProduct &p, void *stream)
{
    constexpr bool kFused = !std::is_same<X, T>::value;
    const int64_t b = sizeof(T);
    const bool aligned = (((uintptr_t)p.B | (uintptr_t)(p.K * b)) & 15) == 0 && (kFused || (((uintptr_t)p.A | (uintptr_t)(p.a_stride * b)) & 15) == 0);
    const int32_t col_tiles = few_tiles(p.N, kFewCols);
    const int64_t workgroups = few_workgroups(p, kFewCols);
    if (!fits_launch(workgroups, kFewThreads)) return kErrTooManyTiles;
    const size_t lds = kFused ? (size_t)p.n * ((p.K + 127) / 128 * 128) : 0;
    if (aligned) few_kernel<T, O, X, true><<<(uint32_t)workgroups, kFewThreads, lds, (hipStream_t)stream>>>(p, col_tiles);
    else few_kernel<T, O, X, false><<<(uint32_t)workgroups, kFewThreads, lds, (hipStream_t)stream>>>(p, col_tiles);
    return (int)hipGetLastError();
}

// Few rows against weights whose rows lie across the contraction ([groups, K, N]: the forward products): 64 columns to a workgroup, its
// eight wavefronts take 32 (fp32: 16) rows of the weights in turn.  A lane has four neighbouring columns of 8 (4) rows, so that 16
// lanes read 128 (256) bytes of a row, and puts the values of a column next to one another in registers; column 4 c + j goes through
// the j-th of four instructions.  Three of a wavefront's blocks of rows are on their way while one is multiplied.
constexpr int kAcrossCols = 64, kAcrossAhead = 3;

template <typename T>
struct AcrossBlock {
    static constexpr int kRows = sizeof(T) == 2 ? 32 : 16, kLoads = kRows / 4;
    typedef int W __attribute__((ext_vector_type(sizeof(T))));       // four columns: 2 or 4 words
    W w[kLoads];
    v4i x;

    // rows k0 + kLoads * (lane / 16) .. of the weights from `w0`, the lane's row of X from `x0`
    __device__ __forceinline__ void load(const char *w0, int64_t pitch, const char *x0, int32_t k0, int32_t K, bool short_row)
    {
        const int32_t k = k0 + kLoads * (int32_t)(threadIdx.x % kWave / 16);
        if (k0 + kRows <= K) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) __builtin_memcpy(&w[i], w0 + (int64_t)(k + i) * pitch, sizeof(W));
            __builtin_memcpy(&x, x0 + (int64_t)k * sizeof(T), 16);
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                w[i] = W{};
                if (k + i < K) __builtin_memcpy(&w[i], w0 + (int64_t)(k + i) * pitch, sizeof(W));
            }
            x = load16<T>(x0 + (int64_t)k * sizeof(T), (int64_t)(K - k) * (int64_t)sizeof(T), short_row);
        }
    }
    __device__ __forceinline__ void multiply(v4f (&sums)[4]) const
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (sizeof(T) == 2) {
                v4i a;
#pragma unroll
                for (int i = 0; i < 4; ++i) a[i] = __builtin_amdgcn_perm(w[2 * i + 1][j / 2], w[2 * i][j / 2], j % 2 ? 0x07060302 : 0x05040100);
                sums[j] = FewType<T>::mma(a, x, sums[j]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) sums[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__int_as_float(w[i][j]), __int_as_float(x[i]), sums[j], 0, 0, 0);
            }
        }
    }
};

template <typename T>
__global__ __launch_bounds__(kFewThreads) void few_across_kernel(const RowsProduct p, int32_t col_tiles)
{
    typedef AcrossBlock<T> Block;
    __shared__ v4f part[kFewWaves][4][kWave];
    const RowTile t = find_tile(p.offsets, p.groups, p.n, blockIdx.x / col_tiles, 4);
    if (t.group < 0) return;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, r = lane % 16;
    const int rows = (int)(t.end - t.begin);
    const auto column = [&](int c) {                         // the last lanes repeat columns rather than read past a row's end
        const int32_t col = (int32_t)(blockIdx.x % col_tiles) * kAcrossCols + 4 * c;
        return col < p.N - 4 ? col : p.N - 4;
    };
    const char *const w0 = (const char *)((const T *)p.B + (int64_t)t.group * p.K * p.N + column(r));
    const char *const x0 = (const char *)((const T *)p.A + (t.begin + (r < rows ? r : rows - 1)) * p.a_stride);
    const int64_t pitch = (int64_t)p.N * sizeof(T);
    const bool short_row = (int64_t)p.K * sizeof(T) < 16;
    const int32_t blocks = (p.K + Block::kRows - 1) / Block::kRows;
    Block held[kAcrossAhead];
    v4f sums[4] = {};
#pragma unroll
    for (int i = 0; i < kAcrossAhead; ++i)
        if (wave + i * kFewWaves < blocks) held[i].load(w0, pitch, x0, (wave + i * kFewWaves) * Block::kRows, p.K, short_row);
    for (int32_t b0 = wave; b0 < blocks; b0 += kAcrossAhead * kFewWaves) {
#pragma unroll
        for (int i = 0; i < kAcrossAhead; ++i) {
            const int32_t b = b0 + i * kFewWaves;
            if (b >= blocks) break;
            held[i].multiply(sums);
            if (b + kAcrossAhead * kFewWaves < blocks) held[i].load(w0, pitch, x0, (b + kAcrossAhead * kFewWaves) * Block::kRows, p.K, short_row);
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) part[wave][j][lane] = sums[j];
    __syncthreads();
    // lane l holds row l % 16 and, in its four values, c = 4 (l / 16) .. + 3
    if (threadIdx.x >= 256) return;
    const int m = threadIdx.x / 16, c = threadIdx.x % 16;
    if (m >= rows) return;
    const int32_t col = column(c);
    const int64_t row = t.begin + m, of = (int64_t)t.group * p.N + col;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float y = 0.f;
#pragma unroll
        for (int k = 0; k < kFewWaves; ++k) y += part[k][j][c / 4 * 16 + m][c % 4];
        if (p.bias) y += (float)((const T *)p.bias)[of + j];
        if (p.relu && y < 0.f) y = 0.f;
        ((T *)p.out)[row * p.out_stride + col + j] = (T)y;
    }
}

template <typename T>
int few_across_launch(const RowsProduct &p, void *stream)
{
    const int32_t col_tiles = few_tiles(p.N, kAcrossCols);
    const int64_t workgroups = few_workgroups(p, kAcrossCols);
    if (!fits_launch(workgroups, kFewThreads)) return kErrTooManyTiles;
    few_across_kernel<T><<<(uint32_t)workgroups, kFewThreads, 0, (hipStream_t)stream>>>(p, col_tiles);
    return (int)hipGetLastError();
}

}  // namespace

// Groups of at most 16 rows on average.  Forward products of up to 512 workgroups: above, the tiles' longer pieces of the weights' rows
// bring more than the wavefronts' shares (one row, 4096 x 4096: 12.1 us here, 19.3 in tiles; 15 groups of 2560 x 2176: 35 and 40; 32 of
// 2048 x 2048: 53 and 48.5).  Weights along the contraction: up to what a launch holds, 2^23 workgroups; tiles take fewer.
bool few_rows_serve(const RowsProduct &p)
{
    if (p.n > (int64_t)kFewRows * p.groups) return false;
    return p.b_n_major ? fits_launch(few_workgroups(p, kFewCols), kFewThreads) : p.N >= 4 && (int64_t)p.groups * few_tiles(p.N, kAcrossCols) <= 512;
}

int launch_few_rows(int32_t dtype, const RowsProduct &p, void *stream)
{
    if (!p.b_n_major)
        return dtype == GROOT_F32 ? few_across_launch<float>(p, stream) : dtype == GROOT_BF16 ? few_across_launch<bf16_t>(p, stream) : few_across_launch<f16_t>(p, stream);
    if (dtype == GROOT_F32) return few_launch<float, float, float>(p, stream);
    if (dtype == GROOT_BF16) return few_launch<bf16_t, bf16_t, bf16_t>(p, stream);
    return few_launch<f16_t, f16_t, f16_t>(p, stream);
}

int launch_few_int8(int32_t out_dtype, const RowsProduct &p, void *stream)
{
    if (out_dtype == GROOT_F32) return few_launch<int8_t, float, int8_t>(p, stream);
    if (out_dtype == GROOT_BF16) return few_launch<int8_t, bf16_t, int8_t>(p, stream);
    return few_launch<int8_t, f16_t, int8_t>(p, stream);
}

// Rows in floating point, all of them in every workgroup; of 16 bytes at least.
bool few_linear_serves(const RowsProduct &p)
{
    return p.n <= kFusedRows && p.K >= 8 && p.n * ((p.K + 127) / 128 * 128) <= kFusedBytes && fits_launch(few_workgroups(p, kFewCols), kFewThreads);
}

int launch_few_linear(int32_t dtype, const RowsProduct &p, void *stream)
{
    if (dtype == GROOT_F32) return few_launch<int8_t, float, float>(p, stream);
    if (dtype == GROOT_BF16) return few_launch<int8_t, bf16_t, bf16_t>(p, stream);
    return few_launch<int8_t, f16_t, f16_t>(p, stream);
}

}  // namespace groot

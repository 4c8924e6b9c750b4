// Root-mean-square norm of rows, with the residual's addition in front, an output in 8 bits behind, and its gradients.
//   h = x + residual, rounded to the type;  rstd = 1 / sqrt(mean h^2 + eps), in 64 bits and rounded once;  y = (h rstd) gain in fp32
//   scale = max |y| fl(1 / 127), codes = y / scale to the nearest
//   dx = rstd (a - u mean(a u)) + dh with u = h rstd, a = dy gain;  dgain = sum over the rows of dy u
// The sum of the squares is in 64 bits so that rstd, and with it every code, is the same whatever order the lanes add in.
// Bound by HBM: a row is read once and stays in registers as it is held.  8192 rows of 4096 in float16 with a residual, H and 8 bits out: 41 us
// (5.7 TB/s); 16384 rows in bfloat16, forward 90 us (6.0 TB/s), backward 89 (6.0: three rows in, one out) and 6 for the gain's gradient; 8.4 M
// rows of 64 in fp32 0.73 ms (5.9) and 1.21 (5.3).  Of the backward call's time its instructions take a quarter: more rows on their way at a
// time (1.29 ms) and the next row's loads in front (1.45) made it slower, as did loads that keep their lines (1.28).
// The lanes of a row, and the pieces in each, are the fewest that hold it: with twice the lanes that rows of 4096 need, forward took 112 us.
//
// A piece is 16 bytes of a row; the last one is moved back to end with the row, so that it is whole too: its first values are computed
// twice, alike, and counted once.  Rows of less than 16 bytes go value by value.
#include "groot_tile.h"

namespace groot {

namespace {

// Where a lane's piece lies in every row.
struct Piece {
    int32_t at;                              // its first value
    int32_t first;                           // values that the piece before has counted
    bool real;                               // there is such a piece
};

template <typename T>
__device__ __forceinline__ Piece piece(int32_t i, int32_t K)
{
    constexpr int kPer = 16 / sizeof(T);
    const int32_t begin = i * kPer;
    if (K < kPer) return Piece{0, 0, i == 0};
    if (begin >= K) return Piece{K - kPer, 0, false};        // the row's last one is loaded, and nothing stays of it
    const int32_t at = begin + kPer <= K ? begin : K - kPer;
    return Piece{at, begin - at, true};
}

typedef v4i piece_t __attribute__((aligned(2)));
// kShort: a row of less than 16 bytes; kOnce: rows that no cache is to keep
template <typename T, bool kShort, bool kOnce>
__device__ __forceinline__ v4i load_piece(const T *row, const Piece &p, int32_t K)
{
    if constexpr (kShort) return short16<T>((const char *)row, (int64_t)K * (int64_t)sizeof(T));
    else if constexpr (kOnce) return __builtin_nontemporal_load((const piece_t *)(row + p.at));
    else return *(const piece_t *)(row + p.at);
}
template <typename T, bool kShort>
__device__ __forceinline__ void store_piece(T *row, const Piece &p, int32_t K, v4i v)
{
    if constexpr (kShort) {
        T e[16 / sizeof(T)];
        __builtin_memcpy(e, &v, 16);
#pragma unroll
        for (int k = 0; k < (int)(16 / sizeof(T)); ++k)
            if (k < K) row[k] = e[k];
    } else {
        *(piece_t *)(row + p.at) = v;
    }
}
template <typename T>
__device__ __forceinline__ v4i rounded(const RowValues<T> &x)
{
    constexpr int kPer = 16 / sizeof(T);
    typedef T vt __attribute__((ext_vector_type(kPer)));
    vt e;
#pragma unroll
    for (int k = 0; k < kPer; ++k) e[k] = (T)x.x[k];         // the one rounding
    return __builtin_bit_cast(v4i, e);
}
// ones for where there is no gain
template <typename T>
__device__ __forceinline__ v4i ones()
{
    RowValues<T> x;
#pragma unroll
    for (float &v : x.x) v = 1.f;
    return rounded<T>(x);
}

// Sums and maxima over the kLanes lanes of a row; every lane has them.  `lds`: a word for each wavefront of the workgroup.
template <int kLanes>
__device__ __forceinline__ double row_sum(double x, double *lds)
{
    x = over_lanes<(kLanes < kWave ? kLanes : kWave)>(x, [](double a, double b) { return a + b; });
    if constexpr (kLanes > kWave) {
        __syncthreads();                                     // the row before has read its words
        if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = x;
        __syncthreads();
        x = 0;
#pragma unroll
        for (int w = 0; w < kLanes / kWave; ++w) x += lds[threadIdx.x / kLanes * (kLanes / kWave) + w];
    }
    return x;
}
template <int kLanes>
__device__ __forceinline__ uint32_t row_most(uint32_t x, double *lds)
{
    x = over_lanes<(kLanes < kWave ? kLanes : kWave)>(x, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
    if constexpr (kLanes > kWave) {
        uint32_t *const tops = (uint32_t *)lds;
        __syncthreads();
        if (threadIdx.x % kWave == 0) tops[threadIdx.x / kWave] = x;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kLanes / kWave; ++w) {
            const uint32_t top = tops[threadIdx.x / kLanes * (kLanes / kWave) + w];
            x = top > x ? top : x;
        }
    }
    return x;
}

constexpr int block_of(int lanes) { return lanes > kBlock ? lanes : kBlock; }

// four values cut to 8 bits; r: the scale's reciprocal, where the scale is of an ordinary size
__device__ __forceinline__ uint32_t four_codes(const float *y, float scale, float r)
{
    constexpr float kRound = 12582912.f;                     // 1.5 * 2^23: what is added to it is rounded to an integer
    uint32_t q[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) q[e] = __float_as_uint(quotient(y[e], scale, r) + kRound);
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(q[3], q[2], 0x0C0C0400u), __builtin_amdgcn_perm(q[1], q[0], 0x0C0C0400u), 0x05040100u);
}

template <typename T, int kLanes, int kKeep, bool kShort, bool kOnce>
__global__ __launch_bounds__(block_of(kLanes)) void norm_kernel(NormArgs a)
{
    constexpr int kPer = 16 / sizeof(T), kThreads = block_of(kLanes), kRows = kThreads / kLanes;
    __shared__ double words[kThreads / kWave];
    const int lane = threadIdx.x % kLanes;
    Piece p[kKeep];
    v4i gain[kKeep];
#pragma unroll
    for (int i = 0; i < kKeep; ++i) {
        p[i] = piece<T>(i * kLanes + lane, a.K);
        gain[i] = a.gain ? load_piece<T, kShort, false>((const T *)a.gain, p[i], a.K) : ones<T>();
    }
    for (int64_t first = (int64_t)blockIdx.x * kRows; first < a.n; first += (int64_t)gridDim.x * kRows) {
        const int64_t mine = first + threadIdx.x / kLanes, row = mine < a.n ? mine : a.n - 1;   // rows beyond the last go along and store nothing
        const bool real = mine < a.n;
        const T *const x = (const T *)a.X + row * a.x_stride;
        v4i h[kKeep];
#pragma unroll
        for (int i = 0; i < kKeep; ++i) h[i] = load_piece<T, kShort, kOnce>(x, p[i], a.K);
        if (a.residual) {
            const T *const r = (const T *)a.residual + row * a.residual_stride;
            v4i other[kKeep];
#pragma unroll
            for (int i = 0; i < kKeep; ++i) other[i] = load_piece<T, kShort, kOnce>(r, p[i], a.K);
#pragma unroll
            for (int i = 0; i < kKeep; ++i) {
                RowValues<T> u = row_values<T>(h[i]);
                const RowValues<T> v = row_values<T>(other[i]);
#pragma unroll
                for (int e = 0; e < kPer; ++e) u.x[e] += v.x[e];
                h[i] = rounded<T>(u);
            }
        }
        double sum = 0;
#pragma unroll
        for (int i = 0; i < kKeep; ++i) {
            if (!p[i].real) continue;
            const RowValues<T> u = row_values<T>(h[i]);
            if (p[i].first == 0) {
#pragma unroll
                for (int e = 0; e < kPer; ++e) sum = __builtin_fma((double)u.x[e], (double)u.x[e], sum);
            } else {                                         // the last piece of a row that is no whole number of them
                for (int e = kPer - 1; e >= 0; --e)
                    if (e >= p[i].first) sum = __builtin_fma((double)u.x[e], (double)u.x[e], sum);
            }
        }
        sum = row_sum<kLanes>(sum, words);
        const float rstd = (float)(1.0 / sqrt(sum / a.K + a.eps));
        RowValues<T> y[kKeep];
        uint32_t seen = 0;
#pragma unroll
        for (int i = 0; i < kKeep; ++i) {
            y[i] = row_values<T>(h[i]);
            const RowValues<T> g = row_values<T>(gain[i]);
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                y[i].x[e] = (y[i].x[e] * rstd) * g.x[e];
                const uint32_t m = __float_as_uint(y[i].x[e]) & 0x7FFFFFFFu;
                if (!kShort || e < a.K) seen = m > seen ? m : seen;
            }
            if (!real || !p[i].real) continue;
            if (a.H) store_piece<T, kShort>((T *)a.H + row * a.h_stride, p[i], a.K, h[i]);
            if (a.Y) store_piece<T, kShort>((T *)a.Y + row * a.y_stride, p[i], a.K, rounded<T>(y[i]));
        }
        if (real && a.rstd && lane == 0) a.rstd[row] = rstd;
        if (!a.Q) continue;
        const float scale = row_scale(__uint_as_float(row_most<kLanes>(seen, words)));
        if (!real) continue;
        if (lane == 0) a.q_scale[row] = scale;
        const bool usual = scale > 0x1p-96f;                 // the same for a row
        const float r = usual ? 1.f / scale : 0.f;
#pragma unroll
        for (int i = 0; i < kKeep; ++i) {
            if (!p[i].real) continue;
            uint32_t codes[kPer / 4];
            if (usual) {
#pragma unroll
                for (int e = 0; e < kPer; e += 4) codes[e / 4] = four_codes(y[i].x + e, scale, r);
            } else {
#pragma unroll
                for (int e = 0; e < kPer; e += 4) {
                    const v4f four = {y[i].x[e], y[i].x[e + 1], y[i].x[e + 2], y[i].x[e + 3]};
                    row_codes<float>(__builtin_bit_cast(v4i, four), scale, (int8_t *)&codes[e / 4]);
                }
            }
            int8_t *const to = a.Q + row * a.q_stride + p[i].at;
            if constexpr (kShort) {
#pragma unroll
                for (int e = 0; e < kPer; ++e)
                    if (e < a.K) to[e] = (int8_t)(codes[e / 4] >> (8 * (e % 4)));
            } else {
                __builtin_memcpy(to, codes, kPer);
            }
        }
    }
}

// The rows of a workgroup add up their part of the gain's gradient, each lane its own columns; the parts meet in norm_gain_kernel.
template <typename T, int kLanes, int kKeep, bool kShort, bool kOnce, bool kPast>
__global__ __launch_bounds__(block_of(kLanes)) void norm_backward_kernel(NormBackwardArgs a)
{
    constexpr int kPer = 16 / sizeof(T), kThreads = block_of(kLanes), kRows = kThreads / kLanes;
    __shared__ double words[kThreads / kWave];
    const int lane = threadIdx.x % kLanes;
    Piece p[kKeep];
    v4i gain[kKeep];
#pragma unroll
    for (int i = 0; i < kKeep; ++i) {
        p[i] = piece<T>(i * kLanes + lane, a.K);
        gain[i] = a.gain ? load_piece<T, kShort, false>((const T *)a.gain, p[i], a.K) : ones<T>();
    }
    float parts[kKeep][kPer] = {};
    for (int64_t first = (int64_t)blockIdx.x * kRows; first < a.n; first += (int64_t)gridDim.x * kRows) {
        const int64_t mine = first + threadIdx.x / kLanes, row = mine < a.n ? mine : a.n - 1;
        const bool real = mine < a.n;
        const float rstd = a.rstd[row];
        v4i h[kKeep], dy[kKeep], dh[kKeep];
#pragma unroll
        for (int i = 0; i < kKeep; ++i) {
            h[i] = load_piece<T, kShort, kOnce>((const T *)a.H + row * a.h_stride, p[i], a.K);
            dy[i] = load_piece<T, kShort, kOnce>((const T *)a.dY + row * a.dy_stride, p[i], a.K);
        }
        if (a.dH) {
#pragma unroll
            for (int i = 0; i < kKeep; ++i) dh[i] = load_piece<T, kShort, kOnce>((const T *)a.dH + row * a.dh_stride, p[i], a.K);
        }
        double sum = 0;
#pragma unroll
        for (int i = 0; i < kKeep; ++i) {
            if (!real || !p[i].real) continue;
            const RowValues<T> x = row_values<T>(h[i]), d = row_values<T>(dy[i]), g = row_values<T>(gain[i]);
            float here = 0.f;
            if (p[i].first == 0) {
#pragma unroll
                for (int e = 0; e < kPer; ++e) {
                    const float t = d.x[e] * (x.x[e] * rstd);
                    here += t * g.x[e];
                    parts[i][e] += t;
                }
            } else {
#pragma unroll
                for (int e = 0; e < kPer; ++e) {
                    const float t = d.x[e] * (x.x[e] * rstd);
                    here += e >= p[i].first ? t * g.x[e] : 0.f;
                    parts[i][e] += t;                        // of the values that come twice, one is written
                }
            }
            sum += here;
        }
        sum = row_sum<kLanes>(sum, words);
        const float c = (float)(sum / a.K);
        if (!real) continue;
#pragma unroll
        for (int i = 0; i < kKeep; ++i) {
            if (!p[i].real) continue;
            RowValues<T> u = row_values<T>(dy[i]);
            const RowValues<T> x = row_values<T>(h[i]), g = row_values<T>(gain[i]);
#pragma unroll
            for (int e = 0; e < kPer; ++e) u.x[e] = rstd * (u.x[e] * g.x[e] - (x.x[e] * rstd) * c);
            if (a.dH) {
                const RowValues<T> v = row_values<T>(dh[i]);
#pragma unroll
                for (int e = 0; e < kPer; ++e) u.x[e] += v.x[e];
            }
            if constexpr (!kShort && kPast) __builtin_nontemporal_store(rounded<T>(u), (piece_t *)((T *)a.dX + row * a.dx_stride + p[i].at));
            else store_piece<T, kShort>((T *)a.dX + row * a.dx_stride, p[i], a.K, rounded<T>(u));
        }
    }
    if (!a.dgain) return;
    // the workgroup's rows meet in LDS, in their order; lane by lane, so that a value is counted where its piece is
    float *const to = a.partial + (int64_t)blockIdx.x * a.K;
    if constexpr (kRows > 1) {
        extern __shared__ float sums[];                      // [kRows, kLanes kKeep kPer]
        constexpr int kRow = kLanes * kKeep * kPer;
#pragma unroll
        for (int i = 0; i < kKeep; ++i)
#pragma unroll
            for (int e = 0; e < kPer; ++e) sums[threadIdx.x / kLanes * kRow + (i * kPer + e) * kLanes + lane] = parts[i][e];
        __syncthreads();
        for (int at = threadIdx.x; at < kRow; at += kThreads) {
            float sum = 0.f;
#pragma unroll
            for (int r = 0; r < kRows; ++r) sum += sums[r * kRow + at];
            const int from = at % kLanes, e = at / kLanes % kPer;
            const Piece place = piece<T>(at / kLanes / kPer * kLanes + from, a.K);
            if (place.real && e >= place.first && place.at + e < a.K) to[place.at + e] = sum;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kKeep; ++i) {
#pragma unroll
            for (int e = 0; e < kPer; ++e)
                if (p[i].real && e >= p[i].first && p[i].at + e < a.K) to[p[i].at + e] = parts[i][e];
        }
    }
}

// Rows of more bytes are read past the caches, and a gradient of more is written past them.  Rows of 4096 in bfloat16, past and kept, us, with the product
// in front that makes the rows (or their gradient) and, the second pair, the one behind that takes the norm's:
//   forward loads    32 MB 46 and 44, 65 and 63; 48 MB 67 and 63, 95 and 91; 64 MB 80 and 79, 106 and 115; 96 MB 116 and 121, 160 and 173; 128 MB 151 and 167, 211
//                    and 222; 192 MB 240 and 255, 323 and 328; 256 MB 316 and 335, 421 and 418
//   backward loads   32 MB 56 and 53; 48 MB 78 and 75; 64 MB 91 and 92; 96 MB 128 and 130; 128 MB 165 and 182; 192 MB 233 and 268; 256 MB 305 and 305
//   gradient         by itself and with the product that takes it: 64 MB 61 and 57, 93 and 84; 128 MB 102 and 99, 150 and 139; 256 MB 184 and 181, 275 and 285
// (by itself, all in the caches: forward 64 MB 44 and 41, 128 MB 81 and 94; backward 58 and 55, 97 and 108; with four sets of buffers in turn past is never the
// slower: 32 MB 70 and 76, 48 MB 112 and 115, 64 MB 132 and 133, backward 57 and 60, 82 and 83, 97 and 99, the gradient with two products 128 MB 224 and 227, 192 MB
// 368 and 358, 256 MB 413 and 422).
constexpr int64_t kLoadsPast = 56 << 20, kGradientsPast = 192 << 20;

constexpr int kGainCols = 16, kGainRows = 64;

template <typename O>
__global__ __launch_bounds__(1024) void norm_gain_kernel(const float *__restrict__ partial, int64_t groups, int32_t K, O *__restrict__ dgain)
{
    __shared__ double sums[kGainRows][kGainCols];
    const int col = threadIdx.x % kGainCols, part = threadIdx.x / kGainCols;
    const int32_t k = blockIdx.x * kGainCols + col;
    double sum = 0;
    if (k < K)
    {
#pragma unroll 8
        for (int64_t g = part; g < groups; g += kGainRows) sum += (double)partial[g * K + k];
    }
    sums[part][col] = sum;
    __syncthreads();
    if (part || k >= K) return;
    for (int p = 1; p < kGainRows; ++p) sum += sums[p][col];
    dgain[k] = (O)sum;
}

// Lanes of a row, and its pieces in each, by the pieces that it has: the fewest lanes, in wavefronts, that leave few idle (15910 rows of 1528 in fp32,
// 382 pieces: 128 lanes with 3 each 37 and 53 us, 256 with 2 39 and 60; 5031 rows of 1138 in bfloat16, 143 pieces: 64 with 3 12.0 and 17.4, 64 with 4 14.2
// and 18.3).
struct NormShape {
    int lanes, keep;
    bool is_short;
};
NormShape norm_shape(int32_t K, int bytes)
{
    const int64_t pieces = ((int64_t)K * bytes + 15) / 16;
    if (K * (int64_t)bytes < 16) return {16, 1, true};
    if (pieces <= 16) return {16, 1, false};
    if (pieces <= 32) return {16, 2, false};
    if (pieces <= 64) return {64, 1, false};
    if (pieces <= 128) return {64, 2, false};
    if (pieces <= 192) return {64, 3, false};
    if (pieces <= 256) return {64, 4, false};
    if (pieces <= 384) return {128, 3, false};
    if (pieces <= 512) return {256, 2, false};
    if (pieces <= 768) return {256, 3, false};
    if (pieces <= 1024) return {256, 4, false};
    if (pieces <= 2048) return {512, 4, false};
    if (pieces <= 4096) return {1024, 4, false};
    if (pieces <= 8192) return {1024, 8, false};
    return {1024, 16, false};
}

constexpr int rows_of(int lanes) { return block_of(lanes) / lanes; }
int64_t norm_blocks(int64_t n, const NormShape &s, int64_t most)
{
    const int64_t b = (n + rows_of(s.lanes) - 1) / rows_of(s.lanes);
    return b < most ? b : most;
}
// Workgroups of the backward call: whole multiples of the 256 CUs, the least that leave no more than four turns of rows to each while there are fewer than
// `most` (so 256 of them up to 1024 turns, and just above a multiple each has little more than two), as each writes a row of partial sums.  With the sums, us:
// 512, 1024, 1100, 2048 and 3000 rows of 4096 in bfloat16, 256 of them: 13.7, 16.4, 17.8, 22.7 and 28.9, 512: 18.4, 18.5, 18.7, 22.3 and 26.6, 768: 18.4, 22.3,
// 22.3, 25.8 and 30.0; 5031 rows of 1138, 1258 turns, 256 and 512: 18.7 and 16.1; 17600 rows of 64 in fp32, 1100 turns: 8.0 and 6.7; 16384 rows of 4096, 256, 512,
// 768, 1024, 2048: 129, 99, 100, 100, 110; 8.4 M rows of 64, 512, 1024, 2048, 8192: 1541, 1202, 1214, 1388.  Rounded down in place of up: 1100 rows of 4096 18.5 and
// 17.6, 3000 rows 29.7 and 26.4, but 5031 rows of 1138 15.7 and 18.1, 17600 rows of 64 6.8 and 8.1.
int64_t backward_blocks(int64_t n, const NormShape &s)
{
    const int64_t turns = norm_blocks(n, s, INT64_MAX), most = s.lanes <= kWave ? 1024 : s.lanes <= 256 ? 768 : s.lanes == 512 ? 512 : 256;
    const int64_t blocks = (turns / 4 + 255) / 256 * 256;
    return turns < 256 ? turns : blocks < 256 ? 256 : blocks < most ? blocks : most;
}

#define GROOT_NORM_SHAPES(use)                                                                                                           \
    if (s.is_short) use(16, 1, true)                                                                                                     \
    else if (s.lanes == 16 && s.keep == 1) use(16, 1, false)                                                                             \
    else if (s.lanes == 16) use(16, 2, false)                                                                                            \
    else if (s.lanes == 64 && s.keep == 1) use(64, 1, false)                                                                             \
    else if (s.lanes == 64 && s.keep == 2) use(64, 2, false)                                                                             \
    else if (s.lanes == 64 && s.keep == 3) use(64, 3, false)                                                                             \
    else if (s.lanes == 64) use(64, 4, false)                                                                                            \
    else if (s.lanes == 128) use(128, 3, false)                                                                                          \
    else if (s.lanes == 256 && s.keep == 2) use(256, 2, false)                                                                           \
    else if (s.lanes == 256 && s.keep == 3) use(256, 3, false)                                                                           \
    else if (s.lanes == 256) use(256, 4, false)                                                                                          \
    else if (s.lanes == 512) use(512, 4, false)                                                                                          \
    else if (s.keep == 4) use(1024, 4, false)                                                                                            \
    else if (s.keep == 8) use(1024, 8, false)                                                                                            \
    else if constexpr (sizeof(T) == 4) use(1024, 16, false)

template <typename T, bool kOnce>
int norm_launch(const NormArgs &a, hipStream_t stream)
{
    const NormShape s = norm_shape(a.K, sizeof(T));
    const uint32_t blocks = (uint32_t)norm_blocks(a.n, s, 1 << 20);
#define GROOT_NORM(lanes, keep, is_short) { norm_kernel<T, lanes, keep, is_short, kOnce><<<blocks, block_of(lanes), 0, stream>>>(a); }
    GROOT_NORM_SHAPES(GROOT_NORM)
#undef GROOT_NORM
    return (int)hipGetLastError();
}

template <typename T, bool kOnce, bool kPast>
int norm_backward_launch(const NormBackwardArgs &a, hipStream_t stream)
{
    const NormShape s = norm_shape(a.K, sizeof(T));
    const uint32_t blocks = (uint32_t)backward_blocks(a.n, s);
#define GROOT_NORM(lanes, keep, is_short)                                                                                                \
    {                                                                                                                                    \
        norm_backward_kernel<T, lanes, keep, is_short, kOnce, kPast>                                                                                   \
            <<<blocks, block_of(lanes), rows_of(lanes) > 1 ? block_of(lanes) * keep * 16 / sizeof(T) * sizeof(float) : 0, stream>>>(a);  \
    }
    if (blocks) { GROOT_NORM_SHAPES(GROOT_NORM) }
#undef GROOT_NORM
    if (a.dgain) {
        const uint32_t cols = (a.K + kGainCols - 1) / kGainCols;
        const int64_t groups = blocks;
        if (a.grad_f32) norm_gain_kernel<<<cols, 1024, 0, stream>>>(a.partial, groups, a.K, (float *)a.dgain);
        else norm_gain_kernel<<<cols, 1024, 0, stream>>>(a.partial, groups, a.K, (T *)a.dgain);
    }
    return (int)hipGetLastError();
}

}  // namespace

size_t norm_backward_workspace(int32_t dtype, int64_t n, int32_t K)
{
    const NormShape s = norm_shape(K, dtype == GROOT_F32 ? 4 : 2);
    return (size_t)backward_blocks(n, s) * K * sizeof(float);
}

int launch_norm(int32_t dtype, const NormArgs &a, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    const bool once = a.n * a.K * (dtype == GROOT_F32 ? 4 : 2) > kLoadsPast;
    if (dtype == GROOT_F32) return once ? norm_launch<float, true>(a, s) : norm_launch<float, false>(a, s);
    if (dtype == GROOT_BF16) return once ? norm_launch<bf16_t, true>(a, s) : norm_launch<bf16_t, false>(a, s);
    return once ? norm_launch<f16_t, true>(a, s) : norm_launch<f16_t, false>(a, s);
}

template <typename T>
static int norm_backward_for(const NormBackwardArgs &a, hipStream_t stream)
{
    const int64_t bytes = a.n * a.K * (int64_t)sizeof(T);
    return bytes > kGradientsPast ? norm_backward_launch<T, true, true>(a, stream)
           : bytes > kLoadsPast   ? norm_backward_launch<T, true, false>(a, stream)
                                  : norm_backward_launch<T, false, false>(a, stream);
}
int launch_norm_backward(int32_t dtype, const NormBackwardArgs &a, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    if (dtype == GROOT_F32) return norm_backward_for<float>(a, s);
    if (dtype == GROOT_BF16) return norm_backward_for<bf16_t>(a, s);
    return norm_backward_for<f16_t>(a, s);
}

}  // namespace groot

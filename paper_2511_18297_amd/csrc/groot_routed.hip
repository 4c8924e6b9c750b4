// Rows on their way to the experts' places and back:
//   R[places[i,s]] = X[i];   out[i] = addend[i] + sum_s w[i,s] R[places[i,s]];   dR[places[i,s]] = w[i,s] dout[i], dw[i,s] = dout[i] . R[places[i,s]]
// Every kernel goes by the rows i, which know their places: no list of the other direction, no atomics; a slot's row is written by one group
// of lanes.  Bound by HBM: the n k rows at the places are read or written once, the n rows once.  bfloat16: the sum of 2 x 8192 rows of 4096
// with an addend 50 us (5.4 TB/s, the sums stay in the caches), of 2 x 12288 66 (6.1, past them); 7168 rows of 2048 to four places each 28 us (5.3
// TB/s), their sum's gradients 43 (6.2), their sum 41 (4.5) and the gradient of the rows 44 to 48 (3.4: one load of four answers on its way in a lane,
// and the places' before it).  A workgroup takes a whole row at once where it can: with a wavefront to a row, or parts of rows, a sum took 50 to 57
// us that takes 45 so.  Loads of four slots at a time go on their way together, those of a slot without a place to 16 bytes of zeros.
// Large outputs go past the caches (kRowsPast, kSumPast).
//
// A piece is 16 bytes of a row.  A row's last piece is moved back to end with the row, so that it is whole too: its first values are
// copied or computed twice, alike.  Rows of less than 16 bytes go value by value.
#include "groot_tile.h"

namespace groot {

namespace {

// where piece `i` of a row of `bytes` begins
__device__ __forceinline__ int64_t piece_at(int64_t i, int64_t bytes) { return i * 16 + 16 <= bytes || bytes < 16 ? i * 16 : bytes - 16; }

typedef v4i piece_t __attribute__((aligned(1)));
// kOnce: past the caches
template <bool kOnce>
__device__ __forceinline__ v4i get(const char *p)
{
    if constexpr (kOnce) return __builtin_nontemporal_load((const piece_t *)p);
    else return *(const piece_t *)p;
}
template <bool kOnce>
__device__ __forceinline__ void put(char *p, v4i v)
{
    if constexpr (kOnce) __builtin_nontemporal_store(v, (piece_t *)p);
    else *(piece_t *)p = v;
}

// A place of the row, the same in all of its lanes: -1 for none.  Rows of a whole wavefront read it as a scalar.
template <int kLanes>
__device__ __forceinline__ int64_t row_of(int64_t row)
{
    return kLanes >= kWave ? uniform(row) : row;
}
__device__ __forceinline__ int64_t place_at(const RoutedArgs &a, int64_t row, int32_t slot)
{
    const int32_t p = a.places[row * a.k + slot];
    return p >= 0 && p < a.n_places ? p : -1;
}

// A workgroup's rows: kLanes lanes each, blockDim.x / kLanes of them at a time; blockIdx.y is the row's part of a.part pieces.
// kPieces of them in a lane at a time; a lane's beyond the last go along with another one, which is stored more than once, alike.
template <int kLanes, int kPieces, bool kOnce>
__global__ __launch_bounds__(kBlock) void routed_rows_kernel(RoutedArgs a, int64_t bytes, int64_t x_bytes, int64_t r_bytes)
{
    const int lane = threadIdx.x % kLanes, rows = blockDim.x / kLanes;
    const int64_t pieces = (bytes + 15) / 16, begin = (int64_t)blockIdx.y * a.part, end = begin + a.part < pieces ? begin + a.part : pieces;
    for (int64_t r = (int64_t)blockIdx.x * rows + threadIdx.x / kLanes; r < a.n; r += (int64_t)gridDim.x * rows) {
        const int64_t row = row_of<kLanes>(r);
        const char *const x = (const char *)a.X + row * x_bytes;
        if (bytes < 16) {
            if (lane == 0)
                for (int32_t s = 0; s < a.k; ++s) {
                    const int64_t p = place_at(a, row, s);
                    for (int b = 0; b < (int)bytes && p >= 0; ++b) ((char *)a.out + p * r_bytes)[b] = x[b];
                }
        } else {
            for (int64_t i = begin + lane; i < end; i += kLanes * kPieces) {
                int64_t at[kPieces];
                v4i v[kPieces];
#pragma unroll
                for (int j = 0; j < kPieces; ++j) {
                    at[j] = piece_at(i + j * kLanes < end ? i + j * kLanes : i, bytes);
                    v[j] = get<true>(x + at[j]);
                }
                for (int32_t s = 0; s < a.k; ++s) {
                    const int64_t p = place_at(a, row, s);
                    if (p < 0) continue;
                    char *const to = (char *)a.out + p * r_bytes;
#pragma unroll
                    for (int j = 0; j < kPieces; ++j) put<kOnce>(to + at[j], v[j]);
                }
            }
        }
        if (a.scale_in && blockIdx.y == 0)
            for (int32_t s = lane; s < a.k; s += kLanes) {
                const int64_t p = place_at(a, row, s);
                if (p >= 0) a.scale_out[p] = a.scale_in[row];
            }
    }
}

template <typename T, bool kShort, bool kOnce>
__device__ __forceinline__ v4i piece_of(const char *row, int64_t at, int32_t K)
{
    if constexpr (kShort) return short16<T>(row, K * (int64_t)sizeof(T));
    else return get<kOnce>(row + at);
}
template <typename T, bool kShort, bool kOnce>
__device__ __forceinline__ void store_piece(char *row, int64_t at, int32_t K, const float (&x)[16 / sizeof(T)])
{
    constexpr int kPer = 16 / sizeof(T);
    typedef T vt __attribute__((ext_vector_type(kPer)));
    vt e;
#pragma unroll
    for (int k = 0; k < kPer; ++k) e[k] = (T)x[k];           // the one rounding
    if constexpr (kShort) {
#pragma unroll
        for (int k = 0; k < kPer; ++k)
            if (k < K) ((T *)row)[k] = e[k];
    } else {
        put<kOnce>(row + at, __builtin_bit_cast(v4i, e));
    }
}
// the pieces of the rows at kBatch places from `slot` on; a slot without a place has a row of zeros, so that no load waits for a branch
template <typename T, int kBatch, int kPieces, bool kShort>
__device__ __forceinline__ void slot_pieces(const RoutedArgs &a, int64_t row, int32_t slot, int32_t slots, const int64_t (&at)[kPieces], int64_t (&p)[kBatch],
                                            v4i (&v)[kBatch][kPieces])
{
#pragma unroll
    for (int s = 0; s < kBatch; ++s) p[s] = slot + s < slots ? place_at(a, row, slot + s) : -1;
#pragma unroll
    for (int s = 0; s < kBatch; ++s)
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const char *const from = (const char *)((const T *)a.R + (p[s] < 0 ? 0 : p[s]) * a.r_stride);
            if constexpr (kShort) v[s][j] = p[s] < 0 ? v4i{0, 0, 0, 0} : piece_of<T, true, false>(from, at[j], a.K);
            else v[s][j] = piece_of<T, false, false>(p[s] < 0 ? (const char *)&g_zeros : from, p[s] < 0 ? 0 : at[j], a.K);
        }
}

template <typename T, int kLanes, int kPieces, bool kShort, bool kOnce>
__global__ __launch_bounds__(kBlock) void routed_sum_kernel(RoutedArgs a)
{
    constexpr int kPer = 16 / sizeof(T), kBatch = 4;
    const int lane = threadIdx.x % kLanes, rows = blockDim.x / kLanes;
    const int64_t bytes = (int64_t)a.K * sizeof(T), pieces = (bytes + 15) / 16;
    const int64_t begin = (int64_t)blockIdx.y * a.part, end = begin + a.part < pieces ? begin + a.part : pieces;
    for (int64_t r = (int64_t)blockIdx.x * rows + threadIdx.x / kLanes; r < a.n; r += (int64_t)gridDim.x * rows) {
        const int64_t row = row_of<kLanes>(r);
        const char *const addend = a.addend ? (const char *)((const T *)a.addend + row * a.addend_stride) : nullptr;
        for (int64_t i = begin + lane; i < end; i += kLanes * kPieces) {
            int64_t at[kPieces];
            float sum[kPieces][kPer];
#pragma unroll
            for (int j = 0; j < kPieces; ++j) {
                at[j] = piece_at(i + j * kLanes < end ? i + j * kLanes : i, bytes);
                const RowValues<T> v = a.addend ? row_values<T>(piece_of<T, kShort, true>(addend, at[j], a.K)) : RowValues<T>{};
#pragma unroll
                for (int e = 0; e < kPer; ++e) sum[j][e] = v.x[e];
            }
            for (int32_t slot = 0; slot < a.k; slot += kBatch) {
                int64_t p[kBatch];
                v4i v[kBatch][kPieces];
                slot_pieces<T, kBatch, kPieces, kShort>(a, row, slot, a.k, at, p, v);
#pragma unroll
                for (int s = 0; s < kBatch; ++s) {
                    if (slot + s >= a.k) break;
                    const float w = a.weights ? a.weights[row * a.k + slot + s] : 1.f;    // a NaN shows without a place too
#pragma unroll
                    for (int j = 0; j < kPieces; ++j) {
                        const RowValues<T> x = row_values<T>(v[s][j]);
#pragma unroll
                        for (int e = 0; e < kPer; ++e) sum[j][e] += w * x.x[e];
                    }
                }
            }
            char *const to = (char *)((T *)a.out + row * a.out_stride);
#pragma unroll
            for (int j = 0; j < kPieces; ++j) store_piece<T, kShort, kOnce>(to, at[j], a.K, sum[j]);
        }
    }
}

// kPieces > 0: a row's gradient stays in registers over its slots, kPieces pieces in each of kLanes lanes; 0: rows of any width, whose
// gradient is read again for every slot
template <typename T, int kLanes, int kPieces, bool kShort>
__global__ __launch_bounds__(kBlock) void routed_sum_backward_kernel(RoutedArgs a)
{
    constexpr int kPer = 16 / sizeof(T), kBatch = 2, kHeld = kPieces ? kPieces : 1, kParts = kLanes > kWave ? kLanes / kWave : 1;
    __shared__ float dots[kLanes > kWave ? 32 * kParts : 1];     // top_k is 32 at the most
    const int lane = threadIdx.x % kLanes, rows = blockDim.x / kLanes;
    const int64_t bytes = (int64_t)a.K * sizeof(T);
    const int32_t pieces = (int32_t)((bytes + 15) / 16);
    const int32_t first_slot = blockIdx.y * a.part, slots = first_slot + a.part < a.k ? first_slot + a.part : a.k;   // of this workgroup
    for (int64_t r = (int64_t)blockIdx.x * rows + threadIdx.x / kLanes; r < a.n; r += (int64_t)gridDim.x * rows) {
        const int64_t row = row_of<kLanes>(r);
        const char *const d_row = (const char *)((const T *)a.X + row * a.x_stride);
        v4i d[kHeld];
        int64_t at[kHeld];
        int counted[kHeld];                                  // values that the piece before has counted
        auto locate = [&](int32_t i, int j) {
            at[j] = piece_at(i < pieces ? i : pieces - 1, bytes);
            counted[j] = i >= pieces ? kPer : bytes < 16 ? 0 : (int)((i * (int64_t)16 - at[j]) / (int64_t)sizeof(T));
            d[j] = piece_of<T, kShort, true>(d_row, at[j], a.K);
        };
        if (kPieces) {
#pragma unroll
            for (int j = 0; j < kHeld; ++j) locate(lane + j * kLanes, j);
        }
        for (int32_t slot = first_slot; slot < slots; slot += kBatch) {
            float dot[kBatch] = {}, w[kBatch];
#pragma unroll
            for (int s = 0; s < kBatch; ++s) w[s] = a.weights && slot + s < slots ? a.weights[row * a.k + slot + s] : 1.f;
            for (int32_t i = 0; i < (kPieces ? 1 : pieces); i += kLanes) {
                if (!kPieces) locate(i + lane, 0);
                int64_t p[kBatch];
                v4i v[kBatch][kHeld];
                if (a.dweights) slot_pieces<T, kBatch, kHeld, kShort>(a, row, slot, slots, at, p, v);
#pragma unroll
                for (int s = 0; s < kBatch; ++s) {
                    if (!a.dweights) p[s] = slot + s < slots ? place_at(a, row, slot + s) : -1;
                    if (p[s] < 0) continue;
#pragma unroll
                    for (int j = 0; j < kHeld; ++j) {
                        const RowValues<T> g = row_values<T>(d[j]);
                        if (a.dweights) {
                            const RowValues<T> x = row_values<T>(v[s][j]);
                            float sum = 0.f;
                            if (counted[j] == 0) {
#pragma unroll
                                for (int e = 0; e < kPer; ++e) sum += g.x[e] * x.x[e];
                            } else {
#pragma unroll
                                for (int e = 0; e < kPer; ++e) sum += e >= counted[j] ? g.x[e] * x.x[e] : 0.f;
                            }
                            dot[s] += sum;
                        }
                        if (a.out) {
                            float x[kPer];
#pragma unroll
                            for (int e = 0; e < kPer; ++e) x[e] = w[s] * g.x[e];
                            store_piece<T, kShort, false>((char *)((T *)a.out + p[s] * a.out_stride), at[j], a.K, x);
                        }
                    }
                }
            }
            if (a.dweights) {
#pragma unroll
                for (int s = 0; s < kBatch; ++s) {
                    dot[s] = over_lanes<(kLanes < kWave ? kLanes : kWave)>(dot[s], [](float x, float y) { return x + y; });
                    if constexpr (kLanes > kWave) {
                        if (threadIdx.x % kWave == 0 && slot + s < slots) dots[(slot + s) * kParts + threadIdx.x / kWave] = dot[s];
                    } else {
                        if (lane == 0 && slot + s < slots) a.dweights[row * a.k + slot + s] = dot[s];
                    }
                }
            }
        }
        if constexpr (kLanes > kWave) {
            if (a.dweights) {                                // the wavefronts' parts of every slot
                __syncthreads();
                const int32_t slot = first_slot + threadIdx.x;
                if (slot < slots) {
                    float sum = 0.f;
#pragma unroll
                    for (int w = 0; w < kParts; ++w) sum += dots[slot * kParts + w];
                    a.dweights[row * a.k + slot] = sum;
                }
                __syncthreads();                             // before the next row's
            }
        }
    }
}

// Threads of a workgroup and the grid: where rows alone are too few wavefronts for the GPU, each is cut into parts.
struct RoutedShape {
    int threads;
    dim3 grid;
};
constexpr int64_t kEnoughWaves = 4096;       // four to a SIMD
RoutedShape routed_shape(RoutedArgs *a, int64_t pieces, int lanes)
{
    const int64_t waves = lanes >= kWave ? a->n * (lanes / kWave) : (a->n + kWave / lanes - 1) / (kWave / lanes);
    const int64_t most = (pieces + lanes - 1) / lanes;       // parts of one piece a lane
    int64_t parts = 1;
    while (parts * 2 <= most && waves * parts * 2 <= kEnoughWaves) parts *= 2;
    int64_t part = (pieces + parts - 1) / parts;
    part = (part + lanes - 1) / lanes * lanes;
    a->part = (int32_t)part;
    const int threads = lanes > kWave || waves * parts >= 4 * 256 ? kBlock : kWave;
    const int64_t blocks = (a->n + threads / lanes - 1) / (threads / lanes);
    return {threads, dim3((uint32_t)(blocks < (1 << 20) ? blocks : 1 << 20), (uint32_t)((pieces + part - 1) / part))};
}
// Copied rows and sums from some size on go past the caches.  By the call that makes them and those around it, past and kept (bfloat16, rows of 4096,
// us a set of buffers; first one set over and over, then four in turn):
//   rows, their product           64 MB 64 and 57, 128 MB 91 and 80, 192 MB 144 and 120, 256 MB 174 and 183, 384 MB 259 and 256
//   norm, rows, their product     four sets: 64 MB 77 and 85, 128 MB 111 and 123, 192 MB 168 and 181, 256 MB 203 and 231, 384 MB 305 and 333
//   sum, norm                     32 MB 37 and 36, 64 MB 64 and 63, 96 MB 104 and 106, 192 MB 218 and 224; four: 64 MB 79 and 73, 96 MB 110 and 111
//   sum, product                  32 MB 45 and 45, 64 MB 74 and 68, 96 MB 102 and 105, 128 MB 136 and 147, 256 MB 265 and 283
//   product, sum, norm, product   four sets: 48 MB 157 and 159, 64 MB 198 and 194, 96 MB 270 and 275, 128 MB 351 and 366, 192 MB 539 and 554
// (the sum by itself, four sets: 64 MB 48 and 52, 96 MB 69 and 76).  The sum's gradients are kept at every size: with the two products that read them,
// four sets, 64 MB 116 and 113, 128 MB 173 and 167, 256 MB 319 and 309, 512 MB 595 and 586; one set, 128 MB 161 and 166, 256 MB 319 and 317 (by
// themselves 128 MB 67 and 69).
constexpr int64_t kRowsPast = 224 << 20, kSumPast = 80 << 20;

template <typename T, bool kOnce>
int sum_launch(RoutedArgs a, hipStream_t stream)
{
    const int64_t pieces = ((int64_t)a.K * sizeof(T) + 15) / 16;
#define GROOT_SUM(lanes, per_lane, is_short)                                                                                             \
    {                                                                                                                                    \
        const RoutedShape s = routed_shape(&a, pieces, lanes);                                                                           \
        routed_sum_kernel<T, lanes, per_lane, is_short, kOnce><<<s.grid, s.threads, 0, stream>>>(a);                                     \
    }
    // a workgroup takes a whole row at once where it can
    if (a.K * sizeof(T) < 16) GROOT_SUM(16, 1, true)
    else if (pieces <= 16) GROOT_SUM(16, 1, false)
    else if (pieces <= 64) GROOT_SUM(64, 1, false)
    else if (pieces <= 128) GROOT_SUM(64, 2, false)
    else if (pieces <= 256) GROOT_SUM(256, 1, false)
    else GROOT_SUM(256, 2, false)
#undef GROOT_SUM
    return (int)hipGetLastError();
}
template <typename T>
int sum_backward_launch(RoutedArgs a, hipStream_t stream)
{
    const int64_t pieces = ((int64_t)a.K * sizeof(T) + 15) / 16;
#define GROOT_SUM(lanes, held, is_short)                                                                                                 \
    {                                                                                                                                    \
        RoutedShape s = routed_shape(&a, 1, lanes);                                                                                      \
        a.part = few_rows ? 2 : a.k;                                                                                                     \
        s.grid.y = (a.k + a.part - 1) / a.part;                                                                                          \
        routed_sum_backward_kernel<T, lanes, held, is_short><<<s.grid, s.threads, 0, stream>>>(a);                                       \
    }
    // a wavefront to a row, and a workgroup where rows are wide or few (1024 rows of 2048 in bfloat16, 4 slots: 9.8 and 7.5 us; 4096: 25.0 and 26.9);
    // very few rows: one for every two slots (29 rows of 4160, 9 slots: 15.2 us without, 6.1)
    const bool few = a.n < 2048, few_rows = a.n < 1024;
    if (a.K * sizeof(T) < 16) GROOT_SUM(16, 1, true)
    else if (pieces <= 16) GROOT_SUM(16, 1, false)
    else if (pieces <= 64) GROOT_SUM(64, 1, false)
    else if (pieces <= 128) GROOT_SUM(64, 2, false)
    else if (pieces <= 256 && !few) GROOT_SUM(64, 4, false)
    else if (pieces <= 256) GROOT_SUM(256, 1, false)
    else if (pieces <= 512) GROOT_SUM(256, 2, false)
    else if (pieces <= 1024) GROOT_SUM(256, 4, false)
    else GROOT_SUM(256, 0, false)
#undef GROOT_SUM
    return (int)hipGetLastError();
}
template <bool kOnce>
int rows_launch(RoutedArgs a, int32_t value_bytes, hipStream_t stream)
{
    const int64_t bytes = (int64_t)a.K * value_bytes, pieces = (bytes + 15) / 16;
#define GROOT_ROWS(lanes, per_lane)                                                                                                      \
    {                                                                                                                                    \
        const RoutedShape s = routed_shape(&a, pieces, lanes);                                                                           \
        routed_rows_kernel<lanes, per_lane, kOnce>                                                                                       \
            <<<s.grid, s.threads, 0, stream>>>(a, bytes, a.x_stride * value_bytes, a.out_stride * value_bytes);                          \
    }
    if (pieces <= 16) GROOT_ROWS(16, 1)
    else if (pieces <= 64) GROOT_ROWS(64, 1)
    else if (pieces <= 128) GROOT_ROWS(64, 2)
    else if (pieces <= 256) GROOT_ROWS(256, 1)
    else GROOT_ROWS(256, 2)
#undef GROOT_ROWS
    return (int)hipGetLastError();
}

}  // namespace

int launch_routed_rows(int32_t value_bytes, const RoutedArgs &a, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    return a.n * a.k * a.K * value_bytes > kRowsPast ? rows_launch<true>(a, value_bytes, s) : rows_launch<false>(a, value_bytes, s);
}

int launch_routed_sum(int32_t dtype, const RoutedArgs &a, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    const bool once = a.n * a.K * (dtype == GROOT_F32 ? 4 : 2) > kSumPast;
    if (dtype == GROOT_F32) return once ? sum_launch<float, true>(a, s) : sum_launch<float, false>(a, s);
    if (dtype == GROOT_BF16) return once ? sum_launch<bf16_t, true>(a, s) : sum_launch<bf16_t, false>(a, s);
    return once ? sum_launch<f16_t, true>(a, s) : sum_launch<f16_t, false>(a, s);
}

int launch_routed_sum_backward(int32_t dtype, const RoutedArgs &a, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    if (dtype == GROOT_F32) return sum_backward_launch<float>(a, s);
    if (dtype == GROOT_BF16) return sum_backward_launch<bf16_t>(a, s);
    return sum_backward_launch<f16_t>(a, s);
}

}  // namespace groot

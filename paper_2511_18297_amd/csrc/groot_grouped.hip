// Products grouped by node type or expert: every tile of the output belongs to one group, whose weights it takes.
//   Y[i,:] = act(X[i,:] W[g] + b[g]), dX[i,:] = dY[i,:] W[g]^T, dW[g] = X_g^T dY_g, db[g] = sum of dY_g; sums in fp32, one rounding.
// A call cannot do without n (K + N) + groups K N values and 2 n K N operations.  Tiles of seven kinds (choose_tile) serve all sizes:
// large ones where products bound (rows_kernel), small ones in many stages where the latency of a step does; rows of at most 512
// bytes are streamed past weights that stay in LDS (narrow_kernel); few rows against much weight are in groot_few.hip.
#include "groot_tile.h"

namespace groot {

namespace {

constexpr int log2_of(int64_t x)
{
    int l = 0;
    while (((int64_t)1 << l) < x) ++l;
    return l;
}

// A wavefront's 32 x 32 block of sums through 4 KB of its LDS: a lane writes its four quads of neighbouring columns of one row, and
// reads places lane % 8 of rows lane / 8 + 8 e.
template <typename S>
__device__ __forceinline__ void block_to_lds(char *scratch, const S &sums)
{
    const int lane = threadIdx.x % kWave, m = lane % 32, half = lane / 32;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const v4f x = {(float)sums[4 * q], (float)sums[4 * q + 1], (float)sums[4 * q + 2], (float)sums[4 * q + 3]};
        *(v4f *)(scratch + m * 128 + (((2 * q + half) ^ swizzle_along(m)) * 16)) = x;
    }
    wave_sync();
}
__device__ __forceinline__ v4f row_of_block(const char *scratch, int r)
{
    return *(const v4f *)(scratch + r * 128 + ((threadIdx.x % 8 ^ swizzle_along(r)) * 16));
}

// The epilogue of a wavefront's 32 x 32 blocks.  A lane's four neighbouring columns of one row would make stores of 16 bytes in 32
// rows; the block goes through 4 KB of the wavefront's LDS (its pieces where swizzle_along has them), and every store covers eight rows of 32
// whole columns.  A lane keeps one place in the columns, with its bias and scales, for all rows.
template <typename T, typename O, int kJ>
struct Epilogue {
    v4f bias[kJ], scale[kJ];
    int32_t col[kJ];

    __device__ __forceinline__ void init(const RowsProduct &p, int32_t group, int32_t first)
    {
#pragma unroll
        for (int j = 0; j < kJ; ++j) {
            col[j] = first + 32 * j + threadIdx.x % 8 * 4;
            const int64_t of = (int64_t)group * p.N + col[j];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const bool in = col[j] + k < p.N;
                scale[j][k] = std::is_same<T, int8_t>::value && in ? p.b_scale[of + k] : 1.f;
                bias[j][k] = !p.bias || !in ? 0.f : std::is_same<T, int8_t>::value ? ((const float *)p.bias)[of + k] : (float)((const O *)p.bias)[of + k];
            }
        }
    }

    // rows from `row` of the output on, of which `rows` exist
    __device__ __forceinline__ void store(const RowsProduct &p, char *scratch, const typename TileType<T>::Sum (&sums)[kJ], int64_t row, int64_t rows, bool whole)
    {
#pragma clang fp contract(off)                               // scales and bias round one by one, here as for few rows: a row's result is the same in any batch
        const int lane = threadIdx.x % kWave;
#pragma unroll
        for (int j = 0; j < kJ; ++j) {
            block_to_lds(scratch, sums[j]);
            const int32_t left = p.N - col[j];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = 8 * i + lane / 8;
                v4f y = row_of_block(scratch, r);
                if (r < rows && left > 0) {
                    const float s = std::is_same<T, int8_t>::value ? p.a_scale[row + r] : 1.f;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (std::is_same<T, int8_t>::value) y[k] = y[k] * s * scale[j][k];
                        if (p.bias) y[k] += bias[j][k];
                        if (p.relu && y[k] < 0.f) y[k] = 0.f;
                    }
                    store_quad((O *)p.out + (row + r) * p.out_stride + col[j], y, left, whole);
                }
            }
            wave_sync();
        }
    }
};

// Decoding 128 rows over 32 groups of 2048 x 2048 in bfloat16: 48 us, 5.5 TB/s of weights; 16384 rows over 8 groups of 4096 x 4096:
// 570 to 590 us, 0.93 to 0.97 PFLOP/s (1088 tiles of 256 x 256 on 256 CUs: five rounds where 4.25 would do).
// out[i,:] = epilogue(A[i,:] B[g]): a workgroup takes kM rows of a group and kN columns, a wavefront kM / kWavesM x kN / kWavesN
template <typename T, typename O, int kM, int kN, int kWavesM, int kWavesN, int kStages, bool kNMajor, bool kAligned>
__global__ __launch_bounds__(kWavesM *kWavesN *kWave) void rows_kernel(const RowsProduct p, const TileOrder order, int32_t col_tiles, bool whole)
{
    constexpr int kThreads = kWavesM * kWavesN * kWave, kI = kM / kWavesM / 32, kJ = kN / kWavesN / 32;
    typedef Stage<T, kM, kThreads, false, kAligned> StageA;
    typedef Stage<T, kN, kThreads, !kNMajor, kAligned> StageB;
    __shared__ __align__(16) char lds[(kAligned ? kStages : 2) * (StageA::kBytes + StageB::kBytes)];
    int64_t row_tile;
    int32_t col_tile;
    order.find(blockIdx.x, &row_tile, &col_tile);
    if (col_tile >= col_tiles) return;
    const RowTile t = find_tile(p.offsets, p.groups, p.n, row_tile, log2_of(kM));
    if (t.group < 0) return;
    const int32_t j0 = col_tile * kN;
    const int64_t rows = t.end - t.begin;
    const T *B = (const T *)p.B + (int64_t)t.group * p.K * p.N;
    StageA a;
    StageB b;
    a.init((const T *)p.A + t.begin * p.a_stride, p.a_stride, rows, p.K, p.K);
    if (kNMajor) b.init(B + (int64_t)j0 * p.K, p.K, p.N - j0, p.K, p.K);
    else b.init(B + j0, p.N, p.N - j0, p.K, p.N);
    const int wave = threadIdx.x / kWave;
    const int row0 = wave / kWavesN * (kM / kWavesM), col0 = wave % kWavesN * (kN / kWavesN);
    typename TileType<T>::Sum sums[kI][kJ];
    tile_product<T, kStages>(a, b, lds, (p.K + StageA::kValues - 1) / StageA::kValues, row0, col0, sums);
    __syncthreads();                                         // LDS is free
    Epilogue<T, O, kJ> epilogue;
    epilogue.init(p, t.group, j0 + col0);
#pragma unroll
    for (int i = 0; i < kI; ++i) {
        const int64_t r = row0 + 32 * i;
        epilogue.store(p, lds + wave * 4096, sums[i], t.begin + r, rows - r, whole);
    }
}

// Typed layers: rows of at most 512 bytes, at most 128 columns.  A workgroup takes 2^log_rows rows of one group and keeps the group's
// weights in LDS; its wavefronts walk over blocks of 32 rows on their own, without a barrier: every one has kStages steps of rows
// on their way or in LDS, across the blocks' borders.
// Bound by HBM: 64 x 64 in fp32 is 512 bytes and 8192 operations a row; 8.4 M rows take 0.87 ms, 4.9 TB/s, where the bytes alone take
// 0.69 and the fp32 matrix instructions 0.44.  Through tiles, the weights staged for 128 rows at a time, they took 1.3 ms.
// kSteps: how many steps of weights LDS holds.
constexpr int kNarrowBytes = 512, kNarrowRows = 32, kNarrowStage = kNarrowRows * kStepBytes;

template <typename T, typename O, int kN, int kWaves, int kStages, int kSteps, bool kNMajor, bool kAligned>
__global__ __launch_bounds__(kWaves *kWave) void narrow_kernel(const RowsProduct p, int log_rows, int32_t steps, bool whole)
{
    constexpr int kThreads = kWaves * kWave, kJ = kN / 32, kEach = kNarrowStage / 16 / kWave;
    typedef Stage<T, kN, kThreads, !kNMajor, false> StageB;  // once, through registers: from any address
    typedef Stage<T, kNarrowRows, kBlock, false, kAligned> Rows;       // its layout in LDS
    constexpr int kRing = kStages * kNarrowStage;
    __shared__ __align__(16) char lds[kWaves * kRing + kSteps * StageB::kBytes];       // every wavefront's steps, then the weights
    const RowTile t = find_tile(p.offsets, p.groups, p.n, blockIdx.x, log_rows);
    if (t.group < 0) return;
    const T *B = (const T *)p.B + (int64_t)t.group * p.K * p.N;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    char *const ring = lds + wave * kRing, *const weights = lds + kWaves * kRing;
    const int64_t rows = t.end - t.begin, pitch = p.a_stride * (int64_t)sizeof(T);
    const int32_t blocks = (int32_t)((rows + kNarrowRows - 1) / kNarrowRows), mine = (blocks - wave + kWaves - 1) / kWaves;
    const int32_t bytes = p.K * (int32_t)sizeof(T), items = mine * steps;
    const int own = lane / 8;
    const char *const from = (const char *)((const T *)p.A + t.begin * p.a_stride);
    v4i held[kAligned ? 1 : kEach];
    int32_t valid[kAligned ? 1 : kEach];
    const bool short_row = bytes < 16;
    // the next step to load: its block of rows and its place in the rows
    int32_t load_block = wave, load_step = 0;
    auto begin = [&](int slot) {
        const int64_t row = (int64_t)load_block * kNarrowRows + own;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int32_t at = load_step * kStepBytes + (lane % 8 ^ swizzle_along(8 * i + own)) * 16;
            const int32_t left = load_block < blocks ? bytes - at : 0;
            int64_t r = row + 8 * i;
            r = r < rows ? r : rows - 1;
            const char *q = from + r * pitch + at;
            if constexpr (kAligned) dma16(left > 0 ? q : (const char *)&g_zeros, lds_offset(ring) + slot * kNarrowStage + i * (kWave * 16));
            else {
                valid[i] = left;
                held[i] = short_row ? short16<T>(q, left) : raw16(load_block < blocks ? q : from + r * pitch + bytes, left);
            }
        }
        if (++load_step == steps) {
            load_step = 0;
            load_block += kWaves;
        }
    };
    if constexpr (kAligned) {
#pragma unroll
        for (int k = 0; k < kStages - 1; ++k) begin(k);
    } else {
        begin(0);
    }
    StageB b;
    b.init(B, kNMajor ? p.K : p.N, p.N, p.K, kNMajor ? p.K : p.N);
    for (int s = 0; s < steps; ++s) {
        typename StageB::Held h;
        b.template load<true>(s, h);
        b.template put<true>(h, weights + s * StageB::kBytes);
    }
    Epilogue<T, O, kJ> epilogue;
    epilogue.init(p, t.group, 0);
    __syncthreads();                                         // the weights are there
    if (mine <= 0) {
        if constexpr (kAligned) dma_wait();                  // its first loads, of zeros
        return;
    }
    typename TileType<T>::Sum sums[1][kJ];
    int now = 0, next = kStages - 1;
    int32_t s = 0, block = wave;
#pragma unroll 1
    for (int32_t item = 0; item < items; ++item) {
        if constexpr (kAligned) {
            // the stores of the last block are among what is waited for where they were issued late enough: less depth, not less safety
            dma_wait<(kStages - 2) * kEach>();
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the fragments of the step before have left its place
            begin(next);
        } else {
            wave_sync();
#pragma unroll
            for (int i = 0; i < kEach; ++i) *(v4i *)(ring + now * kNarrowStage + (i * kWave + lane) * 16) = short_row ? held[i] : cut16(held[i], valid[i]);
            wave_sync();
            begin(0);
        }
        if (s == 0) {
#pragma unroll
            for (int j = 0; j < kJ; ++j) sums[0][j] = {};
        }
        const char *const a = ring + now * kNarrowStage, *const w = weights + s * StageB::kBytes;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (s * kStepBytes + q * 32 >= bytes) break;
            const v4i fa = Rows::fragment(a, 0, q);
            v4i fb[kJ];
#pragma unroll
            for (int j = 0; j < kJ; ++j) fb[j] = StageB::fragment(w, 32 * j, q);
#pragma unroll
            for (int n = 0; n < kJ * TileType<T>::kParts; ++n) sums[0][n % kJ] = TileType<T>::mma(fb[n % kJ], fa, sums[0][n % kJ], n / kJ);
        }
        if (++s == steps) {
            const int64_t r = (int64_t)block * kNarrowRows;  // through the place of this step, which is loaded again at the next one
            epilogue.store(p, ring + now * kNarrowStage, sums[0], t.begin + r, rows - r, whole);
            s = 0;
            block += kWaves;
        }
        if constexpr (kAligned) {
            now = now + 1 == kStages ? 0 : now + 1;
            next = next + 1 == kStages ? 0 : next + 1;
        }
    }
    if constexpr (kAligned) dma_wait();
}

bool on16(const void *a, int64_t bytes) { return (((uintptr_t)a | (uintptr_t)bytes) & 15) == 0; }

template <typename T, bool kNMajor>
bool rows_aligned(const RowsProduct &p)
{
    const int64_t b = sizeof(T);
    return on16(p.A, p.a_stride * b) && on16(p.B, (kNMajor ? p.K : p.N) * b) && p.K * b % 16 == 0;
}

template <typename O>
bool out_whole(const RowsProduct &p) { return (((uintptr_t)p.out | (uintptr_t)(p.out_stride * sizeof(O))) & (4 * sizeof(O) - 1)) == 0; }

template <typename T, typename O, int kM, int kN, int kWavesM, int kWavesN, int kStages, bool kNMajor, bool kAligned>
int rows_launch(const RowsProduct &p, void *stream)
{
    const int32_t col_tiles = (p.N + kN - 1) / kN;
    const TileOrder order((p.n + kM - 1) / kM + (p.offsets ? p.groups : 0), col_tiles);
    constexpr int kThreads = kWavesM * kWavesN * kWave;
    if (!fits_launch(order.workgroups, kThreads)) return kErrTooManyTiles;
    rows_kernel<T, O, kM, kN, kWavesM, kWavesN, kStages, kNMajor, kAligned>
        <<<(uint32_t)order.workgroups, kThreads, 0, (hipStream_t)stream>>>(p, order, col_tiles, out_whole<O>(p));
    return (int)hipGetLastError();
}

template <typename T, typename O, int kN, int kStages, int kSteps, bool kNMajor, bool kAligned>
int narrow_launch_as(const RowsProduct &p, int log_rows, int32_t steps, void *stream)
{
    constexpr int kWaves = 8;
    const int64_t workgroups = ((p.n - 1) >> log_rows) + 1 + (p.offsets ? p.groups : 0);
    if (!fits_launch(workgroups, kWaves * kWave)) return kErrTooManyTiles;
    narrow_kernel<T, O, kN, kWaves, kStages, kSteps, kNMajor, kAligned>
        <<<(uint32_t)workgroups, kWaves * kWave, 0, (hipStream_t)stream>>>(p, log_rows, steps, out_whole<O>(p));
    return (int)hipGetLastError();
}

// LDS of as many steps as leave a CU the workgroups that the row's own number would: 160 KB hold two of 80, three of 48 or 53, four of 40.
// (A size at the launch would have to be asked of the runtime first, above 64 KB, for every device.)
template <typename T, typename O, int kN, bool kNMajor>
int narrow_launch(const RowsProduct &p, void *stream)
{
    const int32_t steps = (int32_t)((p.K * sizeof(T) + kStepBytes - 1) / kStepBytes);
    static_assert(kNarrowBytes == 4 * kStepBytes, "at most four steps");
    const bool aligned = on16(p.A, p.a_stride * (int64_t)sizeof(T)) && p.K * (int64_t)sizeof(T) % 16 == 0;
    int log_rows = 8;                                        // about 1024 workgroups, of 256 rows at least
    while (log_rows < 20 && ((int64_t)1024 << log_rows) < p.n) ++log_rows;
    // 16 wavefronts to a CU with a step of their own on the way each; 8 with two or three were 8 % slower at 64 x 64, 14 % at 128 x 128
    if (aligned) {
        constexpr int kSome = kN == 64 ? 2 : 1;              // 80 KB, else 96 or 128
        return steps <= kSome ? narrow_launch_as<T, O, kN, 2, kSome, kNMajor, true>(p, log_rows, steps, stream)
                              : narrow_launch_as<T, O, kN, 2, 4, kNMajor, true>(p, log_rows, steps, stream);
    }
    constexpr int kSome = kN == 64 ? 2 : 3;                  // 40, 48 or 64 KB; 48, 80 or 96
    return steps == 1       ? narrow_launch_as<T, O, kN, 1, 1, kNMajor, false>(p, log_rows, steps, stream)
           : steps <= kSome ? narrow_launch_as<T, O, kN, 1, kSome, kNMajor, false>(p, log_rows, steps, stream)
                            : narrow_launch_as<T, O, kN, 1, 4, kNMajor, false>(p, log_rows, steps, stream);
}

// What a step of the contraction (128 bytes of every row) takes, in ns, with up to 256 and with up to 512 tiles of a kind on the GPU's
// 256 CUs, measured over K of 4096 bytes on one group whose tiles come out even.  fp32 is bound by its matrix instructions at every
// size; the others by theirs in large tiles, by the latency of a step's loads in small ones.  The kinds, rows x columns and stages:
//   256 x 256, 2; 128 x 128, 2; 128 x 128, 4; 64 x 128, 3; 64 x 64, 5; 32 x 128, 4; 32 x 64, 6
struct TileCost {
    int32_t rows, cols, to256, to512;        // to512 0: one tile to a CU; to256 0: not built, as it would never be the least
};
constexpr int kTileKinds = 7;
constexpr TileCost kTile16[kTileKinds] = {{256, 256, 2060, 0}, {128, 128, 1000, 1270}, {128, 128, 790, 0}, {64, 128, 550, 840},
                                          {64, 64, 380, 570}, {32, 128, 410, 630}, {32, 64, 400, 420}};
constexpr TileCost kTile32[kTileKinds] = {{256, 256, 0, 0}, {128, 128, 2360, 4540}, {128, 128, 0, 0}, {64, 128, 1330, 2370},
                                          {64, 64, 830, 1370}, {32, 128, 870, 1430}, {32, 64, 820, 880}};

// The kind of tile that takes the least time by that table; rows that do not begin on 16 bytes go through registers, for which three
// of the kinds are built.
template <typename T>
int choose_tile(int64_t n, int32_t groups, bool offsets, int32_t N, bool aligned)
{
    int best = -1;
    double least = 0;
    for (int k = 0; k < kTileKinds; ++k) {
        if (!aligned && k != 1 && k != 4 && k != 6) continue;
        const TileCost &c = sizeof(T) == 4 ? kTile32[k] : kTile16[k];
        if (!c.to256) continue;
        // a group's last tile is half full, on average
        double rows = offsets ? (double)n / c.rows + 0.5 * groups : (double)((n + c.rows - 1) / c.rows);
        const double least_rows = (double)(n < groups ? n : groups);
        rows = rows < least_rows ? least_rows : rows;
        const double tiles = rows * ((N + c.cols - 1) / c.cols), at_once = c.to512 ? 512 : 256;
        const double full = (double)(int64_t)(tiles / at_once), rest = tiles - full * at_once, all = c.to512 ? c.to512 : c.to256;
        double time = full * all + (rest <= 0 ? 0 : rest > 256 ? c.to512 : c.to256);
        // ragged groups: the number is a guess, and near or above a full GPU half a round more is
        if (offsets && tiles > 0.8 * at_once) time = (tiles / at_once + 0.5) * all;
        if (best < 0 || time < least) best = k, least = time;
    }
    return best;
}

template <typename T, typename O, bool kNMajor>
int rows_choose(const RowsProduct &p, void *stream)
{
    const int64_t each = p.n / p.groups;                      // rows of a group, on average
    if (p.K * (int)sizeof(T) <= kNarrowBytes && p.N <= 128 && each >= 64)
        return p.N <= 64 ? narrow_launch<T, O, 64, kNMajor>(p, stream) : narrow_launch<T, O, 128, kNMajor>(p, stream);
    const bool aligned = rows_aligned<T, kNMajor>(p);
    const int kind = choose_tile<T>(p.n, p.groups, p.offsets != nullptr, p.N, aligned);
    if (!aligned) {
        if (kind == 1) return rows_launch<T, O, 128, 128, 2, 2, 2, kNMajor, false>(p, stream);
        if (kind == 4) return rows_launch<T, O, 64, 64, 2, 2, 2, kNMajor, false>(p, stream);
        return rows_launch<T, O, 32, 64, 1, 2, 2, kNMajor, false>(p, stream);
    }
    switch (kind) {
    case 0:
        if constexpr (sizeof(T) < 4) return rows_launch<T, O, 256, 256, 2, 4, 2, kNMajor, true>(p, stream);
    case 1: return rows_launch<T, O, 128, 128, 2, 2, 2, kNMajor, true>(p, stream);
    case 2:
        if constexpr (sizeof(T) < 4) return rows_launch<T, O, 128, 128, 2, 2, 4, kNMajor, true>(p, stream);
    case 3: return rows_launch<T, O, 64, 128, 2, 2, 3, kNMajor, true>(p, stream);
    case 4: return rows_launch<T, O, 64, 64, 2, 2, 5, kNMajor, true>(p, stream);
    case 5: return rows_launch<T, O, 32, 128, 1, 4, 4, kNMajor, true>(p, stream);
    default: return rows_launch<T, O, 32, 64, 1, 2, 6, kNMajor, true>(p, stream);
    }
}

// How the weight gradients are cut.  Tiles of dW of 256 x 256 where all groups' fill the GPU, else of 128, or 64 along a side that is
// no longer (typed layers).  The contraction, a group's rows, is cut into pieces of 2^log_rows rows where there are fewer tiles than
// workgroups that the GPU holds; a piece of 512 rows reads eight times what its partial sums are written and read again for.  A
// group of one piece needs no partial sums, and a group without rows is one piece of zeros.
struct WeightsSplit {
    int32_t k_tile, n_tile;                  // 64 or 128 each, or both 256
    int32_t k_tiles, n_tiles;
    int log_rows;
    int64_t tiles;                           // pieces of all groups, at most
    int64_t slots;                           // pieces of groups that are cut, at most
    WeightsSplit(int32_t dtype, int64_t n, int32_t groups, bool offsets, int32_t K, int32_t N)
    {
        const auto tiles_of = [](int32_t width, int32_t by) { return (width + by - 1) / by; };
        k_tile = K <= 64 ? 64 : 128;
        n_tile = N <= 64 ? 64 : 128;
        if (dtype != GROOT_F32 && (int64_t)tiles_of(K, 256) * tiles_of(N, 256) * groups >= 192 && n >= (int64_t)256 * groups) k_tile = n_tile = 256;
        k_tiles = tiles_of(K, k_tile);
        n_tiles = tiles_of(N, n_tile);
        const int64_t wanted = k_tile == 64 || n_tile == 64 ? 1024 : 256;
        log_rows = 9;
        while (log_rows < 40 && (wanted << log_rows) < n * k_tiles * n_tiles) ++log_rows;
        // enough tiles without cutting: only groups of four times the average are cut
        if ((int64_t)groups * k_tiles * n_tiles >= wanted)
            while (log_rows < 40 && ((int64_t)groups << log_rows) < 4 * n) ++log_rows;
        const int64_t rows = (int64_t)1 << log_rows;
        tiles = (n + rows - 1) / rows + (offsets ? groups : 0);
        if (tiles < 1) tiles = 1;
        slots = n <= rows ? 0 : 2 * (n / rows);
        if (slots > tiles) slots = tiles;
    }
};

// dW[g] = X_g^T dY_g and the column sums of dY_g: a workgroup takes kK x kN of one group's product and one piece of the group's
// rows.  The partial sums of a group in several pieces lie in the workspace, piece after piece, K x N and N floats each.
// 8.4 M rows, 64 x 64, fp32: 0.80 ms, 5.4 TB/s of X and dY; 16384 rows, 4096 x 4096, bfloat16: 490 us, 1.12 PFLOP/s.
template <typename T, typename O, int kK, int kN, int kWavesK, int kWavesN, int kStages, bool kAligned>
__global__ __launch_bounds__(kWavesK *kWavesN *kWave) void weights_kernel(const WeightsProduct p, const TileOrder order, int log_rows, int64_t slots,
                                                                         int32_t k_tiles, int32_t n_tiles)
{
    constexpr int kThreads = kWavesK * kWavesN * kWave, kI = kK / kWavesK / 32, kJ = kN / kWavesN / 32;
    typedef Stage<T, kK, kThreads, true, kAligned> StageX;
    typedef Stage<T, kN, kThreads, true, kAligned> StageY;
    __shared__ __align__(16) char lds[(kAligned ? kStages : 2) * (StageX::kBytes + StageY::kBytes)];
    int64_t row_tile;
    int32_t n_tile;
    order.find(blockIdx.x, &row_tile, &n_tile);
    if (n_tile >= n_tiles) return;
    const RowTile t = find_tile<true, true>(p.offsets, p.groups, p.n, row_tile / k_tiles, log_rows);
    if (t.group < 0) return;
    const int32_t n0 = n_tile * kN, k0 = (int32_t)(row_tile % k_tiles) * kK;
    StageX x;
    StageY y;
    x.init((const T *)p.X + t.begin * p.x_stride + k0, p.x_stride, p.K - k0, t.end - t.begin, p.K);
    y.init((const T *)p.dY + t.begin * p.dy_stride + n0, p.dy_stride, p.N - n0, t.end - t.begin, p.N);
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int row0 = wave / kWavesN * (kK / kWavesK), col0 = wave % kWavesN * (kN / kWavesN);
    typename TileType<T>::Sum sums[kI][kJ];
    float columns[kJ] = {};
    const bool bias = p.dbias && k0 == 0 && row0 == 0;
    tile_product<T, kStages, true>(x, y, lds, (t.end - t.begin + kStepValues<T> - 1) / kStepValues<T>, row0, col0, sums, &columns, bias);
    const bool alone = t.count == 1;
    if (!alone && t.shared_before + t.place >= slots) return;   // offsets that do not ascend: more pieces than there are rows for
    float *const part = (float *)p.workspace + (t.shared_before + t.place) * ((int64_t)p.K * p.N + p.N);
    const bool whole = p.N % 4 == 0 && (!alone || ((uintptr_t)p.dW & (4 * sizeof(O) - 1)) == 0);
    __syncthreads();                                         // LDS is free
    char *const scratch = lds + wave * 4096;
#pragma unroll
    for (int i = 0; i < kI; ++i)
#pragma unroll
        for (int j = 0; j < kJ; ++j) {
            block_to_lds(scratch, sums[i][j]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = 8 * e + lane / 8;
                const int32_t k = k0 + row0 + 32 * i + r, n = n0 + col0 + 32 * j + lane % 8 * 4;
                const v4f v = row_of_block(scratch, r);
                if (k >= p.K || n >= p.N) continue;
                if (alone) store_quad((O *)p.dW + ((int64_t)t.group * p.K + k) * p.N + n, v, p.N - n, whole);
                else store_quad(part + (int64_t)k * p.N + n, v, p.N - n, whole);
            }
            wave_sync();
        }
    if (bias) {
#pragma unroll
        for (int j = 0; j < kJ; ++j) {
            const float s = columns[j] + __shfl_xor(columns[j], 32);
            const int32_t n = n0 + col0 + 32 * j + lane % 32;
            if (lane >= 32 || n >= p.N) continue;
            if (alone) ((O *)p.dbias)[(int64_t)t.group * p.N + n] = (O)s;
            else part[(int64_t)p.K * p.N + n] = s;
        }
    }
}

// The partial sums of groups in several pieces, added up in fp64.  A lane takes four neighbouring values; `shares` (a power of two)
// lanes of a workgroup take the same four, each a share of the pieces, and their sums meet in LDS.  dbias lies behind dW.
constexpr int kSumLanes = 512;

template <typename O>
__global__ __launch_bounds__(kSumLanes) void weights_sum_kernel(const WeightsProduct p, int log_rows, int64_t slots, uint32_t per_group, int shares)
{
    typedef double v4d __attribute__((ext_vector_type(4)));
    __shared__ v4d sums[kSumLanes];
    const int32_t g = (int32_t)(blockIdx.x / per_group);
    const int lane = threadIdx.x % kWave, quads = kSumLanes / shares, quad = threadIdx.x % quads, share = threadIdx.x / quads;
    const int64_t rows = (int64_t)1 << log_rows;
    int64_t begin, end, before = 0;
    group_rows(p.offsets, p.n, g, &begin, &end);
    int64_t count = (end - begin + rows - 1) >> log_rows;
    if (count <= 1) return;
    for (int32_t g0 = 0; g0 < g; g0 += kWave) {
        int64_t b = 0, e = 0;
        if (g0 + lane < g) group_rows(p.offsets, p.n, g0 + lane, &b, &e);
        const int64_t c = (e - b + rows - 1) >> log_rows;
        before += __shfl(sum_upto(c > 1 ? c : 0), kWave - 1);
    }
    count = before + count <= slots ? count : before < slots ? slots - before : 0;
    const int64_t dw = (int64_t)p.K * p.N, slot = dw + p.N, values = p.dbias ? slot : dw;
    for (int64_t first = (int64_t)(blockIdx.x % per_group) * quads * 4; first < values; first += (int64_t)per_group * quads * 4) {
        const int64_t at = first + quad * 4;
        const float *from = (const float *)p.workspace + before * slot + at;
        v4d sum = {0, 0, 0, 0};
        if (slot % 4 == 0 && at + 4 <= values) {
#pragma unroll 4
            for (int64_t c = share; c < count; c += shares) {
                const v4f x = *(const v4f *)(from + c * slot);
#pragma unroll
                for (int k = 0; k < 4; ++k) sum[k] += (double)x[k];
            }
        } else {
            for (int64_t c = share; c < count; c += shares)
                for (int k = 0; k < 4; ++k)
                    if (at + k < values) sum[k] += (double)from[c * slot + k];
        }
        if (shares > 1) {
            sums[threadIdx.x] = sum;
            __syncthreads();
            if (share == 0)
                for (int w = 1; w < shares; ++w) sum += sums[w * quads + quad];
            __syncthreads();
            if (share) continue;
        }
        const v4f total = {(float)sum[0], (float)sum[1], (float)sum[2], (float)sum[3]};
        if (at + 4 <= dw) {
            store_quad((O *)p.dW + g * dw + at, total, 4, ((uintptr_t)p.dW | (uintptr_t)(dw * sizeof(O))) % (4 * sizeof(O)) == 0);
        } else {
            for (int k = 0; k < 4; ++k) {
                const int64_t i = at + k;
                if (i < dw) ((O *)p.dW)[g * dw + i] = (O)total[k];
                else if (i < values) ((O *)p.dbias)[(int64_t)g * p.N + (i - dw)] = (O)total[k];
            }
        }
    }
}

template <typename T, typename O, int kK, int kN, int kWavesK, int kWavesN, int kStages, bool kAligned>
int weights_launch_tile(const WeightsProduct &p, const WeightsSplit &split, hipStream_t stream)
{
    constexpr int kThreads = kWavesK * kWavesN * kWave;
    const int32_t k_tiles = (p.K + kK - 1) / kK, n_tiles = (p.N + kN - 1) / kN;
    const TileOrder order(split.tiles * k_tiles, n_tiles);
    if (!fits_launch(order.workgroups, kThreads)) return kErrTooManyTiles;
    weights_kernel<T, O, kK, kN, kWavesK, kWavesN, kStages, kAligned>
        <<<(uint32_t)order.workgroups, kThreads, 0, stream>>>(p, order, split.log_rows, split.slots, k_tiles, n_tiles);
    return (int)hipGetLastError();
}

template <typename T, typename O, bool kAligned>
int weights_launch_as(const WeightsProduct &p, const WeightsSplit &split, hipStream_t s)
{
    if (split.k_tile == 64 && split.n_tile == 64) return weights_launch_tile<T, O, 64, 64, 2, 2, 2, kAligned>(p, split, s);
    if (split.k_tile == 64) return weights_launch_tile<T, O, 64, 128, 2, 2, 2, kAligned>(p, split, s);
    if (split.n_tile == 64) return weights_launch_tile<T, O, 128, 64, 2, 2, 2, kAligned>(p, split, s);
    if constexpr (kAligned) {
        if constexpr (sizeof(T) == 2)
            if (split.k_tile == 256) return weights_launch_tile<T, O, 256, 256, 2, 4, 2, true>(p, split, s);
        // four stages where a CU has one tile at most
        if ((int64_t)p.groups * split.k_tiles * split.n_tiles <= 256 && split.slots == 0) return weights_launch_tile<T, O, 128, 128, 2, 2, 4, true>(p, split, s);
    }
    return weights_launch_tile<T, O, 128, 128, 2, 2, 2, kAligned>(p, split, s);   // also for 256 x 256, not built for rows through registers
}

template <typename T, typename O>
int weights_launch(int32_t dtype, const WeightsProduct &p, void *stream)
{
    const int64_t b = sizeof(T);
    const bool aligned = on16(p.X, p.x_stride * b) && on16(p.dY, p.dy_stride * b) && p.K * b % 16 == 0 && p.N * b % 16 == 0;
    const WeightsSplit split(dtype, p.n, p.groups, p.offsets != nullptr, p.K, p.N);
    const hipStream_t s = (hipStream_t)stream;
    const int err = aligned ? weights_launch_as<T, O, true>(p, split, s) : weights_launch_as<T, O, false>(p, split, s);
    if (err) return err;
    if (split.slots == 0) return 0;
    int shares = 1;                                          // a share for every four pieces that a group has on average, 64 at most
    while (shares < 64 && (int64_t)shares * 4 * p.groups < split.tiles) shares *= 2;
    const int64_t parts = ((int64_t)p.K * p.N + p.N + kSumLanes / shares * 4 - 1) / (kSumLanes / shares * 4);
    int64_t per_group = 4096 / p.groups;
    per_group = per_group < 1 ? 1 : per_group > parts ? parts : per_group;
    weights_sum_kernel<O><<<(uint32_t)(per_group * p.groups), kSumLanes, 0, s>>>(p, split.log_rows, split.slots, (uint32_t)per_group, shares);
    return (int)hipGetLastError();
}

}  // namespace

int launch_grouped_rows(int32_t dtype, const RowsProduct &p, void *stream)
{
    if (few_rows_serve(p)) return launch_few_rows(dtype, p, stream);
    if (dtype == GROOT_F32) return p.b_n_major ? rows_choose<float, float, true>(p, stream) : rows_choose<float, float, false>(p, stream);
    if (dtype == GROOT_BF16) return p.b_n_major ? rows_choose<bf16_t, bf16_t, true>(p, stream) : rows_choose<bf16_t, bf16_t, false>(p, stream);
    return p.b_n_major ? rows_choose<f16_t, f16_t, true>(p, stream) : rows_choose<f16_t, f16_t, false>(p, stream);
}

int launch_int8_rows(int32_t out_dtype, const RowsProduct &p, void *stream)
{
    if (few_rows_serve(p)) return launch_few_int8(out_dtype, p, stream);
    if (out_dtype == GROOT_F32) return rows_choose<int8_t, float, true>(p, stream);
    if (out_dtype == GROOT_BF16) return rows_choose<int8_t, bf16_t, true>(p, stream);
    return rows_choose<int8_t, f16_t, true>(p, stream);
}

size_t grouped_weights_workspace(int32_t dtype, int64_t n, int32_t groups, int32_t K, int32_t N)
{
    // whether the call will have offsets is not known here: without, there is one group and no more pieces than with
    const WeightsSplit split(dtype, n, groups, true, K, N);
    return (size_t)split.slots * ((size_t)K * N + N) * 4;
}

int launch_grouped_weights(int32_t dtype, const WeightsProduct &p, void *stream)
{
    if (dtype == GROOT_F32) return weights_launch<float, float>(dtype, p, stream);
    if (dtype == GROOT_BF16) return p.grad_f32 ? weights_launch<bf16_t, float>(dtype, p, stream) : weights_launch<bf16_t, bf16_t>(dtype, p, stream);
    return p.grad_f32 ? weights_launch<f16_t, float>(dtype, p, stream) : weights_launch<f16_t, f16_t>(dtype, p, stream);
}

}  // namespace groot

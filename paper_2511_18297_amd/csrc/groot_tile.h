// Matrix-core tiles shared by the grouped products and the products in 8-bit integers.
//
// A step of the contraction is 128 bytes of a row whose elements lie along it ("along": 64 values of 16 bits, 32 of fp32, 128 of
// 8 bits), or as many rows of a matrix whose rows lie across it ("across").  Both operands of a step are staged in LDS by loads
// that go there directly (16 bytes a lane, no registers), twice: one pair of tiles is computed while the next one arrives.
//   along   row r at r * 128, its 16-byte piece c at place c ^ (r & 7): the 32 rows that a fragment reads fall on all banks
//   across  row k of the contraction at k * width, its piece c at c ^ ((k & 3) << 1) (16-bit types): the four rows that a
//           transposing read of 16 lanes takes fall on different banks
// A fragment of the 32 x 32 matrix instructions is 16 bytes a lane, from row (lane & 31) and piece 2 s + (lane >> 5) of sub-step
// s = 0 .. 3; for fp32 that is four instructions of two values of the contraction each, in an order of their own that both
// operands share.  The operands change places (columns of the result first), so that a lane holds four neighbouring columns.
#pragma once

#include "groot_dense_device.h"

namespace groot {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef int v16i __attribute__((ext_vector_type(16)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef bf16_t v8bf __attribute__((ext_vector_type(8)));
typedef f16_t v8h __attribute__((ext_vector_type(8)));

typedef __attribute__((address_space(3))) char lds_char;

template <typename T>
struct TileType;
template <>
struct TileType<bf16_t> {
    typedef v16f Sum;
    // the sum of a fragment's values
    static __device__ __forceinline__ float total(v4i a)
    {
        const v8bf x = __builtin_bit_cast(v8bf, a);
        return (((float)x[0] + (float)x[1]) + ((float)x[2] + (float)x[3])) + (((float)x[4] + (float)x[5]) + ((float)x[6] + (float)x[7]));
    }
    static __device__ __forceinline__ Sum mma(v4i a, v4i b, Sum c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
    }
};
template <>
struct TileType<f16_t> {
    typedef v16f Sum;
    static __device__ __forceinline__ float total(v4i a)
    {
        const v8h x = __builtin_bit_cast(v8h, a);
        return (((float)x[0] + (float)x[1]) + ((float)x[2] + (float)x[3])) + (((float)x[4] + (float)x[5]) + ((float)x[6] + (float)x[7]));
    }
    static __device__ __forceinline__ Sum mma(v4i a, v4i b, Sum c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
    }
};
template <>
struct TileType<int8_t> {
    typedef v16i Sum;
    static __device__ __forceinline__ Sum mma(v4i a, v4i b, Sum c) { return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0); }
};
template <>
struct TileType<float> {
    typedef v16f Sum;
    static __device__ __forceinline__ float total(v4i a)
    {
        return (__int_as_float(a[0]) + __int_as_float(a[1])) + (__int_as_float(a[2]) + __int_as_float(a[3]));
    }
    static __device__ __forceinline__ Sum mma(v4i a, v4i b, Sum c)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            c = __builtin_amdgcn_mfma_f32_32x32x2f32(__int_as_float(a[j]), __int_as_float(b[j]), c, 0, 0, 0);
        return c;
    }
};

constexpr int kStepBytes = 128;
template <typename T>
constexpr int kStepValues = kStepBytes / (int)sizeof(T);

__device__ __forceinline__ uint32_t lds_offset(const void *p) { return (uint32_t)(uintptr_t)(lds_char *)p; }

// 16 bytes of every lane from its own address to LDS, lane after lane from `to` on.  The compiler does not see the load: dma_wait
// before anything reads what arrived.  (A write to m0 needs one wait state before a load that goes by it.)
__device__ __forceinline__ void dma16(const void *from, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(__builtin_amdgcn_readfirstlane(to)), "v"(from) : "memory");
}

// until at most kMost of the wavefront's latest loads are on their way
template <int kMost = 0>
__device__ __forceinline__ void dma_wait()
{
    static_assert(kMost >= 0 && kMost < 64, "vmcnt");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kMost) : "memory");
}

static __device__ const v4i g_zeros = {0, 0, 0, 0};          // what lies past an end of the contraction

// 16 bytes from any address, of which the first `valid` exist
template <typename T>
__device__ __forceinline__ v4i load16(const char *p, int64_t valid)
{
    v4i x = {0, 0, 0, 0};
    if (valid >= 16) {
        __builtin_memcpy(&x, p, 16);
    } else {
        T e[16 / sizeof(T)] = {};
        for (int k = 0; k < (int)(16 / sizeof(T)); ++k)
            if ((int64_t)(k * sizeof(T)) < valid) e[k] = ((const T *)p)[k];
        __builtin_memcpy(&x, e, 16);
    }
    return x;
}

// Rows cut to 8 bits.  The 16 bytes of a load as floats; the scale of a row from its largest magnitude (not finite: NaN); the codes of
// a load, halves to even, zeros where the scale is zero or NaN.
template <typename X>
struct RowValues {
    float x[16 / sizeof(X)];
};
template <typename X>
__device__ __forceinline__ RowValues<X> row_values(v4i v)
{
    typedef X vx __attribute__((ext_vector_type(16 / sizeof(X))));
    const vx e = __builtin_bit_cast(vx, v);
    RowValues<X> r;
#pragma unroll
    for (int k = 0; k < (int)(16 / sizeof(X)); ++k) r.x[k] = (float)e[k];
    return r;
}

__device__ __forceinline__ float row_scale(float top) { return __builtin_isfinite(top) ? top * (1.f / 127.f) : __builtin_nanf(""); }

template <typename X>
__device__ __forceinline__ void row_codes(v4i v, float scale, int8_t *to)
{
    constexpr int kPer = 16 / sizeof(X);
    const RowValues<X> e = row_values<X>(v);
    union {
        int8_t c[kPer];
        uint32_t u[kPer / 4];
    } q;
#pragma unroll
    for (int k = 0; k < kPer; ++k) q.c[k] = scale > 0.f ? (int8_t)fminf(fmaxf(rintf(e.x[k] / scale), -127.f), 127.f) : (int8_t)0;
    __builtin_memcpy(__builtin_assume_aligned(to, kPer), q.u, kPer);
}

// One operand's tile: kWide rows ("along") or columns ("across").  begin(s) starts the loads of step s, end(s) has them in LDS once
// the workgroup has passed a barrier.
template <typename T, int kWide, int kThreads, bool kAcross, bool kAligned>
struct Stage {
    static constexpr bool kDirect = kAligned;
    static constexpr int kBytes = kWide * kStepBytes, kEach = kBytes / 16 / kThreads;
    static constexpr int kRowBytes = kAcross ? kWide * (int)sizeof(T) : kStepBytes, kPieces = kRowBytes / 16;
    static constexpr int kRowsEach = kThreads / kPieces;     // rows of the tile that one load of the workgroup takes
    static_assert(kBytes % (16 * kThreads) == 0 && kThreads % kPieces == 0, "a whole number of loads of whole rows");
    static_assert(kAcross ? sizeof(T) == 4 || (kRowsEach % 4 == 0 && kPieces >= 8) : kRowsEach % 8 == 0, "a lane's piece is the same in all its loads");

    const char *src[kAcross ? 1 : kEach];
    int64_t pitch, limit;                                    // bytes between rows; bytes ("along") or rows ("across") of the contraction
    int64_t width;                                           // across: bytes of a row from the lane's piece on
    int32_t piece, row;
    v4i held[kAligned ? 1 : kEach];

    static __device__ __forceinline__ int swizzle(int r) { return kAcross ? (sizeof(T) == 2 ? (r & 3) << 1 : 0) : r & 7; }

    // along: `base` is the first row's first value, `rows` rows exist, `extent` values of the contraction
    // across: `base` is the first value of the tile's first column in the contraction's first row, `columns` columns exist
    __device__ __forceinline__ void init(const T *base, int64_t stride, int64_t exist, int64_t extent)
    {
        const int tid = threadIdx.x;
        row = tid / kPieces;
        piece = (tid % kPieces) ^ swizzle(row);
        pitch = stride * (int64_t)sizeof(T);
        if (kAcross) {
            limit = extent;
            width = exist * (int64_t)sizeof(T) - piece * 16;
            const int64_t last = (exist * (int64_t)sizeof(T) - 1) / 16 * 16;       // a piece past the last column reads the last one
            src[0] = (const char *)base + row * pitch + (kAligned && width <= 0 ? last : (int64_t)piece * 16);
        } else {
            limit = extent * (int64_t)sizeof(T);
#pragma unroll
            for (int i = 0; i < kEach; ++i) {                // rows that do not exist read the last one that does
                const int64_t r = row + i * kRowsEach;
                src[i] = (const char *)base + (r < exist ? r : exist - 1) * pitch + piece * 16;
            }
        }
    }

    __device__ __forceinline__ void begin(int64_t s, char *tile)
    {
        const uint32_t to = lds_offset(tile) + threadIdx.x / kWave * (kWave * 16);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const char *p;
            int64_t left;
            if (kAcross) {
                const int64_t k = s * kStepValues<T> + row + i * kRowsEach;
                p = src[0] + (s * kStepValues<T> + i * kRowsEach) * pitch;
                left = k < limit ? width : 0;
                if (kAligned) p = k < limit ? p : (const char *)&g_zeros;
            } else {
                p = src[i] + s * kStepBytes;
                left = limit - s * kStepBytes - piece * 16;
                if (kAligned) p = left > 0 ? p : (const char *)&g_zeros;
            }
            if constexpr (kAligned) dma16(p, to + i * (kThreads * 16));
            else held[i] = load16<T>(p, left);
        }
    }

    __device__ __forceinline__ void end(char *tile)
    {
        if constexpr (!kAligned) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) *(v4i *)(tile + (i * kThreads + threadIdx.x) * 16) = held[i];
        }
    }

    // the lane's 16 bytes of the 32 rows (columns) from `first` on, sub-step s
    static __device__ __forceinline__ v4i fragment(const char *tile, int first, int s)
    {
        const int lane = threadIdx.x % kWave, half = lane / 32;
        if constexpr (!kAcross) {
            const int r = first + lane % 32;
            return *(const v4i *)(tile + r * kStepBytes + (((2 * s + half) ^ swizzle(r)) * 16));
        } else if constexpr (sizeof(T) == 2) {
            // 16 lanes give the addresses of four rows of 16 columns and get a column's four values each
            const int i = lane % 16, k = 16 * s + 8 * half + i / 4, c = (first + (lane / 16 % 2) * 16) / 8;
            const char *p = tile + k * kRowBytes + ((c ^ swizzle(k)) * 16) + (i % 4) * 8;
            const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)p);
            const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)(p + 4 * kRowBytes));
            return __builtin_bit_cast(v4i, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            v4i x;
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = *(const int *)(tile + (8 * s + 4 * half + j) * kRowBytes + (first + lane % 32) * 4);
            return x;
        }
    }
};

// One step's products of the wavefront's 32 x 32 blocks.
template <typename T, bool kColumns, class StageA, class StageB, int kI, int kJ>
__device__ __forceinline__ void tile_step(const char *now, int row0, int col0, typename TileType<T>::Sum (&sums)[kI][kJ], float (*columns)[kJ], bool mine)
{
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        v4i fa[kI], fb[kJ];
#pragma unroll
        for (int i = 0; i < kI; ++i) fa[i] = StageA::fragment(now, row0 + 32 * i, q);
#pragma unroll
        for (int j = 0; j < kJ; ++j) fb[j] = StageB::fragment(now + StageA::kBytes, col0 + 32 * j, q);
#pragma unroll
        for (int i = 0; i < kI; ++i)
#pragma unroll
            for (int j = 0; j < kJ; ++j) sums[i][j] = TileType<T>::mma(fb[j], fa[i], sums[i][j]);
        if constexpr (kColumns) {
            if (mine) {
#pragma unroll
                for (int j = 0; j < kJ; ++j) (*columns)[j] += TileType<T>::total(fb[j]);
            }
        }
    }
}

// The product of two staged operands over `steps` steps: sums[i][j] of the wavefront's 32 x 32 blocks, rows of `A` from row0 on,
// columns of `B` from col0 on.  kStages pairs of tiles lie in LDS, so that kStages - 1 steps are on their way while one is computed.
// `columns` (where kColumns; wavefronts with `mine`): the sums of B's values, lanes l and l + 32 hold the two halves of column l.
template <typename T, int kStages, bool kColumns = false, class StageA, class StageB, int kI, int kJ>
__device__ __forceinline__ void tile_product(StageA &a, StageB &b, char *lds, int64_t steps, int row0, int col0,
                                             typename TileType<T>::Sum (&sums)[kI][kJ], float (*columns)[kJ] = nullptr, bool mine = false)
{
    constexpr int kBoth = StageA::kBytes + StageB::kBytes;
#pragma unroll
    for (int i = 0; i < kI; ++i)
#pragma unroll
        for (int j = 0; j < kJ; ++j) sums[i][j] = {};
    if (steps <= 0) return;
    if constexpr (StageA::kDirect) {
        // a step past the last one loads zeros that nothing reads: every step has the same number of loads to count
        constexpr int kEach = StageA::kEach + StageB::kEach;
        auto begin = [&](int64_t s, int at) {
            a.begin(s, lds + at);
            b.begin(s, lds + at + StageA::kBytes);
        };
#pragma unroll
        for (int s = 0; s < kStages - 1; ++s) begin(s, s * kBoth);
        int now = 0, next = (kStages - 1) * kBoth;
#pragma unroll 1
        for (int64_t s = 0; s < steps; ++s) {
            dma_wait<(kStages - 2) * kEach>();
            __syncthreads();                                 // step s has arrived, and nobody reads the tile that is loaded next
            begin(s + kStages - 1, next);
            tile_step<T, kColumns, StageA, StageB>(lds + now, row0, col0, sums, columns, mine);
            now = now + kBoth == kStages * kBoth ? 0 : now + kBoth;
            next = next + kBoth == kStages * kBoth ? 0 : next + kBoth;
        }
        dma_wait();                                          // before the workgroup's LDS is anybody else's
    } else {
        auto begin = [&](int64_t s) {
            a.begin(s, lds);
            b.begin(s, lds);
        };
        begin(0);
        int at = 0;
#pragma unroll 1
        for (int64_t s = 0; s < steps; ++s) {
            a.end(lds + at);
            b.end(lds + at + StageA::kBytes);
            __syncthreads();                                 // two tiles: the other one is read no more once all are here
            if (s + 1 < steps) begin(s + 1);
            tile_step<T, kColumns, StageA, StageB>(lds + at, row0, col0, sums, columns, mine);
            at = kBoth - at;
        }
    }
}

// four neighbouring values, `left` of which exist
template <typename O>
__device__ __forceinline__ void store_quad(O *p, v4f x, int left, bool whole)
{
    typedef O v4o __attribute__((ext_vector_type(4)));
    if (whole && left >= 4) {
        v4o r;
#pragma unroll
        for (int k = 0; k < 4; ++k) r[k] = (O)x[k];          // the one rounding to the output's type
        *(v4o *)p = r;
    } else {
        for (int k = 0; k < 4; ++k)
            if (k < left) p[k] = (O)x[k];
    }
}

// Workgroup -> tile: consecutive workgroups go to the eight XCDs in turn, so an XCD takes every eighth one.  Its workgroups are
// numbered in blocks of `rows` x `cols` neighbouring tiles, which share their operands in its L2.
struct TileOrder {
    int32_t rows, cols;                      // of a block, powers of two
    int32_t col_blocks;
    int64_t workgroups;
    __host__ TileOrder(int64_t row_tiles, int32_t col_tiles)
    {
        int32_t block = 32;                  // workgroups that an XCD runs at a time, less where there are not enough for all XCDs
        while (block > 1 && row_tiles * col_tiles < 8 * block) block /= 2;
        rows = cols = 1;
        while (rows < 4 && rows < row_tiles && rows < block) rows *= 2;
        while (rows * cols < block && cols < col_tiles) cols *= 2;
        while (rows * cols < block && rows < row_tiles) rows *= 2;
        block = rows * cols;
        col_blocks = (col_tiles + cols - 1) / cols;
        const int64_t blocks = (row_tiles + rows - 1) / rows * col_blocks;
        workgroups = (blocks + kXcds - 1) / kXcds * kXcds * block;
    }
    __device__ __forceinline__ void find(uint32_t id, int64_t *row_tile, int32_t *col_tile) const
    {
        const uint32_t xcd = id % kXcds, seq = id / kXcds, block = rows * cols;
        const uint32_t b = seq / block * kXcds + xcd, in = seq % block;
        *row_tile = (int64_t)(b / col_blocks) * rows + in % rows;
        *col_tile = (int32_t)(b % col_blocks) * cols + in / rows;
    }
};

}  // namespace groot

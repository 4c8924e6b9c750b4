// Matrix-core tiles shared by the grouped products and the products in 8-bit integers.
//
// Bound, for 256 x 256 tiles of 16-bit types (16384 x 4096 x 4096, bfloat16: 490 us, 1.12 PFLOP/s; a library's product of the size 403):
// the matrix units are busy in 55 % of 0.95 M cycles, at the 1.6 to 2.0 GHz that the power limit leaves; LDS serves reads in 23 % of them,
// without bank conflicts, and 8.9 TB/s come in from L2.  More stages of smaller steps, 4 or 16 wavefronts, 128-wide tiles and
// fragments read earlier were all measured and are within 5 % or slower.
//
// A step of the contraction is 128 bytes of a row whose elements lie along it ("along": 64 values of 16 bits, 32 of fp32,
// 128 of 8 bits), or as many rows of a matrix whose rows lie across it ("across").  Both operands of a step are staged in LDS by loads
// that go there directly (16 bytes a lane, no registers), twice: one pair of tiles is computed while the next one arrives.
// LDS has 64 banks: 16 lanes of a 16-byte read, 32 of an 8-byte and 64 of a 4-byte one are served at a time, if they fall on different
// ones.  So pieces of 16 bytes are kept at other places than their own, by the row that they belong to (swizzle_along / _across):
//   along   the 16 rows that 16 lanes read at one piece cover all places of 256 bytes
//   across  16-bit types: the four rows that a transposing read takes 64 bytes of cover 256 bytes; fp32: the two rows of 128 bytes
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
    static constexpr int kParts = 1;         // instructions that a fragment takes
    // the sum of a fragment's values
    static __device__ __forceinline__ float total(v4i a)
    {
        const v8bf x = __builtin_bit_cast(v8bf, a);
        return (((float)x[0] + (float)x[1]) + ((float)x[2] + (float)x[3])) + (((float)x[4] + (float)x[5]) + ((float)x[6] + (float)x[7]));
    }
    static __device__ __forceinline__ Sum mma(v4i a, v4i b, Sum c, int part)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
    }
};
template <>
struct TileType<f16_t> {
    typedef v16f Sum;
    static constexpr int kParts = 1;
    static __device__ __forceinline__ float total(v4i a)
    {
        const v8h x = __builtin_bit_cast(v8h, a);
        return (((float)x[0] + (float)x[1]) + ((float)x[2] + (float)x[3])) + (((float)x[4] + (float)x[5]) + ((float)x[6] + (float)x[7]));
    }
    static __device__ __forceinline__ Sum mma(v4i a, v4i b, Sum c, int part)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
    }
};
template <>
struct TileType<int8_t> {
    typedef v16i Sum;
    static constexpr int kParts = 1;
    static __device__ __forceinline__ Sum mma(v4i a, v4i b, Sum c, int part) { return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0); }
};
template <>
struct TileType<float> {
    typedef v16f Sum;
    static constexpr int kParts = 4;
    static __device__ __forceinline__ float total(v4i a)
    {
        return (__int_as_float(a[0]) + __int_as_float(a[1])) + (__int_as_float(a[2]) + __int_as_float(a[3]));
    }
    static __device__ __forceinline__ Sum mma(v4i a, v4i b, Sum c, int part)
    {
        return __builtin_amdgcn_mfma_f32_32x32x2f32(__int_as_float(a[part]), __int_as_float(b[part]), c, 0, 0, 0);
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

// 16 bytes of a row from any address p, of which the first `valid` exist (none: 0 or less): where some do not, the row's last 16 bytes
// are loaded in their place, so that no load waits for a branch, and cut16 moves them to their places with zeros behind.  Rows of
// less than 16 bytes (short_row) go value by value.
__device__ __forceinline__ v4i raw16(const char *p, int64_t valid)
{
    v4i x;
    __builtin_memcpy(&x, valid >= 16 ? p : p + (valid - 16), 16);
    return x;
}
__device__ __forceinline__ v4i cut16(v4i x, int64_t valid)
{
    if (valid >= 16) return x;
    if (valid <= 0) return v4i{0, 0, 0, 0};
    return __builtin_bit_cast(v4i, __builtin_bit_cast(unsigned __int128, x) >> (8 * (16 - (int)valid)));
}
template <typename T>
__device__ __forceinline__ v4i short16(const char *p, int64_t valid)
{
    v4i x;
    T e[16 / sizeof(T)] = {};
#pragma unroll
    for (int k = 0; k < (int)(16 / sizeof(T)); ++k)
        if ((int64_t)(k * sizeof(T)) < valid) e[k] = ((const T *)p)[k];
    __builtin_memcpy(&x, e, 16);
    return x;
}
template <typename T>
__device__ __forceinline__ v4i load16(const char *p, int64_t valid, bool short_row)
{
    return short_row ? short16<T>(p, valid) : cut16(raw16(p, valid), valid);
}

// Rows cut to 8 bits: the 16 bytes of a load as floats, their largest magnitude, the scale of a row, its codes.  (A wavefront's
// instruction takes four cycles: 25 a value, with a division each, bound cutting 8192 x 4096 values at 38 us where the bytes take 16.)
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

// Magnitudes compare like their bits without the sign, infinities and NaN above all numbers.  `top`: the largest so far, one value of
// fp32 or two of 16 bits.
template <typename X>
__device__ __forceinline__ uint32_t row_look(v4i v, uint32_t top)
{
    typedef unsigned short u2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (sizeof(X) == 4) {
            const uint32_t a = (uint32_t)v[k] & 0x7FFFFFFFu;
            top = a > top ? a : top;
        } else {
            top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u2, (uint32_t)v[k] & 0x7FFF7FFFu), __builtin_bit_cast(u2, top)));
        }
    }
    return top;
}
// the larger magnitude of two looks, or of one's two halves, as a float
template <typename X>
__device__ __forceinline__ float row_top(uint32_t top)
{
    if constexpr (sizeof(X) == 4) {
        return __uint_as_float(top);
    } else {
        const uint16_t a = (uint16_t)top, b = (uint16_t)(top >> 16), c = a > b ? a : b;
        return (float)__builtin_bit_cast(X, c);
    }
}
// ... over kLanes neighbouring lanes; NaN where a value is not finite
template <int kLanes>
__device__ __forceinline__ float row_top_of(float top)
{
    uint32_t t = __float_as_uint(top);
#pragma unroll
    for (int d = 1; d < kLanes; d *= 2) {
        const uint32_t o = __shfl_xor(t, d);
        t = o > t ? o : t;
    }
    return __uint_as_float(t);
}

__device__ __forceinline__ float row_scale(float top) { return __builtin_isfinite(top) ? top * (1.f / 127.f) : __builtin_nanf(""); }

// The codes of a load: x / scale, halves to even; zeros where the scale is zero or NaN.
template <typename X>
__device__ __forceinline__ void row_codes(v4i v, float scale, int8_t *to)
{
    constexpr int kPer = 16 / sizeof(X);
    constexpr float kRound = 12582912.f;                     // 1.5 * 2^23: what is added to it is rounded to an integer
    const RowValues<X> e = row_values<X>(v);
    uint32_t q[kPer];
    if (scale > 0x1p-96f) {                                  // the same for a row
        const float r = 1.f / scale;
#pragma unroll
        for (int k = 0; k < kPer; ++k) q[k] = __float_as_uint(quotient(e.x[k], scale, r) + kRound);
    } else {
#pragma unroll
        for (int k = 0; k < kPer; ++k) q[k] = scale > 0.f ? (uint32_t)(int)fminf(fmaxf(rintf(e.x[k] / scale), -127.f), 127.f) : 0u;
    }
    uint32_t u[kPer / 4];
#pragma unroll
    for (int k = 0; k < kPer / 4; ++k)
        u[k] = (q[4 * k] & 0xFFu) | (q[4 * k + 1] & 0xFFu) << 8 | (q[4 * k + 2] & 0xFFu) << 16 | q[4 * k + 3] << 24;
    __builtin_memcpy(__builtin_assume_aligned(to, kPer), u, kPer);
}

// row r of kStepBytes
__device__ __forceinline__ int swizzle_along(int r) { return r / 2 & 7; }
// row k of kRowBytes
template <typename T, int kRowBytes>
__device__ __forceinline__ int swizzle_across(int k)
{
    return sizeof(T) == 4 ? (k / 4 & 1) << 3 : kRowBytes == 128 ? (k / 2 & 1) << 2 : (k & 3) << 2;
}

// One operand's tile: kWide rows ("along") or columns ("across").  begin(s) starts the loads of step s, end(s) has them in LDS once
// the workgroup has passed a barrier.
template <typename T, int kWide, int kThreads, bool kAcross, bool kAligned>
struct Stage {
    static constexpr bool kDirect = kAligned;
    static constexpr int kBytes = kWide * kStepBytes, kValues = kStepBytes / (int)sizeof(T), kSubSteps = kStepBytes / 32, kEach = kBytes / 16 / kThreads;
    static constexpr int kRowBytes = kAcross ? kWide * (int)sizeof(T) : kStepBytes, kPieces = kRowBytes / 16;
    static constexpr int kRowsEach = kThreads / kPieces;     // rows of the tile that one load of the workgroup takes
    static_assert(kBytes % (16 * kThreads) == 0 && kThreads % kPieces == 0, "a whole number of loads of whole rows");
    static_assert(kAcross ? kRowsEach % (sizeof(T) == 4 ? 8 : 4) == 0 && kRowBytes >= (sizeof(T) == 4 ? 256 : 128) : kRowsEach % 16 == 0, "a lane's piece is the same in all its loads");

    // what is on its way through registers where rows begin anywhere, and how much of it exists
    struct Held {
        v4i x[kEach];
        int32_t valid[kEach];
    };

    const char *src[kAcross ? 1 : kEach];
    int64_t pitch, limit;                                    // bytes between rows; bytes ("along") or rows ("across") of the contraction
    int64_t width;                                           // across: bytes of a row from the lane's piece on
    int32_t piece, row;
    bool short_row;

    static __device__ __forceinline__ int swizzle(int r)
    {
        return kAcross ? swizzle_across<T, kRowBytes>(r) : swizzle_along(r);
    }

    // along: `base` is the first row's first value, `exist` rows exist, `extent` values of the contraction
    // across: `base` is the first value of the tile's first column in the contraction's first row, `exist` columns exist from there on
    // row_values: of a whole row
    __device__ __forceinline__ void init(const T *base, int64_t stride, int64_t exist, int64_t extent, int64_t row_values)
    {
        short_row = row_values * (int64_t)sizeof(T) < 16;
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

    // where a lane's load i of step s begins, and how many bytes of its row are left there (none: 0 or less)
    __device__ __forceinline__ const char *place(int64_t s, int i, int64_t *left) const
    {
        if constexpr (kAcross) {
            const int64_t k = s * kValues + row + i * kRowsEach;
            const char *p = src[0] + (s * kValues + i * kRowsEach) * pitch;
            *left = k < limit ? width : 0;
            if (!kAligned && k >= limit) p += (limit - 1 - k) * pitch + width;   // behind the end of the last row
            return p;
        } else {
            *left = limit - s * kStepBytes - piece * 16;
            return src[i] + s * kStepBytes;
        }
    }
    // direct: the loads [first, last) of a lane's kEach, zeros for what does not exist
    __device__ __forceinline__ void begin(int64_t s, char *tile, int first = 0, int last = kEach) const
    {
        const uint32_t to = lds_offset(tile) + threadIdx.x / kWave * (kWave * 16);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if (i < first || i >= last) continue;
            int64_t left;
            const char *p = place(s, i, &left);
            // across, a piece past the last column has the last column's place: only the row decides
            const bool in = kAcross ? s * kValues + row + i * kRowsEach < limit : left > 0;
            dma16(in ? p : (const char *)&g_zeros, to + i * (kThreads * 16));
        }
    }
    // through registers
    template <bool kShort>
    __device__ __forceinline__ void load(int64_t s, Held &h) const
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            int64_t left;
            const char *p = place(s, i, &left);
            h.valid[i] = left >= 16 ? 16 : left <= 0 ? 0 : (int32_t)left;
            h.x[i] = kShort && short_row ? short16<T>(p, left) : raw16(p, left);
        }
    }
    template <bool kShort>
    __device__ __forceinline__ void put(const Held &h, char *tile) const
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            *(v4i *)(tile + (i * kThreads + threadIdx.x) * 16) = kShort && short_row ? h.x[i] : cut16(h.x[i], h.valid[i]);
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
            for (int j = 0; j < 4; ++j) {
                const int k = 8 * s + 4 * half + j, c = (first + lane % 32) / 4;
                x[j] = *(const int *)(tile + k * kRowBytes + ((c ^ swizzle(k)) * 16) + lane % 4 * 4);
            }
            return x;
        }
    }
};

// The fragments of one sub-step of the wavefront's blocks, and their products.
template <typename T, class StageA, class StageB, int kI, int kJ>
struct Fragments {
    v4i a[kI], b[kJ];

    __device__ __forceinline__ void read(const char *tile, int row0, int col0, int q)
    {
#pragma unroll
        for (int j = 0; j < kJ; ++j) b[j] = StageB::fragment(tile + StageA::kBytes, col0 + 32 * j, q);
#pragma unroll
        for (int i = 0; i < kI; ++i) a[i] = StageA::fragment(tile, row0 + 32 * i, q);
    }
    // the first or second half of the products (0, 1): instructions that follow one another add to different blocks
    __device__ __forceinline__ void multiply(typename TileType<T>::Sum (&sums)[kI][kJ], int half) const
    {
        constexpr int kBlocks = kI * kJ, kAll = kBlocks * TileType<T>::kParts;
#pragma unroll
        for (int n = 0; n < kAll; ++n) {
            if (n < half * kAll / 2 || n >= (half + 1) * kAll / 2) continue;
            const int i = n % kBlocks / kJ, j = n % kJ;
            sums[i][j] = TileType<T>::mma(b[j], a[i], sums[i][j], n / kBlocks);
        }
    }
    __device__ __forceinline__ void add_columns(float (&columns)[kJ]) const
    {
#pragma unroll
        for (int j = 0; j < kJ; ++j) columns[j] += TileType<T>::total(b[j]);
    }
};

// ... of operands that go through registers: kSets steps are on their way in them, two tiles lie in LDS.  More of them pay where a CU
// has few small tiles (2000 rows, K = 3001, N = 301: 51 us with one, 34 with more); elsewhere the registers cost wavefronts.
template <typename T, bool kColumns, bool kShort, class StageA, class StageB, int kI, int kJ>
__device__ __forceinline__ void tile_product_held(const StageA &a, const StageB &b, char *lds, int64_t steps, int row0, int col0,
                                                  typename TileType<T>::Sum (&sums)[kI][kJ], float (*columns)[kJ], bool mine)
{
    constexpr int kBoth = StageA::kBytes + StageB::kBytes, kSets = kShort || kColumns || kI * kJ > 1 ? 1 : 2;
    typename StageA::Held ha[kSets];
    typename StageB::Held hb[kSets];
    Fragments<T, StageA, StageB, kI, kJ> f;
#pragma unroll
    for (int u = 0; u < kSets; ++u) {                        // a step past the last one loads the ends of rows, which nothing reads
        a.template load<kShort>(u, ha[u]);
        b.template load<kShort>(u, hb[u]);
    }
    int at = 0;
#pragma unroll 1
    for (int64_t s0 = 0; s0 < steps; s0 += kSets) {
#pragma unroll
        for (int u = 0; u < kSets; ++u) {
            if (s0 + u >= steps) break;
            a.template put<kShort>(ha[u], lds + at);
            b.template put<kShort>(hb[u], lds + at + StageA::kBytes);
            __syncthreads();                                 // two tiles: the other one is read no more once all are here
            a.template load<kShort>(s0 + u + kSets, ha[u]);
            b.template load<kShort>(s0 + u + kSets, hb[u]);
#pragma unroll
            for (int q = 0; q < StageA::kSubSteps; ++q) {
                f.read(lds + at, row0, col0, q);
                f.multiply(sums, 0);
                f.multiply(sums, 1);
                if constexpr (kColumns)
                    if (mine) f.add_columns(*columns);
            }
            at = kBoth - at;
        }
    }
}

// The product of two staged operands over `steps` steps: sums[i][j] of the wavefront's 32 x 32 blocks, rows of `A` from row0 on,
// columns of `B` from col0 on.  kStages pairs of tiles lie in LDS, so that kStages - 1 steps are on their way while one is computed.
// The fragments of a sub-step are read while the one before is multiplied, across the steps' borders too: the barrier lies before the
// last sub-step's products, whose fragments are in registers by then.
// `columns` (where kColumns; wavefronts with `mine`): the sums of B's values, lanes l and l + 32 hold the two halves of column l.
template <typename T, int kStages, bool kColumns = false, class StageA, class StageB, int kI, int kJ>
__device__ __forceinline__ void tile_product(StageA &a, StageB &b, char *lds, int64_t steps, int row0, int col0,
                                             typename TileType<T>::Sum (&sums)[kI][kJ], float (*columns)[kJ] = nullptr, bool mine = false)
{
    constexpr int kBoth = StageA::kBytes + StageB::kBytes, kQ = StageA::kSubSteps;
    static_assert(kQ % 2 == 0, "the two sets of fragments take turns");
#pragma unroll
    for (int i = 0; i < kI; ++i)
#pragma unroll
        for (int j = 0; j < kJ; ++j) sums[i][j] = {};
    if (steps <= 0) return;
    if constexpr (StageA::kDirect) {
        Fragments<T, StageA, StageB, kI, kJ> f[2];
        // a step past the last one loads zeros that nothing reads: every step has the same number of loads to count
        constexpr int kEach = StageA::kEach + StageB::kEach;
        auto begin = [&](int64_t s, int at, int first, int last) {
            a.begin(s, lds + at, first, last);
            b.begin(s, lds + at + StageA::kBytes, first - StageA::kEach, last - StageA::kEach);
        };
#pragma unroll
        for (int s = 0; s < kStages - 1; ++s) begin(s, s * kBoth, 0, kEach);
        int now = 0, free = (kStages - 1) * kBoth;           // the tiles that are read, and those that are loaded next
        dma_wait<(kStages - 2) * kEach>();
        __syncthreads();
        f[0].read(lds, row0, col0, 0);
#pragma unroll 1
        for (int64_t s = 0; s < steps; ++s) {
#pragma unroll
            for (int q = 0; q < kQ; ++q) {
                // the loads are issued between the products, half at a time: all at once they hold the wavefront up (2 to 3 % of a
                // 256 x 256 tile), later ones arrive too late where there are two stages
                if (q + 1 < kQ) f[(q + 1) % 2].read(lds + now, row0, col0, q + 1);
                __builtin_amdgcn_sched_barrier(0);
                f[q % 2].multiply(sums, 0);
                __builtin_amdgcn_sched_barrier(0);
                constexpr int kSpread = kStages == 2 ? 2 : kQ;
                if (q < kSpread) begin(s + kStages - 1, free, q * kEach / kSpread, (q + 1) * kEach / kSpread);
                if (q + 1 == kQ && s + 1 < steps) {
                    free = now;
                    now = now + kBoth == kStages * kBoth ? 0 : now + kBoth;
                    dma_wait<(kStages - 2) * kEach>();
                    __syncthreads();                         // the next step has arrived, and nobody reads the tiles of this one
                    f[0].read(lds + now, row0, col0, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
                f[q % 2].multiply(sums, 1);
                if constexpr (kColumns)
                    if (mine) f[q % 2].add_columns(*columns);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        dma_wait();                                          // before the workgroup's LDS is anybody else's
    } else {
        if (a.short_row || b.short_row) tile_product_held<T, kColumns, true>(a, b, lds, steps, row0, col0, sums, columns, mine);
        else tile_product_held<T, kColumns, false>(a, b, lds, steps, row0, col0, sums, columns, mine);
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
